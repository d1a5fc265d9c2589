"""The text-side operators whose speed is measured, in their plain form and
through `paper_2605_08835_amd.ops`.

A denoiser that serves requests with texts of their own lengths normalises
encoder states and tokens (`rmsnorm`, optionally with the residual's addition
and an 8-bit output), sends a few rows per request through layers whose cost
is their weights (`linear_rows_w4`), and attends from image tokens, or from
one pooled token, to each request's own text (`cross_attention`).

Case kinds and their values:
  norm   rows x C; dt: type of x, the sum and (unless fp8) y; resid: x + resid
         is normed and returned; fp8: y leaves as e4m3 with one scale per
         `group` channels (0: per row)
  w4     m x k times n x k codes in groups of `group`, scales of type st, with
         `zero` points or without; xt: type of x (f32, bf16, e4m3 with a scale
         per `xgroup` channels, 0: per row); silu on the way in / out; add; ot:
         type of the output
  attn   n rows of nq queries, heads / kvh heads of width d, texts of lo..hi
         tokens; `pad`: texts in one padded [n_ctx, hi] array, else packed one
         after another; `mask`: keys switched off inside the texts; `guided`: the last n // 3
         rows read one shared text
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "e4m3": 1}
_ops = None


def _own_ops():
    global _ops
    if _ops is None:
        from paper_2605_08835_amd import ops
        _ops = ops
    return _ops


def _norm(**kw):
    return dict(dict(kind="norm", dt="bf16", resid=False, fp8=False, group=0), **kw)


def _w4(**kw):
    return dict(dict(kind="w4", group=128, st="bf16", zero=False, xt="bf16", xgroup=0, silu_in=False, silu_out=False,
                     add=False, ot="bf16"), **kw)


def _attn(**kw):
    return dict(dict(kind="attn", dt="bf16", pad=False, mask=False, guided=False), **kw)


def listed():
    return [
        # one pooled token of one request, with the block's residual: latency
        _norm(name="norm_one_row", rows=1, c=1280, dt="f32", resid=True),
        # encoder states of 48 ragged texts on the way to 8-bit products
        _norm(name="norm_states_8bit", rows=12301, c=1280, resid=True, fp8=True, group=128),
        # the 64x64 level's tokens of a full 48-row batch
        _norm(name="norm_image_tokens", rows=196608, c=320, resid=True),
        # the time embedding's first layer for a lone request: latency
        _w4(name="w4_time_mlp", m=1, k=320, n=1280, group=64, st="f32", xt="f32", silu_out=True, ot="f32"),
        # the added embedding of 7 requests from 8-bit inputs, with zero points and a residual
        _w4(name="w4_added_embedding", m=7, k=2816, n=1280, group=32, zero=True, xt="e4m3", xgroup=128, add=True),
        # every ResBlock's time projection for 32 requests
        _w4(name="w4_time_projections", m=32, k=1280, n=20160, xt="f32", silu_in=True, ot="f32"),
        # a wide square layer, 16 rows
        _w4(name="w4_wide", m=16, k=8192, n=8192),
        # one pooled query per request over its own text, shared K/V heads: latency
        _attn(name="attn_pooled", n=9, nq=1, heads=16, kvh=4, d=64, lo=3, hi=231),
        # one query over long documents, packed one after another
        _attn(name="attn_one_query_long", n=4, nq=1, heads=20, kvh=20, d=64, lo=9000, hi=16384),
        # the 64x64 level's tokens of 48 rows over texts of up to 77 tokens, the unguided rows on one null text
        _attn(name="attn_image_tokens", n=48, nq=4096, heads=8, kvh=8, d=40, lo=5, hi=77, guided=True),
        # 64-wide heads over long padded prompts with padding masked out
        _attn(name="attn_long_prompts", n=16, nq=1024, heads=20, kvh=20, d=64, lo=200, hi=512, pad=True, mask=True),
        # the reference-precision path
        _attn(name="attn_fp32", n=6, nq=1024, heads=8, kvh=4, d=32, lo=8, hi=231, dt="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "w4", "attn"])
    if kind == "norm":
        c = rng.choice([_log(rng, 8, 8192), 8 * _log(rng, 1, 1024)])
        fp8 = rng.random() < 0.4
        dt = rng.choice(["bf16", "bf16", "f32"])
        rows = min(_log(rng, 1, 200000), 120000000 // SIZE[dt] // c)
        return _norm(rows=rows, c=c, dt=dt, resid=rng.random() < 0.6, fp8=fp8,
                     group=rng.choice([0, 128]) if fp8 else 0)
    if kind == "w4":
        k, n = 8 * _log(rng, 8, 1280), _log(rng, 16, 20160)
        k = min(k, 64000000 // n // 8 * 8)
        xt = rng.choice(["bf16", "bf16", "f32", "e4m3"])
        return _w4(m=_log(rng, 1, 64), k=k, n=n, group=rng.choice([32, 64, 128]), st=rng.choice(["bf16", "f32"]),
                   zero=rng.random() < 0.5, xt=xt, xgroup=rng.choice([0, 128]) if xt == "e4m3" else 0,
                   silu_in=xt != "e4m3" and rng.random() < 0.3, silu_out=rng.random() < 0.3, add=rng.random() < 0.3,
                   ot=rng.choice(["bf16", "f32"]))
    dt = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kvh, rep = rng.choice([1, 2, 4, 5, 8, 10]), rng.choice([1, 1, 1, 2, 3, 4, 8])
    d = 8 * rng.choice([2, 4, 5, 8, 8, 10, 12, 16, 20, 32])
    few = rng.random() < 0.4
    nq = rng.choice([1, 1, 2, _log(rng, 2, 40)]) if few else _log(rng, 48, 6144)
    hi = _log(rng, 1, 20000) if few else _log(rng, 4, 700)
    heads = kvh * rep
    flops = 4.0 * nq * hi * heads * d * (4 if dt == "f32" else 1)
    n = max(1, min(_log(rng, 1, 48), int(2.4e10 / flops), int(1.2e8 / (nq * heads * hi)), int(8e7 / (hi * kvh * d)),
                   int(6e7 / (nq * heads * d))))
    return _attn(n=n, nq=nq, heads=heads, kvh=kvh, d=d, lo=rng.randint(0, hi), hi=hi, dt=dt, pad=rng.random() < 0.4,
                 mask=rng.random() < 0.4, guided=n > 2 and rng.random() < 0.4)


# ------------------------------------------------------------------ inputs
def _texts(case):
    """(contexts, shared context or None) of an attn case."""
    n = case["n"]
    own_texts = n - n // 3 if case["guided"] else n
    return own_texts + 1 if case["guided"] else own_texts


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    if case["kind"] == "norm":
        t = TYPES[case["dt"]]
        s = dict(case=case, x=(0.3 + r(case["rows"], case["c"])).to(t), gamma=1 + 0.2 * r(case["c"]))
        # a residual stream grows from block to block and has a few large channels
        s["resid"] = (4 * r(case["rows"], case["c"]) * (1 + r(case["c"]).abs())).to(t) if case["resid"] else None
        return s
    if case["kind"] == "w4":
        m, k, n, G = case["m"], case["k"], case["n"], case["group"]
        ng = -(-k // G)
        s = dict(case=case, w=torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8))
        s["scale"] = ((0.5 + torch.rand(n, ng, generator=g, device=DEV)) * 0.2 / math.sqrt(k)).to(TYPES[case["st"]])
        s["zero"] = torch.randint(5, 11, (n, ng), generator=g, device=DEV, dtype=torch.uint8) if case["zero"] else None
        x = r(m, k)
        s["x_scale"] = None
        if case["xt"] == "e4m3":
            xg = case["xgroup"] or k
            top = torch.nn.functional.pad(x.abs(), (0, -k % xg)).view(m, -1, xg).amax(2)
            s["x_scale"] = top / 448
            x = x / s["x_scale"].repeat_interleave(xg, 1)[:, :k]
        s["x"] = x.to(TYPES[case["xt"]])
        s["bias"] = 0.1 * r(n)
        s["add"] = r(m, n) if case["add"] else None
        return s
    n, nq, heads, kvh, d, hi = (case[i] for i in ("n", "nq", "heads", "kvh", "d", "hi"))
    t, nc = TYPES[case["dt"]], _texts(case)
    length = torch.randint(case["lo"], hi + 1, (nc,), generator=g, device=DEV, dtype=torch.int32)
    length[0] = hi
    # K and V come from one projection of the texts: two halves of each row
    tokens = nc * hi if case["pad"] else int(length.sum())
    kv = r(tokens, 2, kvh, d).to(t)
    s = dict(case=case, q=(1.5 * r(n, nq, heads, d)).to(t), kv_len=length, max_len=hi)
    if case["pad"]:
        s["k"], s["v"], s["kv_start"] = (*kv.view(nc, hi, 2, kvh, d).unbind(2), None)
    else:
        s["k"], s["v"] = kv.unbind(1)
        s["kv_start"] = (length.cumsum(0) - length).to(torch.int32)
    s["mask"] = None
    if case["mask"]:
        keep = torch.rand(tokens, generator=g, device=DEV) > 0.15
        s["mask"] = keep.view(nc, hi) if case["pad"] else keep
    s["kv_index"] = None
    if case["guided"]:
        s["kv_index"] = torch.arange(n, device=DEV, dtype=torch.int32).clamp_(max=nc - 1)
    return s


# ------------------------------------------------------------------ passes
def run(s):
    case = s["case"]
    if own:
        ops = _own_ops()
        if case["kind"] == "norm":
            return ops.rmsnorm(s["x"], s["gamma"], 1e-6, resid=s["resid"], fp8=case["fp8"], scale_group=case["group"])
        if case["kind"] == "w4":
            return ops.linear_rows_w4(s["x"], s["w"], s["scale"], case["group"], zero=s["zero"], x_scale=s["x_scale"],
                                      bias=s["bias"], add=s["add"], silu_in=case["silu_in"], silu_out=case["silu_out"],
                                      out_dtype=TYPES[case["ot"]])
        return ops.cross_attention(s["q"], s["k"], s["v"], s["max_len"], kv_start=s["kv_start"], kv_len=s["kv_len"],
                                   kv_index=s["kv_index"], mask=s["mask"])
    return {"norm": _plain_norm, "w4": _plain_w4, "attn": _plain_attn}[case["kind"]](case, s)


def _plain_norm(case, s):
    x, t = s["x"].float(), s["x"].dtype
    h = x + s["resid"].float() if case["resid"] else x
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6) * s["gamma"]
    if not case["fp8"]:
        return (y.to(t), h.to(t)) if case["resid"] else y.to(t)
    rows, c = y.shape
    G = case["group"] or c
    z = torch.zeros(rows, -(-c // G) * G, device=y.device)
    z[:, :c] = y
    z = z.view(rows, -1, G)
    scale = z.abs().amax(2).clamp(min=2.0 ** -100) / 448
    q = (z / scale[:, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(rows, -1)[:, :c]
    return (q, scale, h.to(t)) if case["resid"] else (q, scale)


def _plain_w4(case, s):
    m, k, n, G = case["m"], case["k"], case["n"], case["group"]
    x = s["x"].float()
    if s["x_scale"] is not None:
        x = x * s["x_scale"].repeat_interleave(case["xgroup"] or k, 1)[:, :k]
    if case["silu_in"]:
        x = x / (1 + torch.exp(-x))
    q = torch.stack((s["w"] & 15, s["w"] >> 4), 2).view(n, k).float()
    q = q - (s["zero"].float().repeat_interleave(G, 1)[:, :k] if case["zero"] else 8.0)
    w = q * s["scale"].float().repeat_interleave(G, 1)[:, :k]
    y = x @ w.t() + s["bias"]
    if case["add"]:
        y = y + s["add"]
    if case["silu_out"]:
        y = y / (1 + torch.exp(-y))
    return y.to(TYPES[case["ot"]])


def _keys(case, s):
    """Row of K / V of key t of each row's text, and whether it takes part: [n, hi]."""
    n, hi = case["n"], case["hi"]
    ctx = s["kv_index"].long() if s["kv_index"] is not None else torch.arange(n, device=s["q"].device)
    t = torch.arange(hi, device=s["q"].device)
    start = ctx * hi if case["pad"] else s["kv_start"].long()[ctx]
    live = t < s["kv_len"][ctx][:, None]
    at = (start[:, None] + t) * live
    if s["mask"] is not None:
        live = live & s["mask"].reshape(-1)[at]
    return at, live


def _plain_attn(case, s):
    n, nq, heads, kvh, d, hi = (case[i] for i in ("n", "nq", "heads", "kvh", "d", "hi"))
    rep = heads // kvh
    at, live = _keys(case, s)
    k = s["k"].reshape(-1, kvh, d)[at].float().permute(0, 2, 3, 1).contiguous()  # [n, kvh, d, hi]
    v = s["v"].reshape(-1, kvh, d)[at].float().masked_fill(~live[:, :, None, None], 0).transpose(1, 2).contiguous()
    q = s["q"].float().view(n, nq, kvh, rep, d).permute(0, 2, 3, 1, 4).reshape(n, kvh, rep * nq, d)
    a = (q @ k / math.sqrt(d)).masked_fill(~live[:, None, None, :], -math.inf)
    top = a.amax(3, keepdim=True)
    p = torch.exp(a - top.masked_fill(top == -math.inf, 0))
    total = p.sum(3, keepdim=True)
    o = p @ v / total.masked_fill(total == 0, 1)
    return o.view(n, kvh, rep, nq, d).permute(0, 3, 1, 2, 4).reshape(n, nq, heads, d).to(s["q"].dtype)


# ------------------------------------------------------------------ work
def work(case):
    if case["kind"] == "norm":
        e, b = float(case["rows"]) * case["c"], SIZE[case["dt"]]
        out = e + 4.0 * case["rows"] * (-(-case["c"] // (case["group"] or case["c"]))) if case["fp8"] else e * b
        return {"bytes": e * b * (3 if case["resid"] else 1) + out + 4 * case["c"], "flops": 5 * e}
    if case["kind"] == "w4":
        m, k, n = case["m"], case["k"], case["n"]
        ng = -(-k // case["group"])
        x = m * k * SIZE[case["xt"]] + (4 * m * (-(-k // case["xgroup"]) if case["xgroup"] else 1) if case["xt"] == "e4m3" else 0)
        return {"bytes": n * k / 2 + n * ng * (SIZE[case["st"]] + int(case["zero"])) + x + 4 * n
                + m * n * (SIZE[case["ot"]] + 4 * int(case["add"])), "flops": 2.0 * m * n * k}
    n, nq, heads, kvh, d = (case[i] for i in ("n", "nq", "heads", "kvh", "d"))
    b, nc = SIZE[case["dt"]], _texts(case)
    mean = (case["lo"] + case["hi"]) / 2  # lengths are drawn evenly
    kept = 0.85 if case["mask"] else 1.0
    tokens = (nc - 1) * mean + case["hi"]
    return {"bytes": 2.0 * n * nq * heads * d * b + 2 * tokens * kept * kvh * d * b + tokens * int(case["mask"]) + 8 * nc,
            "flops": 4.0 * n * nq * heads * d * mean * kept}


# ------------------------------------------------------------------ 64 bits
def _e4m3(v):
    """v rounded to the nearest e4m3 value, ties to the even one, in 64 bits: steps of 2^(e - 3) from 2^e on, 2^-9 below 2^-6."""
    e = torch.frexp(v.abs().clamp(min=2.0 ** -6))[1].double() - 1
    step = torch.exp2(e - 3)
    return torch.round(v / step) * step


def _exact_norm(case, s):
    parts = []
    for a in range(0, case["rows"], 1 << 15):  # a slice of rows at a time
        h = s["x"][a:a + (1 << 15)].double()
        if case["resid"]:
            h = h + s["resid"][a:a + (1 << 15)].double()
        norm = torch.sqrt(h.square().sum(1) / case["c"] + 1e-6)
        y = h / norm[:, None] * s["gamma"].double()
        if not case["fp8"]:
            parts.append((y, h))
            continue
        G, qs, scales = case["group"] or case["c"], [], []
        for c in range(0, case["c"], G):
            piece = y[:, c:c + G]
            sc = torch.clamp(piece.abs().max(1).values, min=2.0 ** -100) / 448.0
            scales.append(sc)
            qs.append(_e4m3(piece / sc[:, None]))
        parts.append((torch.cat(qs, 1), torch.stack(scales, 1), h))
    whole = [torch.cat(p) for p in zip(*parts)]
    if not case["resid"]:
        whole = whole[:-1]
    return whole[0] if len(whole) == 1 else tuple(whole)


def _exact_w4(case, s):
    m, k, n, G = case["m"], case["k"], case["n"], case["group"]
    y = s["bias"].double().repeat(m, 1)
    if case["add"]:
        y += s["add"].double()
    x = s["x"].double()
    if case["xt"] == "e4m3":
        x = x * s["x_scale"].double()[:, torch.arange(k, device=DEV) // (case["xgroup"] or k)]
    if case["silu_in"]:
        x = x * torch.sigmoid(x)
    even, odd = x[:, 0::2], x[:, 1::2]
    for j, a in enumerate(range(0, k, G)):  # group by group: the products of the codes, then the group's scale
        codes = s["w"][:, a // 2:(a + G) // 2]
        part = even[:, a // 2:(a + G) // 2] @ (codes % 16).double().t() + odd[:, a // 2:(a + G) // 2] @ (codes // 16).double().t()
        z = s["zero"][:, j].double() if case["zero"] else torch.full((n,), 8.0, device=DEV, dtype=torch.float64)
        y += (part - x[:, a:a + G].sum(1)[:, None] * z) * s["scale"][:, j].double()
    return y * torch.sigmoid(y) if case["silu_out"] else y


def _exact_attn(case, s):
    rep = case["heads"] // case["kvh"]
    out = torch.zeros(case["n"], case["nq"], case["heads"], case["d"], device=DEV, dtype=torch.float64)
    lens = s["kv_len"].tolist()
    starts = [c * case["hi"] for c in range(len(lens))] if case["pad"] else s["kv_start"].tolist()
    ks, vs = s["k"].reshape(-1, case["kvh"], case["d"]), s["v"].reshape(-1, case["kvh"], case["d"])
    for i in range(case["n"]):  # row by row, only the keys that take part
        c = int(s["kv_index"][i]) if case["guided"] else i
        rows = torch.arange(starts[c], starts[c] + lens[c], device=DEV)
        if case["mask"]:
            rows = rows[s["mask"].reshape(-1)[rows]]
        if not len(rows):
            continue
        k, v = ks[rows].double(), vs[rows].double()
        for g in range(case["kvh"]):
            q = s["q"][i, :, g * rep:(g + 1) * rep].double().reshape(-1, case["d"])
            p = torch.softmax(q @ k[:, g].t().contiguous() / math.sqrt(case["d"]), 1)
            out[i, :, g * rep:(g + 1) * rep] = (p @ v[:, g].contiguous()).view(case["nq"], rep, case["d"])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "w4": _exact_w4, "attn": _exact_attn}[case["kind"]](case, s)
