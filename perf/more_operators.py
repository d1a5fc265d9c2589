"""Two more operators whose speed is measured, in their plain form and through
`paper_2605_08835_amd.ops`.

Before its texts reach the denoiser they pass an encoder, whose layers attend
inside each text (`text_attention`), and requests of one batch bring styles of
their own: low-rank additions to projections that all of them share
(`linear_adapters`).

Case kinds and their values:
  text   n texts of lo..hi tokens, heads / kvh heads of width d; `pad`: padded
         [n, hi] arrays, else packed one after another; `mask`: keys switched
         off inside the texts; `causal`: keys up to the query only; `prefix`:
         and the first 0..hi // 2 keys of each text for all; `cap`: scores
         pass cap tanh(s / cap) (0: not); `reach`: a bias per head and
         distance up to so far, constant past it (0: none); `slope`: a penalty
         per head that grows with the distance
  lora   n x t rows of k channels times n_out x k weights, plus one of `na`
         adapters of rank r per x[i] (`ragged`: n runs of 1..t packed rows,
         an adapter per row), none for every `bare`-th
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
_ops = None


def _own_ops():
    global _ops
    if _ops is None:
        from paper_2605_08835_amd import ops
        _ops = ops
    return _ops


def _text(**kw):
    return dict(dict(kind="text", dt="bf16", pad=False, mask=False, causal=False, prefix=False, cap=0.0, reach=0,
                     slope=False), **kw)


def _lora(**kw):
    return dict(dict(kind="lora", dt="bf16", ragged=False, bare=0), **kw)


def listed():
    return [
        # the prompt of a lone request in a causal encoder: latency
        _text(name="text_one_prompt", n=1, lo=77, hi=77, heads=12, kvh=12, d=64, causal=True),
        # the prompts of a full batch, packed
        _text(name="text_prompts", n=48, lo=5, hi=77, heads=20, kvh=20, d=64, causal=True),
        # long padded prompts in an encoder with a bias per distance, padding masked out
        _text(name="text_distance_bias", n=16, lo=200, hi=512, heads=20, kvh=20, d=64, pad=True, mask=True, reach=128),
        # documents read by a causal model with capped scores and shared K/V heads
        _text(name="text_documents_capped", n=6, lo=500, hi=8192, heads=16, kvh=4, d=128, causal=True, cap=50.0),
        # instructions that all tokens see, the rest causal, far tokens penalised
        _text(name="text_prefix_slope", n=12, lo=700, hi=2500, heads=10, kvh=5, d=80, causal=True, prefix=True, slope=True),
        # the reference-precision path
        _text(name="text_fp32", n=6, lo=8, hi=231, heads=8, kvh=4, d=32, dt="f32", causal=True, cap=30.0, reach=16),
        # one pooled row of one request with its style: latency
        _lora(name="lora_one_row", n=1, t=1, k=1280, n_out=1280, na=4, r=16),
        # 32 requests' time embeddings, a style each
        _lora(name="lora_rows", n=32, t=1, k=1280, n_out=1280, na=32, r=32),
        # K of the texts of a full batch, packed, some requests without a style
        _lora(name="lora_texts", n=48, t=77, k=768, n_out=640, na=8, r=16, ragged=True, bare=5),
        # the 64x64 level's tokens of a 48-row batch
        _lora(name="lora_image_tokens", n=48, t=4096, k=320, n_out=320, na=6, r=16, bare=4),
        # the 32x32 level's wide layer, 16 rows, high ranks
        _lora(name="lora_wide", n=16, t=1024, k=1280, n_out=5120, na=9, r=128),
        # the reference-precision path
        _lora(name="lora_fp32", n=6, t=1024, k=320, n_out=320, na=3, r=8, dt="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        dt = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kvh, rep = rng.choice([1, 2, 4, 5, 8, 12, 20]), rng.choice([1, 1, 1, 2, 4])
        d = 8 * rng.choice([4, 5, 8, 8, 8, 10, 12, 16, 16, 20, 32])
        hi = _log(rng, 1, 8192)
        heads = kvh * rep
        causal = rng.random() < 0.6
        flops = 4.0 * hi * hi * heads * d * (8 if dt == "f32" else 1)
        n = max(1, min(_log(rng, 1, 64), int(3e11 / flops), int(2e9 / (heads * hi * hi)), int(1e8 / (hi * heads * d))))
        return _text(n=n, lo=rng.randint(0, hi), hi=hi, heads=heads, kvh=kvh, d=d, dt=dt, pad=rng.random() < 0.4,
                     mask=rng.random() < 0.4, causal=causal, prefix=causal and rng.random() < 0.4,
                     cap=rng.choice([0.0, 0.0, 20.0, 50.0]), reach=rng.choice([0, 0, _log(rng, 1, 1000)]),
                     slope=rng.random() < 0.25)
    dt = rng.choice(["bf16", "bf16", "bf16", "f32"])
    few = rng.random() < 0.4
    t = 1 if few else _log(rng, 2, 6000)
    n = _log(rng, 1, 64)
    k, n_out = 8 * rng.choice([_log(rng, 4, 640), 8 * _log(rng, 1, 80)]), 8 * rng.choice([_log(rng, 2, 640), 8 * _log(rng, 1, 80)])
    n = max(1, min(n, int(6e10 / (2.0 * t * k * n_out * (4 if dt == "f32" else 1))), int(6e7 / (t * max(k, n_out)))))
    return _lora(n=n, t=t, k=k, n_out=n_out, na=rng.randint(1, n + 3), r=8 * rng.choice([1, 1, 2, 2, 3, 4, 8, 16]), dt=dt,
                 ragged=t > 1 and rng.random() < 0.4, bare=rng.choice([0, 0, 1, 2, 5]))


# ------------------------------------------------------------------ inputs
def _lengths(n, lo, hi):
    """n lengths spread evenly over lo..hi, hi among them; the seed orders them."""
    return [hi - (hi - lo) * i // max(n - 1, 1) for i in range(n)]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    t = TYPES[case["dt"]]
    n = case["n"]
    if case["kind"] == "lora":
        k, n_out, na, rank = case["k"], case["n_out"], case["na"], case["r"]
        index = torch.randint(0, na, (n,), generator=g, device=DEV, dtype=torch.int32)
        if case["bare"]:
            index[case["bare"] - 1::case["bare"]] = -1
        s = dict(case=case)
        if case["ragged"]:
            rows = torch.tensor(_lengths(n, 1, case["t"]), device=DEV)[torch.randperm(n, generator=g, device=DEV)]
            s["index"] = index.repeat_interleave(rows)
            s["x"] = r(int(rows.sum()), k).to(t)
        else:
            s["index"], s["x"] = index, (r(n, case["t"], k) if case["t"] > 1 else r(n, k)).to(t)
        s["w"] = (r(n_out, k) / math.sqrt(k)).to(t)
        s["bias"] = 0.1 * r(n_out)
        # adapters are trained from zero: their product stays below the layer's own
        s["a"], s["b"] = (r(na, rank, k) / math.sqrt(k)).to(t), (0.4 * r(na, n_out, rank) / math.sqrt(rank)).to(t)
        s["scale"] = 0.5 + torch.rand(na, generator=g, device=DEV)
        return s
    heads, kvh, d, hi = (case[i] for i in ("heads", "kvh", "d", "hi"))
    length = torch.tensor(_lengths(n, case["lo"], hi), device=DEV, dtype=torch.int32)
    length = length[torch.randperm(n, generator=g, device=DEV)]
    tokens = n * hi if case["pad"] else int(length.sum())
    # q, k and v come from one projection: pieces of each row
    qkv = r(tokens, heads + 2 * kvh, d)
    qkv[:, :heads] *= 1.5
    qkv = qkv.to(t)
    s = dict(case=case, max_len=hi, start=None, length=None)
    if case["pad"]:
        s["length"] = length
        qkv = qkv.view(n, hi, heads + 2 * kvh, d)
    else:
        s["start"] = torch.nn.functional.pad(length.cumsum(0), (1, 0)).to(torch.int32)
    s["q"], s["k"], s["v"] = qkv.split([heads, kvh, kvh], -2)
    s["mask"] = None
    if case["mask"]:
        keep = torch.rand(tokens, generator=g, device=DEV) > 0.15
        s["mask"] = keep.view(n, hi) if case["pad"] else keep
    s["prefix"] = None
    if case["prefix"]:
        s["prefix"] = torch.randint(0, hi // 2 + 1, (n,), generator=g, device=DEV, dtype=torch.int32)
    s["bias"] = 1.5 * r(heads, 2 * case["reach"] + 1) if case["reach"] else None
    s["slope"] = torch.exp2(-8 * (1 + torch.arange(heads, device=DEV)) / heads) if case["slope"] else None
    return s


# ------------------------------------------------------------------ passes
def run(s):
    case = s["case"]
    if own:
        ops = _own_ops()
        if case["kind"] == "lora":
            return ops.linear_adapters(s["x"], s["w"], s["a"], s["b"], s["index"], scale=s["scale"], bias=s["bias"])
        o = ops.text_attention(s["q"], s["k"], s["v"], s["max_len"], start=s["start"], length=s["length"], mask=s["mask"],
                               causal=case["causal"], prefix=s["prefix"], cap=case["cap"] or None, bias=s["bias"],
                               slope=s["slope"])
        return o
    return _plain_lora(case, s) if case["kind"] == "lora" else _plain_text(case, s)


def _plain_lora(case, s):
    x, rank = s["x"].float(), case["r"]
    y = x @ s["w"].float().t() + s["bias"]
    live = s["index"] >= 0
    at = s["index"].long().clamp(min=0)
    if x.dim() == 3:  # one adapter per x[i]
        v = x @ s["a"].float()[at].transpose(1, 2).contiguous()
        delta = v @ s["b"].float()[at].transpose(1, 2).contiguous()
        y = y + delta * (s["scale"][at] * live)[:, None, None]
    else:  # one per row: all adapters' products with every row, its own picked
        na = case["na"]
        v = (x @ s["a"].float().reshape(na * rank, -1).t()).view(-1, na, rank)
        pick = (at[:, None] == torch.arange(na, device=x.device)) & live[:, None]
        v = (v * (pick * s["scale"])[:, :, None]).view(-1, na * rank)
        y = y + v @ s["b"].float().transpose(1, 2).reshape(na * rank, -1)
    return y.to(s["x"].dtype)


def _plain_text(case, s):
    n, heads, kvh, d, hi = (case[i] for i in ("n", "heads", "kvh", "d", "hi"))
    rep, dev = heads // kvh, s["q"].device
    pos = torch.arange(hi, device=dev)
    if case["pad"]:
        inside = pos < s["length"][:, None]
        at = (torch.arange(n, device=dev)[:, None] * hi + pos)
    else:
        inside = pos < (s["start"][1:] - s["start"][:-1])[:, None]
        at = (s["start"][:-1, None].long() + pos) * inside
    qs, ks, vs = s["q"].reshape(-1, heads, d), s["k"].reshape(-1, kvh, d), s["v"].reshape(-1, kvh, d)
    far = pos[None, :] - pos[:, None]  # key less query
    extra = None
    if s["bias"] is not None:
        extra = s["bias"][:, far.clamp(-case["reach"], case["reach"]) + case["reach"]]
    if s["slope"] is not None:
        fall = s["slope"][:, None, None] * -far.abs().float()
        extra = fall if extra is None else extra + fall
    if extra is not None:
        extra = extra.view(kvh, rep, hi, hi)
    out = torch.zeros_like(qs)
    step = max(1, (1 << 28) // (heads * hi * hi))
    for c in range(0, n, step):
        rows = at[c:c + step]
        q = qs[rows].float().view(-1, hi, kvh, rep, d).permute(0, 2, 3, 1, 4).reshape(-1, kvh, rep * hi, d)
        live = inside[c:c + step]
        k = ks[rows].float().permute(0, 2, 3, 1).contiguous()
        v = vs[rows].float().masked_fill(~live[:, :, None, None], 0).transpose(1, 2).contiguous()
        a = (q @ k / math.sqrt(d)).view(-1, kvh, rep, hi, hi)
        if case["cap"]:
            a = case["cap"] * torch.tanh(a / case["cap"])
        if extra is not None:
            a = a + extra
        if s["mask"] is not None:
            live = live & s["mask"].reshape(-1)[rows]
        see = live[:, None, :]
        if case["causal"]:
            order = far <= 0
            if s["prefix"] is not None:
                order = order | (pos < s["prefix"][c:c + step, None])[:, None, :]
            see = see & order
        a = a.masked_fill(~see.expand(-1, hi, hi)[:, None, None], -math.inf)
        top = a.amax(4, keepdim=True)
        p = torch.exp(a - top.masked_fill(top == -math.inf, 0))
        total = p.sum(4, keepdim=True)
        o = (p / total.masked_fill(total == 0, 1)).view(-1, kvh, rep * hi, hi) @ v
        o = o.view(-1, kvh, rep, hi, d).permute(0, 3, 1, 2, 4).reshape(-1, hi, heads, d).to(out.dtype)
        keep = inside[c:c + step]
        if case["pad"]:
            out.view(n, hi, heads, d)[c:c + step] = o * keep[:, :, None, None]
        else:  # (rows past a text's end fall on its first row, which then is added zeros)
            out.index_add_(0, rows.reshape(-1), (o * keep[:, :, None, None]).reshape(-1, heads, d))
    return out.view(s["q"].shape)


# ------------------------------------------------------------------ work
def work(case):
    b, n = SIZE[case["dt"]], case["n"]
    if case["kind"] == "lora":
        k, n_out, rank = case["k"], case["n_out"], case["r"]
        m = sum(_lengths(n, 1, case["t"])) if case["ragged"] else n * case["t"]
        bare = n // case["bare"] if case["bare"] else 0
        used = case["na"] * (1 - (1 - 1 / case["na"]) ** (n - bare))
        return {"bytes": b * (m * (k + n_out) + n_out * k + used * rank * (k + n_out)) + 4.0 * (n_out + n),
                "flops": 2.0 * m * n_out * k + 2.0 * m * (n - bare) / n * rank * (k + n_out)}
    lo, hi, heads, kvh, d = (case[i] for i in ("lo", "hi", "heads", "kvh", "d"))
    lengths = _lengths(n, lo, hi)

    def pairs(length):
        if not case["causal"]:
            return length * length
        p = min(length, hi / 4) if case["prefix"] else 0
        return length * (length + 1) / 2 + p * p / 2

    tokens = sum(lengths)
    seen = sum(pairs(length) for length in lengths) * (0.85 if case["mask"] else 1.0)
    return {"bytes": 2.0 * tokens * (heads + kvh) * d * b + tokens * int(case["mask"]) + 4.0 * heads * (2 * case["reach"] + 1),
            "flops": 4.0 * seen * heads * d}


# ------------------------------------------------------------------ 64 bits
def _exact_lora(case, s):
    x = s["x"].double().reshape(-1, case["k"])
    y = x @ s["w"].double().t().contiguous()
    y += s["bias"].double()
    index = s["index"].repeat_interleave(s["x"].shape[1]) if s["x"].dim() == 3 else s["index"]
    for a in range(case["na"]):  # adapter by adapter, its own rows
        rows = torch.nonzero(index == a).flatten()
        if len(rows):
            low = x[rows] @ s["a"][a].double().t().contiguous()
            y[rows] += float(s["scale"][a]) * (low @ s["b"][a].double().t().contiguous())
    return y.view(s["x"].shape[:-1] + (case["n_out"],))


def _exact_text(case, s):
    heads, kvh, d, hi, cap, reach = (case[i] for i in ("heads", "kvh", "d", "hi", "cap", "reach"))
    qs, ks, vs = s["q"].reshape(-1, heads, d), s["k"].reshape(-1, kvh, d), s["v"].reshape(-1, kvh, d)
    out = torch.zeros(qs.shape, device=DEV, dtype=torch.float64)
    if case["pad"]:
        spans = [(c * hi, c * hi + m) for c, m in enumerate(s["length"].tolist())]
    else:
        ends = s["start"].tolist()
        spans = list(zip(ends[:-1], ends[1:]))
    for c, (first, last) in enumerate(spans):
        size = last - first
        if not size:
            continue
        i = torch.arange(size, device=DEV)[:, None]
        j = torch.arange(size, device=DEV)[None, :]
        hidden = torch.zeros(size, size, device=DEV, dtype=torch.bool)
        if case["causal"]:
            hidden = j > i
            if s["prefix"] is not None:
                hidden = hidden & (j >= int(s["prefix"][c]))
        if s["mask"] is not None:
            hidden = hidden | ~s["mask"].reshape(-1)[first:last][None, :]
        blind = hidden.all(1)
        for h in range(heads):
            g = h // (heads // kvh)
            a = qs[first:last, h].double() @ ks[first:last, g].double().t().contiguous()
            a *= d ** -0.5
            if cap:
                a = torch.tanh(a.div_(cap)).mul_(cap)
            if reach:
                a += s["bias"][h].double()[torch.clamp(j - i, -reach, reach) + reach]
            if s["slope"] is not None:
                a -= s["slope"][h].double() * (j - i).abs()
            a[hidden] = -math.inf
            a[blind] = 0.0
            o = torch.softmax(a, 1) @ vs[first:last, g].double()
            o[blind] = 0.0
            out[first:last, h] = o
    return out.view(s["q"].shape)


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_lora(case, s) if case["kind"] == "lora" else _exact_text(case, s)
