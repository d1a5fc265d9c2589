"""Attention inside texts (text_attention) on the GPU against the oracle's
float64 definition.  Tolerances count roundings."""
import math

import numpy as np
import pytest

from oracle import text as O
from tests.test_gpu_text_ops import NAN, U16, U32, _close, _gen, _np, _t, ops  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _case(seed, dt, heads, kvh, d, lens, pad=False, gap=0, mask=0.0, prefix=False, reach=0, slope=False, spread=1.0):
    """(q, k, v, max_len, arguments, texts, rows of the oracle's layout); what takes no part holds NaN."""
    g, cpu = _gen(seed), torch.Generator().manual_seed(seed)
    n, hi = len(lens), max(max(lens), 1)
    ends = np.cumsum([gap] + list(lens))
    texts = [(c * hi if pad else int(ends[c]), lens[c]) for c in range(n)]
    tokens = n * hi if pad else max(int(ends[-1]) + gap, 1)
    live = torch.zeros(tokens, dtype=torch.bool)
    for first, size in texts:
        live[first:first + size] = True
    inside = live.clone()
    kw = {}
    if mask:
        m = torch.rand(tokens, generator=cpu) >= mask
        live &= m
        kw["mask"] = (m.view(n, hi) if pad else m).cuda()
    q = (spread * torch.randn(tokens, heads, d, generator=g, device="cuda")).to(_t(dt))
    k, v = (torch.randn(tokens, kvh, d, generator=g, device="cuda").to(_t(dt)) for _ in range(2))
    q[~inside.cuda()] = NAN
    k[~live.cuda()], v[~live.cuda()] = NAN, NAN
    if prefix:
        kw["prefix"] = torch.tensor([(5 * c + 3) % (m + 4) - 2 for c, m in enumerate(lens)], dtype=torch.int32).cuda()
    if reach is not None and reach >= 0 and not (reach == 0):
        kw["bias"] = 2 * torch.randn(heads, 2 * reach + 1, generator=g, device="cuda")
    if slope:
        kw["slope"] = torch.rand(heads, generator=g, device="cuda")
    if pad:
        kw["length"] = torch.tensor(lens, dtype=torch.int32).cuda()
        q, k, v = (t.view(n, hi, -1, d) for t in (q, k, v))
    else:
        kw["start"] = torch.tensor(ends, dtype=torch.int32).cuda()
    return q, k, v, hi, kw, texts


def _check(got, q, k, v, texts, dt, what, causal=False, cap=None, scale=None, mask=None, prefix=None, bias=None, slope=None,
           **_):
    d, heads = q.shape[-1], q.shape[-2]
    scale = d ** -0.5 if scale is None else scale
    qn, kn, vn = (np.nan_to_num(_np(t).reshape(-1, t.shape[-2], d)) for t in (q, k, v))
    host = lambda t: None if t is None else _np(t)  # noqa: E731
    o, w = O.text_attention(qn, kn, vn, texts, scale, mask=None if mask is None else mask.cpu().numpy().reshape(-1),
                            causal=causal, prefix=host(prefix), cap=cap, bias=host(bias), slope=host(slope))
    # A score: d products and sums and the scale, of terms that add up to at most
    # `top`; exp and its argument 4 more, each weight is off by e^2es.  The cap: the
    # exponential's and the reciprocal's roundings times 2 cap, below 8 cap U.
    # Distance terms: two products, the clamp and the sum with the score.  The sums
    # over keys are chains of at most half the text.  bf16: the weights (twice:
    # they are summed too) and the result are rounded to bf16.
    top = abs(scale) * np.linalg.norm(qn, axis=-1).max() * max(np.linalg.norm(kn, axis=-1).max(), 1e-30)
    longest = max([m for _, m in texts] + [0])
    terms = 0 if bias is None else np.abs(_np(bias)[np.abs(_np(bias)) < 1e30]).max(initial=0)  # (fp32's lowest leaves nothing else)
    terms += 0 if slope is None else np.abs(_np(slope)).max() * longest
    rel = 2 * (d + 16) * U32 * top + 16 * (cap or 0) * U32 + 12 * U32 * terms + (longest / 2 + 40) * U32
    tol = rel * w + U32 * np.abs(o)
    if dt == "bf16":
        tol = tol + 2 * U16 * w + U16 * (np.abs(o) + 2 * U16 * w)
    _close(_np(got).reshape(o.shape), o, tol + 1e-37, what)


SHAPES = [
    # heads, kv heads, d, lengths
    (1, 1, 8, [1]),
    (4, 4, 40, [5, 0, 77]),
    (4, 2, 64, [31, 64, 1, 130]),
    (6, 2, 16, [32, 33, 63]),
    (2, 1, 80, [129, 65]),
    (3, 3, 72, [128, 7]),
    (2, 2, 96, [100]),
    (4, 1, 128, [97, 0, 20]),
    (2, 2, 160, [70, 33]),
    (1, 1, 192, [66]),
    (2, 1, 256, [90, 3]),
    (3, 1, 24, [259]),
]
MODES = [
    dict(),
    dict(causal=True),
    dict(causal=True, prefix=True, mask=0.3),
    dict(mask=0.4, reach=5),
    dict(causal=True, reach=40, slope=True),
    dict(cap=3.0),
    dict(cap=7.0, causal=True, mask=0.5, reach=200),
    dict(cap=50.0, slope=True, causal=True, prefix=True),
]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kvh,d,lens", SHAPES)
def test_text_attention(ops, heads, kvh, d, lens, dt):  # noqa: F811
    for at, mode in enumerate(MODES):
        how = {i: mode[i] for i in ("causal", "cap") if i in mode}
        make = {i: mode[i] for i in mode if i not in how}
        pad = (at + d) % 2 == 0
        q, k, v, hi, kw, texts = _case(at + d, dt, heads, kvh, d, lens, pad=pad, gap=0 if pad else at, **make)
        got = ops.text_attention(q, k, v, hi, **kw, **how)
        _check(got, q, k, v, texts, dt, f"{(heads, kvh, d, lens, dt, mode, pad)}", **kw, **how)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("d", [40, 64])
def test_text_attention_rows_in_no_text(ops, d, dt):  # noqa: F811
    """Zeros in a new result, as they were in a given one; the result may lie inside a wider array."""
    for pad in (False, True):
        q, k, v, hi, kw, texts = _case(d, dt, 4, 2, d, [40, 0, 130, 3], pad=pad, gap=0 if pad else 150)
        more = hi if pad else 140  # (texts shorter than max_len says)
        got = ops.text_attention(q, k, v, more, causal=True, **kw)
        _check(got, q, k, v, texts, dt, f"{(d, dt, pad)}", causal=True, **kw)
        wide = torch.full(q.shape[:-2] + (6, d + 16), 5.0, device="cuda", dtype=_t(dt))
        ops.text_attention(q, k, v, more, causal=True, out=wide[..., 1:5, 8:8 + d], **kw)
        ref = torch.full_like(wide, 5.0)
        flat, rf = got.reshape(-1, 4, d), ref.view(-1, 6, d + 16)
        for first, size in texts:
            rf[first:first + size, 1:5, 8:8 + d] = flat[first:first + size]
        assert torch.equal(wide, ref)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.randn(5, 2, d, device="cuda").to(_t(dt))
    assert not ops.text_attention(q, q, q, 5, start=none).any()
    assert ops.text_attention(q[:0], q[:0], q[:0], 5, start=none).shape == (0, 2, d)
    assert not ops.text_attention(q, q, q, 0, start=torch.tensor([0, 5], dtype=torch.int32, device="cuda")).any()
    bad = torch.tensor([-7, 2, 1, 40], dtype=torch.int32, device="cuda")  # cut to rows 0..1, nothing, 1..4
    a = ops.text_attention(q, q, q, 5, start=bad)
    two = ops.text_attention(q[:2], q[:2], q[:2], 5, start=torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    assert torch.equal(a[0], two[0]) and torch.isfinite(a).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 88, 128, 256])
def test_text_attention_infinities_behind_the_border(ops, d, dt):  # noqa: F811
    """Keys behind a query's causal border may hold anything; seen ones bring what they hold."""
    n = 200
    for prefix in (0, 70):
        q, k, v, hi, kw, texts = _case(d, dt, 2, 1, d, [n])
        kw["prefix"] = torch.tensor([prefix], dtype=torch.int32, device="cuda")
        kw["slope"] = torch.full((2,), 0.01, device="cuda")
        for cap in (None, 10.0):
            clean = ops.text_attention(q, k, v, hi, causal=True, cap=cap, **kw)
            vb = v.clone()
            vb[150, 0, 3], vb[150, 0, d - 1], vb[160, 0, 3] = math.inf, NAN, -math.inf
            got = ops.text_attention(q, k, vb, hi, causal=True, cap=cap, **kw)
            assert torch.equal(got[:150], clean[:150]), (d, dt, prefix, cap)
            assert (got[150:160, :, 3] == math.inf).all() and got[150:, :, d - 1].isnan().all()
            assert got[160:, :, 3].isnan().all()
            cols = [c for c in range(d) if c not in (3, d - 1)]
            assert torch.equal(got[:, :, cols], clean[:, :, cols])
            kb = k.clone()
            kb[130] = NAN
            kb[190, 0, 2] = math.inf
            got = ops.text_attention(q, kb, v, hi, causal=True, cap=cap, **kw)
            assert torch.equal(got[:130], clean[:130]) and got[130:].isnan().all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 0.125, 2.0 ** -50])
def test_text_attention_lowest_bias(ops, scale, dt):  # noqa: F811
    """-inf takes a key out; fp32's lowest value only where others are higher."""
    low = torch.finfo(torch.float32).min
    q, k, v, hi, kw, texts = _case(3, dt, 3, 3, 64, [150, 9], reach=4, spread=1 / (8 * scale) if scale > 2e-15 else 1.0)
    b = kw["bias"]
    b[0, :4], b[1, 5:], b[1, 0] = -math.inf, low, low
    b[2] = low
    for cap in (None, 5.0):
        got = ops.text_attention(q, k, v, hi, scale=scale, cap=cap, **kw)
        _check(got, q, k, v, texts, dt, f"{(scale, dt, cap)}", scale=scale, cap=cap, **kw)
    b[:] = -math.inf
    assert not ops.text_attention(q, k, v, hi, scale=scale, **kw).any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.0, -0.2, 4.0])
def test_text_attention_scales(ops, scale, dt):  # noqa: F811
    """Scores far apart, negative and zero scales, with and without a cap."""
    for cap in (None, 2.0):
        q, k, v, hi, kw, texts = _case(11, dt, 2, 1, 40, [140, 30], reach=9, spread=2.0)
        got = ops.text_attention(q, k, v, hi, scale=scale, cap=cap, causal=True, **kw)
        _check(got, q, k, v, texts, dt, f"{(scale, dt, cap)}", scale=scale, cap=cap, causal=True, **kw)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("mode", [dict(), dict(causal=True, cap=20.0), dict(causal=True)])
def test_text_attention_texts_do_not_depend_on_their_batch(ops, mode, dt):  # noqa: F811
    lens = [300, 17, 128, 1, 64]
    q, k, v, hi, kw, texts = _case(5, dt, 4, 2, 64, lens, reach=30)
    whole = ops.text_attention(q, k, v, hi, **kw, **mode)
    assert torch.equal(ops.text_attention(q, k, v, 4000, **kw, **mode), whole)
    assert torch.equal(ops.text_attention(q, k, v, hi, **kw, **mode), whole)
    for first, size in texts:
        rows = slice(first, first + size)
        one = dict(kw, start=torch.tensor([0, size], dtype=torch.int32, device="cuda"))
        assert torch.equal(ops.text_attention(q[rows], k[rows], v[rows], size, **one, **mode), whole[rows]), size
        alone = dict(bias=kw["bias"])
        got = ops.text_attention(q[rows][None], k[rows][None], v[rows][None], size, **alone, **mode)
        assert torch.equal(got[0], whole[rows]), size


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 48, 64, 96, 192])
def test_text_attention_bits_do_not_depend_on_the_longest_text(ops, d, dt):  # noqa: F811
    """Texts of up to 128 tokens alone, and with a max_len (or a text) past that."""
    q, k, v, hi, kw, texts = _case(d, dt, 2, 2, d, [128, 70, 64, 5], reach=20, mask=0.2)
    for mode in (dict(), dict(causal=True), dict(causal=True, cap=9.0)):
        first = ops.text_attention(q, k, v, hi, **kw, **mode)
        _check(first, q, k, v, texts, dt, f"{(d, dt, mode)}", **kw, **mode)
        for most in (129, 300):
            assert torch.equal(ops.text_attention(q, k, v, most, **kw, **mode), first), (most, mode)
        free = {i: kw[i] for i in kw if i != "bias"}
        assert torch.equal(ops.text_attention(q, k, v, hi, **free, **mode), ops.text_attention(q, k, v, 300, **free, **mode)), mode


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_text_attention_layouts(ops, dt):  # noqa: F811
    """Pieces of one projection, shared heads of stride 0, masks as bytes."""
    q, k, v, hi, kw, texts = _case(8, dt, 4, 2, 40, [90, 33], mask=0.2, pad=True)
    whole = ops.text_attention(q, k, v, hi, causal=True, **kw)
    qkv = torch.cat((q, k, v), 2)
    parts = qkv.split([4, 2, 2], 2)
    kw8 = dict(kw, mask=kw["mask"].to(torch.uint8) * 255)
    assert torch.equal(ops.text_attention(*parts, hi, causal=True, **kw8), whole)
    one = ops.text_attention(q, k[:, :, :1].expand(-1, -1, 2, -1), v, hi, causal=True, **kw)
    ref = ops.text_attention(q, k[:, :, :1].repeat(1, 1, 2, 1), v, hi, causal=True, **kw)
    assert torch.equal(one, ref)
    swapped = q.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)  # heads outermost
    assert torch.equal(ops.text_attention(swapped, k, v, hi, causal=True, **kw), whole)


@pytest.mark.parametrize("dt,cap,reach", [("bf16", None, 0), ("bf16", 30.0, 100), ("f32", None, 2000)])
def test_text_attention_long_texts(ops, dt, cap, reach):  # noqa: F811
    """Some queries of long causal texts with a prefix, against 64-bit sums."""
    lens, heads, d = [5000, 1100], 2, 64
    q, k, v, hi, kw, texts = _case(21, dt, heads, 1, d, lens, prefix=False, reach=reach)
    kw["prefix"] = torch.tensor([2100, 40], dtype=torch.int32, device="cuda")
    got = ops.text_attention(q, k, v, hi, causal=True, cap=cap, **kw)
    bias = kw.get("bias")
    for c, (first, size) in enumerate(texts):
        for i in sorted({0, 63, 64, 127, 128, 1000, 2048, 2100, size - 1}):
            if i >= size:
                continue
            keys = max(i + 1, int(kw["prefix"][c]))
            kk, vv = k[first:first + keys, 0].double(), v[first:first + keys, 0].double()
            for h in range(heads):
                s = kk @ q[first + i, h].double() / 8
                s = cap * torch.tanh(s / cap) if cap else s
                if bias is not None:
                    s = s + bias[h].double()[(torch.arange(keys, device="cuda") - i).clamp(-reach, reach) + reach]
                p = torch.softmax(s, 0)
                o, w = _np(p @ vv), _np(p @ vv.abs())
                rel = 2 * (d + 16) * U32 * 40 + 16 * (cap or 0) * U32 + 120 * U32 + (keys / 2 + 40) * U32
                tol = rel * w + (2 * U16 * w + 1.02 * U16 * (np.abs(o) + 2 * U16 * w) if dt == "bf16" else 0) + U32 * np.abs(o)
                _close(_np(got[first + i, h]), o, tol, f"{(dt, cap, c, i, h)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_text_attention_offsets_past_2_31_elements(ops, dt):  # noqa: F811
    d, heads, ld = 64, 2, 1 << 22
    n = 600  # 600 x 2^22 elements: rows of q, k, v and o lie past 2^31
    if dt == "f32":
        n, ld = 540, 1 << 22
    q, k, v, hi, kw, texts = _case(2, dt, heads, heads, d, [n])
    whole = ops.text_attention(q, k, v, hi, causal=True, **kw)
    buf = torch.empty(n * ld, device="cuda", dtype=_t(dt)).view(n, ld)
    at = lambda i: buf[:, 256 * i:256 * i + heads * d].view(n, heads, d)  # noqa: E731
    for i, t in enumerate((q, k, v)):
        at(i).copy_(t)
    ops.text_attention(at(0), at(1), at(2), hi, causal=True, out=at(3), **kw)
    assert torch.equal(at(3), whole)


def test_text_attention_streams_and_graphs(ops):  # noqa: F811
    q, k, v, hi, kw, texts = _case(4, "bf16", 4, 4, 64, [77, 20, 300], reach=16, mask=0.1)
    q2, k2, v2, _, kw2, _ = _case(9, "bf16", 4, 4, 64, [77, 20, 300], reach=16, mask=0.1)
    ref = ops.text_attention(q, k, v, hi, causal=True, **kw)
    ref2 = ops.text_attention(q2, k2, v2, hi, causal=True, **kw2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ops.text_attention(q, k, v, hi, causal=True, **kw)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.text_attention(q, k, v, hi, causal=True, **kw)
    for _ in range(3):
        for src, want in (((q2, k2, v2, kw2), ref2), ((q.clone(), k.clone(), v.clone(), dict(kw)), ref)):
            keep = [t.clone() for t in (q, k, v)]
            arrays = {i: kw[i].clone() for i in ("bias", "mask")}
            for dst, t in zip((q, k, v), src):
                dst.copy_(t)
            for i in arrays:
                kw[i].copy_(src[3][i])
            graph.replay()
            assert torch.equal(out, want)
            assert torch.equal(ops.text_attention(q, k, v, hi, causal=True, **kw), want)
            for dst, t in zip((q, k, v), keep):
                dst.copy_(t)
            for i in arrays:
                kw[i].copy_(arrays[i])
        torch.cuda.synchronize()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("wild", [math.inf, NAN])
@pytest.mark.parametrize("n,d", [(77, 64), (128, 40), (200, 64), (150, 256)])
def test_text_attention_masked_keys_with_any_bias(ops, n, d, wild, dt):  # noqa: F811
    """A key that the mask leaves out takes no part, whatever the bias holds at its distance."""
    far = n // 2  # keys from here on are masked, and to those alone lead distances of as much
    q, k, v, hi, kw, texts = _case(n, dt, 2, 1, d, [n], reach=n)
    kw["mask"] = torch.arange(n, device="cuda") < far
    bias = kw["bias"].clone()
    bias[:, n + far:] = wild
    for cap in (None, 5.0):
        for how in (dict(), dict(causal=True, prefix=torch.tensor([n], dtype=torch.int32, device="cuda"))):
            clean = ops.text_attention(q, k, v, hi, cap=cap, **how, **kw)
            _check(clean, q, k, v, texts, dt, f"{(n, d, dt, cap)}", cap=cap, **how, **kw)
            got = ops.text_attention(q, k, v, hi, cap=cap, **how, **dict(kw, bias=bias))
            assert torch.equal(got, clean), (cap, list(how))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(77, 64), (128, 40), (200, 64), (150, 256)])
def test_text_attention_masked_keys_and_an_infinite_query(ops, n, d, dt):  # noqa: F811
    """A query whose seen keys all score -inf gives zeros; a masked key is none of them."""
    q, k, v, hi, kw, texts = _case(n, dt, 2, 1, d, [n], mask=0.3)
    k[..., 1] = -k[..., 1].abs() - 0.5
    qb = q.clone()
    qb[n - 3, :, 1] = math.inf
    keep = torch.arange(n, device="cuda") != n - 3
    for how in (dict(), dict(causal=True)):
        clean = ops.text_attention(q, k, v, hi, **how, **kw)
        got = ops.text_attention(qb, k, v, hi, **how, **kw)
        assert torch.equal(got[keep], clean[keep]) and not got[n - 3].any(), list(how)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("value", [math.inf, 1e30])
@pytest.mark.parametrize("n", [128, 200])
def test_text_attention_keys_behind_the_border_leave_the_bits(ops, n, value, dt):  # noqa: F811
    """An infinite or huge key changes no bit of the queries before it, those of its own wave among them."""
    q, k, v, hi, kw, texts = _case(n, dt, 4, 1, 64, [n])
    q, k = 6 + q / 20, 8 + k / 20  # scores of some thousands, a few apart
    at = n - 10
    kb = k.clone()
    kb[at, 0, 2] = value
    clean = ops.text_attention(q, k, v, hi, causal=True, scale=1.0, **kw)
    got = ops.text_attention(q, kb, v, hi, causal=True, scale=1.0, **kw)
    assert torch.isfinite(clean).all() and torch.equal(got[:at], clean[:at])
    assert not torch.equal(got[at:], clean[at:])
