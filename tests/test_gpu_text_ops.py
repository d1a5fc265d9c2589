"""The text-side operators (rmsnorm, linear_rows_w4, cross_attention) on the
GPU against the oracle's float64 definitions.  U32 and U16 are half a step of
fp32 and bf16 relative to the value; every tolerance counts roundings."""
import math

import numpy as np
import pytest

from oracle import text as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U32, U16 = 2.0 ** -24, 2.0 ** -8
NAN = float("nan")


@pytest.fixture(scope="module")
def ops():
    from paper_2605_08835_amd import ops as P
    return P


def _t(dt):
    return torch.bfloat16 if dt == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _np(t):
    return t.detach().cpu().double().numpy()


def _close(got, ref, tol, what):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape and np.isfinite(got).all(), what
    bad = np.abs(got - ref) > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} past the tolerance, worst {np.abs(got - ref)[bad].max():.3e}"


# ------------------------------------------------------------------ rmsnorm
# A row's sum of squares is a chain of at most 64 elements and 10 levels of a
# tree, all terms positive: 74 roundings, halved by the square root; the mean,
# eps, root, products: 11 more at most.
RMS = 48 * U32

ROWS_C = [(1, 1), (3, 7), (5, 8), (70, 9), (300, 64), (33, 127), (9, 128), (9, 129), (2, 257), (64, 320), (5, 768), (1, 1280),
          (300, 1280), (7, 2048), (3, 2056), (4, 5000), (2, 8192), (3, 16383), (2, 16384)]


def _check_norm(got, x, gamma, eps, resid, fp8, group, dt, what):
    y, h = O.rmsnorm(_np(x), None if gamma is None else _np(gamma), eps, None if resid is None else _np(resid))
    half = U16 if dt == "bf16" else U32
    got = list(got) if isinstance(got, tuple) else [got]
    if resid is not None:
        _close(_np(got.pop()), h, (half + U32) * np.abs(h), what + " sum")
    if not fp8:
        _close(_np(got[0]), y, (half + RMS) * np.abs(y) + 1e-38, what + " y")
        return
    s = O.block_scales(y, group)
    _close(_np(got[1]), s, (RMS + 4 * U32) * s, what + " scale")
    full = np.repeat(_np(got[1]), group or y.shape[1], 1)[:, :y.shape[1]]
    _close(_np(got[0]) * full, y, np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * full) * (1 + 1e-4) + RMS * np.abs(y),
           what + " y8")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", ROWS_C)
def test_rmsnorm(ops, rows, C, dt):
    g = _gen(rows * 31 + C)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, res, gamma = (2 * r(rows, C) + 0.3).to(_t(dt)), (5 * r(rows, C)).to(_t(dt)), 1 + 0.3 * r(C)
    for resid in (None, res):
        for fp8, group in ((False, 0), (True, 0), (True, 128)):
            gm = gamma if group == 0 else None
            got = ops.rmsnorm(x, gm, 1e-5, resid=resid, fp8=fp8, scale_group=group)
            _check_norm(got, x, gm, 1e-5, resid, fp8, group, dt, f"{(rows, C, dt, resid is not None, fp8, group)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("C", [2, 4, 12, 16, 17, 24, 32, 40, 100])
def test_rmsnorm_many_narrow_rows(ops, C, dt):
    """Several rows a wave: sums and scales stay each row's own."""
    g = _gen(C)
    x = torch.randn(1037, C, generator=g, device="cuda") * torch.exp2(torch.randint(-6, 7, (1037, 1), generator=g, device="cuda").float())
    x, r = x.to(_t(dt)), torch.randn(1037, C, generator=g, device="cuda").to(_t(dt))
    gamma = torch.randn(C, generator=g, device="cuda")
    for resid in (None, r):
        for fp8, group in ((False, 0), (True, 0), (True, 128)):
            got = ops.rmsnorm(x, gamma, 1e-6, resid=resid, fp8=fp8, scale_group=group)
            _check_norm(got, x, gamma, 1e-6, resid, fp8, group, dt, f"{(C, dt, fp8, group)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("C", [64, 65, 320, 1000])
def test_rmsnorm_strides_alignment_and_neighbours(ops, C, dt):
    """Rows inside wider buffers, aligned and not, one row apart or more; what
    lies around the rows stays as it was."""
    g = _gen(C)
    for off, ld in ((0, C + 8), (8, C + 24), (1, C + 3), (3, C + 16)):
        n = 6
        buf = lambda t: torch.full((n * ld + 16,), 7.0, device="cuda").to(t)  # noqa: E731
        rows = lambda b: b[off:off + n * ld].view(n, ld)[:, :C]  # noqa: E731
        xb, rb, sb, yb = (buf(_t(dt)) for _ in range(4))
        qb = buf(torch.float8_e4m3fn)
        for b in (xb, rb):
            rows(b).copy_(torch.randn(n, C, generator=g, device="cuda") * 3)
        keep = [b.clone() for b in (sb, yb, qb)]
        got = ops.rmsnorm(rows(xb), None, 1e-6, resid=rows(rb), sum_out=rows(sb), out=rows(yb))
        _check_norm(got, rows(xb), None, 1e-6, rows(rb), False, 0, dt, f"{(C, dt, off, ld)}")
        q, s = ops.rmsnorm(rows(xb), None, 1e-6, out=rows(qb), fp8=True, scale_group=128)
        _check_norm((q, s), rows(xb), None, 1e-6, None, True, 128, dt, f"{(C, dt, off, ld)} e4m3")
        for b, k in zip((sb, yb, qb), keep):
            rows(k).copy_(rows(b))
            assert torch.equal(b.view(torch.uint8), k.view(torch.uint8))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("C", [40, 333, 1280, 9000])
def test_rmsnorm_in_place(ops, C, dt):
    g = _gen(C)
    x, r = (torch.randn(5, C, generator=g, device="cuda").to(_t(dt)) for _ in range(2))
    y, h = ops.rmsnorm(x, None, 1e-6, resid=r)
    for ys, hs in ((0, 1), (1, 0), (0, None), (None, 0), (None, 1)):
        a = [x.clone(), r.clone()]
        y2, h2 = ops.rmsnorm(a[0], None, 1e-6, resid=a[1], out=None if ys is None else a[ys],
                             sum_out=None if hs is None else a[hs])
        assert torch.equal(y, y2) and torch.equal(h, h2)


def test_rmsnorm_rows_of_zeros_small_values_and_nan(ops):
    x = torch.zeros(6, 384, device="cuda")
    x[1] = 1e-30
    x[2, 5] = NAN
    x[3, 200] = math.inf
    x[4] = torch.linspace(-1, 1, 384)
    for dt in ("f32", "bf16"):
        xt = x.to(_t(dt))
        y = _np(ops.rmsnorm(xt))
        assert not y[0].any() and not y[5].any() and np.isnan(y[2]).all()
        assert np.isnan(y[3, 200]) and not np.delete(y[3], 200).any()  # inf / inf, finite / inf
        q, s = ops.rmsnorm(xt, fp8=True)
        assert not _np(q[0]).any() and np.isnan(_np(q[2])).all() and np.isnan(_np(s[2])).all() and np.isnan(_np(s[3])).all()
        assert _np(s[0, 0]) == np.float32(2.0 ** -100) / np.float32(448)
        q, s = ops.rmsnorm(xt, fp8=True, scale_group=128)
        assert np.isnan(_np(q[2])).all() and np.isnan(_np(s[2])).all()
        _check_norm((q[4:5], s[4:5]), xt[4:5], None, 1e-6, None, True, 128, dt, "ramp")
    y = ops.rmsnorm(torch.full((2, 64), 3e-39, device="cuda"), eps=0.0)  # squares vanish: 0 * inf or x * inf
    assert not torch.isfinite(y).any()
    assert ops.rmsnorm(torch.zeros(0, 64, device="cuda")).shape == (0, 64)
    assert ops.rmsnorm(torch.ones(2, 3, 64, device="cuda"), fp8=True, scale_group=128)[1].shape == (2, 3, 1)


# ------------------------------------------------------------------ 4-bit weights
def _w4_case(g, M, K, N, group, zero, xt, st, ints=False):
    ng = -(-K // group)
    w = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    if ints:  # every product and partial sum is a whole number below 2^24 times 1/8
        scale = torch.full((N, ng), 0.125, device="cuda") * torch.tensor([1., 2., 4.], device="cuda")[torch.randint(0, 3, (N, ng), generator=g, device="cuda")]
        x = torch.randint(-15, 16, (M, K), generator=g, device="cuda").float()
    else:
        scale = (torch.rand(N, ng, generator=g, device="cuda") + 0.5) * 0.1
        x = torch.randn(M, K, generator=g, device="cuda")
    z = torch.randint(0, 16, (N, ng), generator=g, device="cuda", dtype=torch.uint8) if zero else None
    xs = None
    if xt.startswith("e4m3"):
        b = 1 if xt == "e4m3row" else -(-K // 128)
        xs = torch.rand(M, b, generator=g, device="cuda") + 0.5
        if ints:
            xs = torch.exp2(torch.randint(-1, 2, (M, b), generator=g, device="cuda").float())
        x = x.to(torch.float8_e4m3fn)
    else:
        x = x.to(_t(xt))
    return x, xs, w, scale.to(_t(st)), z


def _w4_ref(x, xs, w, scale, z, group, bias=None, add=None, silu_in=False):
    """(pre-activation, its rms over random signs) in float64."""
    a = _np(x)
    if xs is not None:
        a = a * np.repeat(_np(xs), a.shape[1] if xs.shape[1] == 1 else 128, 1)[:, :a.shape[1]]
    if silu_in:
        a = a / (1 + np.exp(-a))
    wt = O.w4_weights(w.cpu().numpy(), _np(scale), None if z is None else _np(z), group)
    y = a @ wt.T
    size = np.sqrt((a * a) @ (wt * wt).T) + np.sqrt((a * a) @ np.repeat(_np(scale), group, 1)[:, :a.shape[1]].T ** 2)
    for t in (bias, add):
        if t is not None:
            y = y + _np(t)
            size = size + np.abs(_np(t))
    return y, size


# fp32: each of up to K roundings of a group's partial sums, whose terms are
# at most 62 scales (twice a code or zero point of up to 31) against a result
# of rms 4.6: a random walk of 2^-24 * 0.29 * 26 * sqrt(group) at most, relative
# to the rms of the result; 8 times that for the largest of 10^5 values.
W4 = 8 * 0.29 * 26 * math.sqrt(128) * U32

W4_SHAPES = [(1, 8, 1), (1, 32, 16), (2, 24, 5), (1, 320, 1280), (3, 40, 17), (5, 136, 63), (15, 128, 64), (16, 1280, 65),
             (17, 2816, 257), (33, 1288, 100), (64, 512, 130), (65, 264, 48), (130, 96, 33), (7, 8192, 40), (2, 16, 2500), (3, 264, 16401), (20, 328, 16385), (5, 136, 8200)]


@pytest.mark.parametrize("xt", ["f32", "bf16", "e4m3row", "e4m3"])
@pytest.mark.parametrize("M,K,N", W4_SHAPES)
def test_linear_rows_w4(ops, M, K, N, xt):
    for group in (32, 64, 128):
        for zero in (False, True):
            g = _gen(M + K + N + group + zero)
            st = "bf16" if zero == (group == 64) else "f32"
            # whole numbers: every order of the sums gives these bits
            x, xs, w, scale, z = _w4_case(g, M, K, N, group, zero, xt, st, ints=True)
            ref, _ = _w4_ref(x, xs, w, scale, z, group)
            if np.abs(ref).max() * 8 < 2 ** 22:
                assert np.array_equal(_np(ops.linear_rows_w4(x, w, scale, group, zero=z, x_scale=xs)), ref)
            x, xs, w, scale, z = _w4_case(g, M, K, N, group, zero, xt, st)
            what = f"{(M, K, N, xt, group, zero)}"
            ref, size = _w4_ref(x, xs, w, scale, z, group)
            got = ops.linear_rows_w4(x, w, scale, group, zero=z, x_scale=xs)
            _close(_np(got), ref, W4 * size, what)
            got = ops.linear_rows_w4(x, w, scale, group, zero=z, x_scale=xs, out_dtype=torch.bfloat16)
            _close(_np(got), ref, W4 * size + U16 * (np.abs(ref) + W4 * size), what + " bf16")


@pytest.mark.parametrize("xt", ["f32", "bf16"])
def test_linear_rows_w4_activations_bias_and_addition(ops, xt):
    for M, K, N in ((1, 320, 1280), (32, 1280, 100), (70, 72, 31)):
        g = _gen(M)
        x, xs, w, scale, z = _w4_case(g, M, K, N, 64, True, xt, "bf16")
        bias, add = torch.randn(N, generator=g, device="cuda"), torch.randn(M, N, generator=g, device="cuda")
        for si, so in ((0, 0), (1, 0), (0, 1), (1, 1)):
            ref, size = _w4_ref(x, xs, w, scale, z, 64, bias, add, si)
            tol = W4 * size + 8 * U32 * size  # SiLU of x: exp, division; bias, addition
            if so:  # |d silu| <= 1.1; its own exp and division
                ref, tol = ref / (1 + np.exp(-ref)), 1.1 * tol + 8 * U32 * np.abs(ref)
            out = add.clone()
            got = ops.linear_rows_w4(x, w, scale, 64, zero=z, bias=bias, add=out, silu_in=si, silu_out=so, out=out)
            assert got is out
            _close(_np(got), ref, tol, f"{(M, K, N, xt, si, so)}")


@pytest.mark.parametrize("xt", ["f32", "bf16", "e4m3"])
def test_linear_rows_w4_strides_and_row_independence(ops, xt):
    """x and out inside wider buffers; a row's bits do not depend on how many
    rows come with it; what lies around the output stays as it was."""
    g = _gen(3)
    M, K, N = 66, 648, 77
    x, xs, w, scale, z = _w4_case(g, M, K, N, 32, True, xt, "bf16")
    whole = ops.linear_rows_w4(x, w, scale, 32, zero=z, x_scale=xs)
    wide = torch.zeros(M, K + 56, device="cuda").to(x.dtype)
    wide[:, 16:16 + K] = x
    out = torch.full((M, N + 5), 9.0, device="cuda")
    ops.linear_rows_w4(wide[:, 16:16 + K], w, scale, 32, zero=z, x_scale=xs, out=out[:, 2:2 + N])
    assert torch.equal(out[:, 2:2 + N], whole) and (out[:, :2] == 9).all() and (out[:, 2 + N:] == 9).all()
    for rows in (1, 2, 9, 16, 17, 31, 40, 64):
        part = ops.linear_rows_w4(x[:rows], w, scale, 32, zero=z, x_scale=None if xs is None else xs[:rows])
        assert torch.equal(part, whole[:rows]), rows
    assert ops.linear_rows_w4(x[:0], w, scale, 32, zero=z, x_scale=None if xs is None else xs[:0]).shape == (0, N)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(17, 24, 4096), (33, 1160, 4100), (20, 1288, 8200), (49, 2184, 8195), (64, 4232, 4129)])
def test_linear_rows_w4_rows_by_the_dozen(ops, M, K, N, xt):
    """Layers of some thousand outputs: right, and the same bits whether the rows come alone or together."""
    for group, zero in ((32, True), (64, False), (128, True)):
        g = _gen(M + K + N + group)
        x, xs, w, scale, z = _w4_case(g, M, K, N, group, zero, xt, "f32")
        for si in (False, True):
            got = ops.linear_rows_w4(x, w, scale, group, zero=z, silu_in=si)
            for i, rows in ((0, 1), (M // 2, 5), (1, 16), (M - 17, 17)):
                assert torch.equal(ops.linear_rows_w4(x[i:i + rows], w, scale, group, zero=z, silu_in=si), got[i:i + rows]), (i, rows)
        ref, size = _w4_ref(x, xs, w, scale, z, group, silu_in=True)
        _close(_np(got), ref, W4 * size + 8 * U32 * size, f"{(M, K, N, xt, group)}")


def test_linear_rows_w4_large_small_and_non_finite_values(ops):
    g = _gen(8)
    x, xs, w, scale, z = _w4_case(g, 5, 256, 48, 64, False, "f32", "f32")
    for m, f in ((0, 1e30), (1, 1e-30), (2, 1.0)):
        x[m] *= f
    x[2, ::2] *= 2.0 ** -60  # values of both sizes in one row
    ref, size = _w4_ref(x, xs, w, scale, z, 64)
    x[3, 100], x[4, 3] = math.inf, NAN
    got = _np(ops.linear_rows_w4(x, w, scale, 64))
    _close(got[:3], ref[:3], W4 * size[:3], "sizes")
    assert not np.isfinite(got[3:]).any()


# ------------------------------------------------------------------ attention
def _attn_case(seed, dt, n, nq, heads, kvh, d, lens, pad=False, mask=0.0, index=None, spread=1.0):
    """Inputs, and the token rows of every row's text; keys that take no part hold NaN."""
    g = _gen(seed)
    nc, hi = len(lens), max(max(lens), 1)
    length = torch.tensor(lens, dtype=torch.int32)
    start = torch.arange(nc, dtype=torch.int32) * hi if pad else length.cumsum(0).to(torch.int32) - length
    tokens = nc * hi if pad else max(int(length.sum()), 1)
    live = torch.zeros(tokens, dtype=torch.bool)
    for c in range(nc):
        live[int(start[c]):int(start[c]) + lens[c]] = True
    m = None
    if mask:
        m = torch.rand(tokens, generator=torch.Generator().manual_seed(seed)) >= mask
        live &= m
    q = (spread * torch.randn(n, nq, heads, d, generator=g, device="cuda")).to(_t(dt))
    k, v = (torch.randn(tokens, kvh, d, generator=g, device="cuda").to(_t(dt)) for _ in range(2))
    k[~live.cuda()], v[~live.cuda()] = NAN, NAN
    index = list(range(n)) if index is None else index
    texts = [[t for t in range(int(start[c]), int(start[c]) + lens[c]) if live[t]] if 0 <= c < nc else [] for c in index]
    kw = dict(kv_len=length.cuda(), kv_index=None if index == list(range(n)) else torch.tensor(index, dtype=torch.int32).cuda())
    kw["mask"] = None if m is None else (m.view(nc, hi) if pad else m).cuda()
    if pad:
        return q, k.view(nc, hi, kvh, d), v.view(nc, hi, kvh, d), hi, kw, texts
    return q, k, v, hi, dict(kw, kv_start=start.cuda()), texts


def _check_attn(got, q, k, v, texts, dt, what, scale=None):
    d = q.shape[-1]
    scale = d ** -0.5 if scale is None else scale
    kn, vn = (np.nan_to_num(_np(t).reshape(-1, t.shape[-2], d)) for t in (k, v))
    o, w = O.cross_attention(_np(q), kn, vn, texts, scale)
    # A score: d products and sums, the scale, of terms that add up to at most
    # `top` in size; exp and its argument 4 more.  Every weight is off by e^2es,
    # the sums by a chain of len / 8 + 32 roundings.  bf16: the weights (twice:
    # they are summed too) and the result are rounded to bf16.
    top = abs(scale) * np.linalg.norm(_np(q), axis=-1).max() * max(np.linalg.norm(kn, axis=-1).max(), 1e-30)
    rel = 2 * (d + 12) * U32 * top + (max(map(len, texts)) / 8 + 40) * U32
    tol = rel * w + U32 * np.abs(o)
    if dt == "bf16":
        tol = tol + 2 * U16 * w + U16 * (np.abs(o) + 2 * U16 * w)
    _close(_np(got), o, tol + 1e-37, what)


ATTN = [
    # n, nq, heads, kv heads, d, lengths
    (1, 1, 1, 1, 8, [1]),
    (3, 1, 4, 4, 40, [5, 0, 77]),
    (2, 1, 16, 4, 64, [231, 3]),
    (3, 2, 8, 1, 80, [33, 64, 65]),
    (2, 5, 6, 2, 16, [32, 31]),
    (2, 7, 5, 5, 256, [100, 7]),
    (2, 33, 4, 4, 40, [77, 12]),
    (2, 64, 3, 3, 72, [64, 128]),
    (3, 100, 8, 4, 32, [96, 97, 1]),
    (1, 130, 2, 2, 160, [77]),
    (2, 257, 2, 1, 64, [130, 20]),
    (2, 48, 4, 4, 128, [200, 511]),
    (1, 40, 2, 2, 192, [77]),
    (1, 300, 1, 1, 248, [45]),
    (2, 20, 24, 8, 96, [70, 71]),
    (1, 70, 3, 1, 24, [63]),
    (1, 41, 2, 2, 48, [129]),
    (1, 35, 2, 2, 112, [90]),
    (1, 50, 1, 1, 224, [66]),
]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,nq,heads,kvh,d,lens", ATTN)
def test_cross_attention(ops, n, nq, heads, kvh, d, lens, dt):
    for pad, mask in ((False, 0.0), (True, 0.3), (False, 0.3), (True, 0.0)):
        q, k, v, hi, kw, texts = _attn_case(n + nq + d, dt, n, nq, heads, kvh, d, lens, pad, mask)
        got = ops.cross_attention(q, k, v, hi, **kw)
        _check_attn(got, q, k, v, texts, dt, f"{(n, nq, heads, kvh, d, lens, dt, pad, mask)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("nq,heads,kvh,d,lens", [
    (1, 4, 4, 64, [5000, 1, 1023]), (1, 8, 1, 40, [1024, 4097, 2048]), (3, 2, 2, 128, [3000, 0, 700]),
    (20, 2, 1, 64, [2500, 1025, 9]), (1, 1, 1, 256, [20001, 1025, 130]), (40, 2, 2, 40, [1500, 1024, 77])])
def test_cross_attention_long_texts(ops, nq, heads, kvh, d, lens, dt):
    """Texts long enough to be split; whole stretches masked out."""
    for mask in (0.0, 0.5):
        q, k, v, hi, kw, texts = _attn_case(nq + d, dt, 3, nq, heads, kvh, d, lens, False, mask, spread=2.0)
        if mask:
            kw["mask"][:2100] = False
            texts = [[t for t in x if t >= 2100] for x in texts]
        got = ops.cross_attention(q, k, v, hi, **kw)
        _check_attn(got, q, k, v, texts, dt, f"{(nq, heads, kvh, d, lens, dt, mask)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,nq,heads,kvh,d", [(13, 22, 8, 2, 128), (5, 40, 3, 3, 40), (3, 300, 8, 1, 256), (9, 200, 2, 1, 120), (7, 33, 2, 2, 200)])
def test_cross_attention_short_texts(ops, n, nq, heads, kvh, d, dt):
    """Texts of at most one tile, few and many groups of rows: right, and the same bits beside a longer text."""
    lens = [1 + (7 * i) % 32 for i in range(n)]
    q, k, v, hi, kw, texts = _attn_case(n + d, dt, n, nq, heads, kvh, d, lens, False, 0.1)
    got = ops.cross_attention(q, k, v, hi, **kw)
    _check_attn(got, q, k, v, texts, dt, f"{(n, nq, heads, kvh, d, dt)}")
    assert torch.equal(ops.cross_attention(q, k, v, 90, **kw), got)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("nq,d", [(1, 16), (2, 72), (1, 136)])
def test_cross_attention_joins_many_ranges(ops, nq, d, dt):
    """More ranges than a wave has lanes, beside texts of one and of exactly 64."""
    q, k, v, hi, kw, texts = _attn_case(d, dt, 4, nq, 1, 1, d, [70001, 65536, 3, 66561], False, 0.0, spread=2.0)
    got = ops.cross_attention(q, k, v, hi, **kw)
    _check_attn(got, q, k, v, texts, dt, f"{(nq, d, dt)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("nq", [1, 3, 90])
def test_cross_attention_empty_texts_shared_texts_and_bad_indices(ops, nq, dt):
    index = [2, 0, 2, 1, -1, 3, 7, 0, 1 << 30]
    for pad in (False, True):
        q, k, v, hi, kw, texts = _attn_case(5, dt, 9, nq, 4, 2, 40, [50, 0, 77], pad, 0.2, index)
        kw["mask"].view(-1)[:50] = False  # text 0: every key masked
        texts = [[] if c == 0 else x for c, x in zip(index, texts)]
        got = ops.cross_attention(q, k, v, hi, **kw)
        _check_attn(got, q, k, v, texts, dt, f"{(nq, dt, pad)}")
        for i, x in enumerate(texts):
            if not x:
                assert not got[i].any()
        # lengths and starts outside the arrays are cut, not followed
        if not pad:
            n = k.shape[0]
            kw = dict(kv_start=torch.tensor([n - 5, -3, n + 4], dtype=torch.int32).cuda(),
                      kv_len=torch.tensor([1 << 30, 40, 40], dtype=torch.int32).cuda(), kv_index=kw["kv_index"])
            kf, vf = torch.nan_to_num(k), torch.nan_to_num(v)
            got = ops.cross_attention(q, kf, vf, hi, **kw)
            cut = {0: list(range(n - 5, n))}
            _check_attn(got, q, kf, vf, [cut.get(c, []) for c in index], dt, f"{(nq, dt)} cut")
        else:
            kw = dict(kv_len=torch.tensor([-4, 1 << 30, 3], dtype=torch.int32).cuda(), kv_index=kw["kv_index"])
            kf, vf = torch.nan_to_num(k), torch.nan_to_num(v)
            got = ops.cross_attention(q, kf, vf, hi, **kw)
            cut = {1: list(range(hi, 2 * hi)), 2: list(range(2 * hi, 2 * hi + 3))}
            _check_attn(got, q, kf, vf, [cut.get(c, []) for c in index], dt, f"{(nq, dt)} cut")
    q = torch.randn(2, nq, 4, 40, device="cuda").to(_t(dt))
    for k, hi in ((torch.zeros(2, 0, 2, 40, device="cuda").to(q.dtype), 0), (torch.zeros(2, 6, 2, 40, device="cuda").to(q.dtype), 6)):
        got = ops.cross_attention(q, k, k, hi, kv_len=torch.zeros(2, dtype=torch.int32, device="cuda"))
        assert got.shape == q.shape and not got.any()
    assert ops.cross_attention(q[:0], k[:0], k[:0], 6).shape == (0, nq, 4, 40)
    assert ops.cross_attention(q[:, :0], k, k, 6).shape == (2, 0, 4, 40)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("nq,hi", [(1, 90), (1, 1500), (50, 90)])
def test_cross_attention_layouts(ops, nq, hi, dt):
    """Heads before queries, K and V as parts of one projection, K/V heads in
    their own planes, output inside a wider buffer: the same bits as contiguous tensors."""
    n, heads, kvh, d = 3, 6, 2, 40
    q, k, v, hi, kw, texts = _attn_case(hi, dt, n, nq, heads, kvh, d, [hi, 20, hi - 1], True, 0.2)
    whole = ops.cross_attention(q, k, v, hi, **kw)
    _check_attn(whole, q, k, v, texts, dt, f"{(nq, hi, dt)}")
    q2 = q.transpose(1, 2).contiguous().transpose(1, 2)
    kv = torch.stack((k, v), 2)
    assert torch.equal(ops.cross_attention(q2, kv[:, :, 0], kv[:, :, 1], hi, **kw), whole)
    k2, v2 = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (k, v))
    out = torch.full((n, nq + 1, heads + 1, 64), 5.0, device="cuda").to(q.dtype)
    ops.cross_attention(q, k2, v2, hi, out=out[:, :nq, 1:, 8:48], **kw)
    assert torch.equal(out[:, :nq, 1:, 8:48], whole)
    out[:, :nq, 1:, 8:48] = 5
    assert (out == 5).all()
    odd = q.new_empty(3 * nq * heads * d + 64).as_strided((1, nq, heads, d), (13, heads * d, d, 1))  # a stride that nothing steps by
    odd.copy_(q[:1])
    kw1 = dict(kw, kv_len=kw["kv_len"][:1], mask=kw["mask"][:1])
    assert torch.equal(ops.cross_attention(odd, k[:1], v[:1], hi, **kw1), whole[:1])
    one = k[:, :, :1].expand(n, hi, kvh, d)  # a shared head: stride 0
    ref = ops.cross_attention(q, one.contiguous(), v, hi, **kw)
    assert torch.equal(ops.cross_attention(q, one, v, hi, **kw), ref)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("nq", [1, 4, 70])
def test_cross_attention_rows_do_not_depend_on_their_batch(ops, nq, dt):
    lens = [77, 1300, 5, 0, 640, 2600]
    q, k, v, hi, kw, texts = _attn_case(4, dt, 6, nq, 4, 2, 64, lens, False, 0.1)
    whole = ops.cross_attention(q, k, v, hi, **kw)
    for i, c in enumerate(lens):
        part = ops.cross_attention(q[i:i + 1], k, v, max(c, 1), kv_start=kw["kv_start"][i:i + 1], kv_len=kw["kv_len"][i:i + 1],
                                   mask=kw["mask"])
        assert torch.equal(part[0], whole[i]), c


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 40, 96, 120, 160, 256])
def test_cross_attention_bits_do_not_depend_on_the_longest_text(ops, d, dt):
    for nq, heads, kvh in ((1, 3, 3), (2, 8, 2), (40, 2, 2), (200, 2, 1), (530, 1, 1)):
        q, k, v, hi, kw, texts = _attn_case(d + nq, dt, 4, nq, heads, kvh, d, [30, 1, 60, 17], False, 0.2)
        first = ops.cross_attention(q, k, v, hi, **kw)
        _check_attn(first, q, k, v, texts, dt, f"{(nq, heads, kvh, d, dt)}")
        for most in (100, 128, 129, 600, 1100, 5000):
            assert torch.equal(ops.cross_attention(q, k, v, most, **kw), first), (nq, most)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("nq", [1, 40])
def test_cross_attention_scores_far_apart(ops, nq, dt):
    """Scores of +-200 and more: the running maximum moves late and early;
    equal keys share evenly; a negative scale."""
    n, d, hi = 2, 64, 300
    q, k, v, hi, kw, texts = _attn_case(1, dt, n, nq, 2, 2, d, [hi, hi - 7])
    k *= torch.linspace(0.1, 12, k.shape[0], device="cuda").to(k.dtype)[:, None, None]
    for scale in (0.125, -0.3, 0.0):
        _check_attn(ops.cross_attention(q, k, v, hi, scale=scale, **kw), q, k, v, texts, dt, f"{(nq, dt, scale)}", scale)


def test_cross_attention_offsets_past_32_bits(ops):
    """A packed K/V store whose rows lie beyond 2^31 elements."""
    rows, ld, d = 70000, 33024, 40  # 2.3e9 elements, 4.6 GB
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("not enough free memory")
    store = torch.empty(rows * ld, device="cuda", dtype=torch.bfloat16)
    k = store.as_strided((rows, 1, d), (ld, d, 1))
    v = store.as_strided((rows, 1, d), (ld, d, 1), 64)
    a = rows - 90
    k[a:].copy_(torch.randn(90, 1, d, device="cuda")), v[a:].copy_(torch.randn(90, 1, d, device="cuda"))
    q = torch.randn(1, 50, 1, d, device="cuda").to(torch.bfloat16)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    for nq in (1, 50):
        got = ops.cross_attention(q[:, :nq], k, v, 90, kv_start=ints(a), kv_len=ints(90))
        _check_attn(got, q[:, :nq], k[a:], v[a:], [range(90)], "bf16", f"far {nq}")


# ------------------------------------------------------------------ together
def _chain(ops, s):
    """Encoder states -> norm -> 8-bit linear layer; a pooled token per request
    and the image tokens attend to the texts; the pooled row goes on through a
    4-bit layer with the residual's norm."""
    states, res = ops.rmsnorm(s["states"], s["gamma"], 1e-6, resid=s["resid"])
    kv = states.view(-1, 2, 4, 64)
    image = ops.cross_attention(s["q"], kv[:, 0], kv[:, 1], s["hi"], kv_start=s["start"], kv_len=s["len"])
    pooled = ops.cross_attention(s["pool"], kv[:, 0], kv[:, 1], s["hi"], kv_start=s["start"], kv_len=s["len"])
    row = pooled.reshape(pooled.shape[0], -1)
    y8, sc, h = ops.rmsnorm(row, s["gamma"][:256], 1e-6, resid=s["row"], fp8=True, scale_group=128)
    out = ops.linear_rows_w4(y8, s["w"], s["ws"], 32, x_scale=sc, bias=s["bias"], silu_out=1)
    return [states, res, image, pooled, y8, sc, h, out]


def _chain_state(seed):
    g = _gen(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    lens = torch.tensor([77, 5, 1400], dtype=torch.int32)
    b = torch.bfloat16
    return dict(states=r(1482, 512).to(b), resid=r(1482, 512).to(b), gamma=1 + 0.1 * r(512), hi=1400, q=r(3, 96, 4, 64).to(b),
                pool=r(3, 1, 4, 64).to(b), start=(lens.cumsum(0).to(torch.int32) - lens).cuda(), len=lens.cuda(),
                row=r(3, 256).to(b), w=torch.randint(0, 256, (200, 128), generator=g, device="cuda", dtype=torch.uint8),
                ws=0.1 * torch.rand(200, 8, generator=g, device="cuda"), bias=r(200))


def test_a_run_of_the_operators_together(ops):
    s = _chain_state(1)
    states, res, image, pooled, y8, sc, h, out = _chain(ops, s)
    _check_norm((states, res), s["states"], s["gamma"], 1e-6, s["resid"], False, 0, "bf16", "states")
    kv, texts = states.view(-1, 2, 4, 64), [range(0, 77), range(77, 82), range(82, 1482)]
    _check_attn(image, s["q"], kv[:, 0], kv[:, 1], texts, "bf16", "image")
    _check_attn(pooled, s["pool"], kv[:, 0], kv[:, 1], texts, "bf16", "pooled")
    _check_norm((y8, sc, h), pooled.reshape(3, 256), s["gamma"][:256], 1e-6, s["row"], True, 128, "bf16", "row")
    ref, size = _w4_ref(y8, sc, s["w"], s["ws"], None, 32, s["bias"])
    _close(_np(out), ref / (1 + np.exp(-ref)), 1.2 * W4 * size + 8 * U32 * np.abs(ref), "out")


def test_the_operators_in_a_captured_graph(ops):
    """Captured once and replayed on new inputs, eager work between the replays: the eager bits every time."""
    s = _chain_state(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _chain(ops, s)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    outs = []
    for g in graphs:  # two graphs of the same inputs: no workspace of one may serve the other
        with torch.cuda.graph(g):
            outs.append(_chain(ops, s))
    for seed in (3, 4, 5):
        new = _chain_state(seed)
        for key, t in s.items():
            if torch.is_tensor(t):
                t.copy_(new[key])
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        ref = _chain(ops, s)
        torch.cuda.synchronize()
        for out in outs:
            for a, b in zip(out, ref):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_the_operators_on_two_streams(ops):
    """Two streams at once, each on its own inputs: no shared workspace."""
    states = [_chain_state(6), _chain_state(7)]
    refs = [_chain(ops, s) for s in states]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(5):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                outs[i].append(_chain(ops, states[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        for out in outs[i]:
            for a, b in zip(out, refs[i]):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_wrappers_refuse_mixed_devices(ops):
    x, cpu = torch.zeros(2, 64, device="cuda"), torch.zeros(64)
    with pytest.raises(ValueError, match="cpu"):
        ops.rmsnorm(x, cpu)
    with pytest.raises(ValueError, match="cuda"):
        ops.linear_rows_w4(x.cpu(), torch.zeros(4, 32, dtype=torch.uint8, device="cuda"), torch.zeros(4, 2, device="cuda"), 32)
