"""Edge values of the text-side operators on the GPU: scores of -inf, outliers
that meet a weight of zero, values near the ends of a type's range, offsets
past 32 bits.  Against the oracle's float64 definitions; U32 and U16 are half a
step of fp32 and bf16 relative to the value."""
import math

import numpy as np
import pytest

from oracle import text as O
from test_gpu_text_ops import U16, U32, _attn_case, _check_attn, _check_norm, _gen, _np, _t, ops  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ------------------------------------------------------------------ attention: scores of -inf
# n_q, heads, K/V heads, d, length: every form of the kernels, split and whole
FORMS = [(1, 1, 1, 40, 150), (8, 2, 2, 64, 150), (9, 2, 2, 64, 150), (40, 4, 2, 40, 150), (30, 1, 1, 160, 150), (100, 1, 1, 40, 30),
         (200, 2, 2, 40, 120), (200, 2, 1, 64, 150), (200, 1, 1, 128, 150), (530, 1, 1, 72, 300), (200, 1, 1, 256, 150),
         (1, 2, 2, 64, 3000), (20, 2, 2, 40, 3000), (200, 1, 1, 64, 1300)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("nq,heads,kvh,d,length", FORMS)
def test_cross_attention_minus_inf_scores(ops, nq, heads, kvh, d, length, dt):  # noqa: F811
    """Keys that score -inf take no weight, whichever tile, wave or range they
    fall to and also as the first ones; a row that no other key is left to gives zeros."""
    L = length
    dead_sets = {"first": [0], "tile": range(min(32, L - 1)), "two tiles": range(min(64, L - 1)), "most": range(L - 2),
                 "some": range(0, L, 16), "behind": range(L // 2, L), "range": range(min(1100, L - 1)), "all": range(L)}
    for name, dead in dead_sets.items():
        for overflow in (False, True):  # -inf in K; or finite q and k whose product overflows, in every other query
            q, k, v, hi, kw, _ = _attn_case(nq + d, dt, 1, nq, heads, kvh, d, [L])
            q[..., 0], k[..., 0] = 0, 0
            qz, kz = q.clone(), k.clone()
            hit = torch.ones(nq, dtype=torch.bool)
            if overflow:
                hit[1::2] = False
            q[:, hit.cuda(), :, 0] = 2e30 if overflow else 1.0
            k[list(dead), :, 0] = -1e30 if overflow else -math.inf
            got = ops.cross_attention(q, k, v, hi, **kw)
            live = [t for t in range(L) if t not in dead]
            what = f"{(nq, heads, kvh, d, L, dt, name, overflow)}"
            hit = hit.cuda()
            if live:
                _check_attn(got[:, hit], qz[:, hit], kz, v, [live], dt, what)
            else:
                assert not got[:, hit].any(), what
            if overflow and nq > 1:
                _check_attn(got[:, ~hit], qz[:, ~hit], kz, v, [range(L)], dt, what + " others")


# ------------------------------------------------------------------ 4-bit weights: outliers and the ends of the range
W4_FORMS = [(1, 320, 100), (16, 1288, 65), (33, 2184, 130), (5, 264, 4104), (40, 136, 8200), (3, 264, 16401), (20, 136, 16385)]


def _w4(g, M, K, N, group, zero):
    ng = -(-K // group)
    w = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scale = (torch.rand(N, ng, generator=g, device="cuda") + 0.5) * 0.1
    z = torch.randint(0, 16, (N, ng), generator=g, device="cuda", dtype=torch.uint8) if zero else None
    return w, scale, z, torch.randn(M, K, generator=g, device="cuda")


def _w4_bound(x, xs, w, scale, z, group, silu_in=False):
    """The result in float64 and sum |x w|.  Products are exact and summed in
    fp32, each step off by at most a unit in the last place (2 U32: the matrix
    unit's inner sums are not assumed to round to nearest) of no more than that
    sum: (3 K / 4 + 64) steps cover K products in three parts, four or more to
    a step, and the chunks' and waves' sums."""
    a = _np(x)
    if xs is not None:
        a = a * np.repeat(_np(xs), a.shape[1] if xs.shape[1] == 1 else 128, 1)[:, :a.shape[1]]
    if silu_in:
        a = a / (1 + np.exp(-a))
    wt = O.w4_weights(w.cpu().numpy(), _np(scale), None if z is None else _np(z), group)
    return a @ wt.T, np.abs(a) @ np.abs(wt).T


def _w4_close(got, ref, size, K, what, extra=0.0):
    got = _np(got)
    assert np.isfinite(got).all(), what
    err, tol = np.abs(got - ref), 2 * U32 * (0.75 * K + 64) * size + extra
    assert (err <= tol).all(), f"{what}: {err.max():.3e}, {(err / np.maximum(tol, 1e-300)).max():.2f} of the tolerance"


@pytest.mark.parametrize("xt", ["f32", "bf16", "e4m3row", "e4m3"])
@pytest.mark.parametrize("M,K,N", W4_FORMS)
def test_linear_rows_w4_outliers_on_zero_weights(ops, M, K, N, xt):  # noqa: F811
    """Channels of x some 10^4 to 10^6 times the others whose weights are all
    zero (code = zero point) leave the others' sum as exact as without them."""
    for group in (32, 64, 128):
        for zero in (False, True):
            g = _gen(M + K + N + group + zero)
            w, scale, z, x = _w4(g, M, K, N, group, zero)
            big = torch.randint(0, K, (4,), generator=g, device="cuda").tolist()
            for c in big:  # the byte's half that holds channel c takes the zero point
                zc = torch.full((N,), 8, device="cuda", dtype=torch.uint8) if z is None else z[:, c // group]
                b = w[:, c // 2]
                w[:, c // 2] = (b & 0xF0) | zc if c % 2 == 0 else (b & 0x0F) | (zc << 4)
            xs = None
            if xt.startswith("e4m3"):  # the format holds 448 beside 2^-9: a factor of 2^17 at most
                blocks = 1 if xt == "e4m3row" else -(-K // 128)
                xs = torch.rand(M, blocks, generator=g, device="cuda") + 0.5
                x = (x * 2.0 ** -6).to(torch.float8_e4m3fn)
                x[:, big] = torch.tensor(448.0, device="cuda").to(torch.float8_e4m3fn)
            else:
                x[:, big] = torch.tensor([1e4, -1e5, 1e6, 3e6], device="cuda")
                x = x.to(_t(xt))
            ref, size = _w4_bound(x, xs, w, scale, z, group)
            got = ops.linear_rows_w4(x, w, scale, group, zero=z, x_scale=xs)
            # (the e4m3 row scales and their products: 4 more roundings)
            _w4_close(got, ref, size, K, f"{(M, K, N, xt, group, zero)}", 8 * U32 * size)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", W4_FORMS)
def test_linear_rows_w4_ends_of_the_range(ops, M, K, N, xt):  # noqa: F811
    """x near the largest and the smallest numbers of its type, where the
    result is neither.  (Parts of an fp32 x end at bf16's smallest number, 2^-133.)"""
    for group, zero in ((32, True), (64, False), (128, True), (128, False)):
        g = _gen(M + K + group + zero)
        w, scale, z, x = _w4(g, M, K, N, group, zero)
        sign = torch.where(x < 0, -1.0, 1.0)
        top = (sign * torch.finfo(_t(xt)).max).to(_t(xt))
        s = scale / (4 * K)  # sum |x w| < 3.4e38 * 15 * 0.15 / 4
        ref, size = _w4_bound(top, None, w, s, z, group)
        _w4_close(ops.linear_rows_w4(top, w, s, group, zero=z), ref, size, K, f"{(M, K, N, xt, group, zero)} large")
        low = (x * 2.0 ** -118).to(_t(xt))
        ref, size = _w4_bound(low, None, w, scale * 2.0 ** 110, z, group)
        extra = 2.0 ** -133 * K * 15 * 0.15 * 2.0 ** 110 if xt == "f32" else 0.0
        _w4_close(ops.linear_rows_w4(low, w, scale * 2.0 ** 110, group, zero=z), ref, size, K, f"{(M, K, N, xt, group, zero)} small", extra)


# ------------------------------------------------------------------ rmsnorm: squares past fp32's range
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 7, 16, 40, 129, 320, 1280, 2056, 5000, 8192, 16384])
def test_rmsnorm_large_rows(ops, C, dt):  # noqa: F811
    """Rows of 1e19 to 1e38, whole or in one value, beside ordinary ones; the residual alike."""
    g = _gen(C)
    rows = 37
    x = torch.randn(rows, C, generator=g, device="cuda").clamp(-3, 3)
    r = torch.randn(rows, C, generator=g, device="cuda").clamp(-3, 3)
    x[::4] *= 1e38
    x[1::8] *= 2e19
    x[2::8, C // 2] = -2e30
    r[::4] *= 1e10
    r[3::8] *= 3e25
    x, r, gamma = x.to(_t(dt)), r.to(_t(dt)), 1 + 0.1 * torch.randn(C, generator=g, device="cuda")
    for eps in (1e-6, 0.0, 1e30):
        for resid in (None, r):
            for fp8, group in ((False, 0), (True, 0), (True, 128)):
                got = ops.rmsnorm(x, gamma, eps, resid=resid, fp8=fp8, scale_group=group)
                _check_norm(got, x, gamma, eps, resid, fp8, group, dt, f"{(C, dt, eps, resid is not None, fp8, group)}")


@pytest.mark.parametrize("C", [16, 96, 160, 320, 2056, 5000])
def test_rmsnorm_e4m3_codes_are_of_the_quotient(ops, C):  # noqa: F811
    """y8 = e4m3(y / s) to the bit, with values near the middle between two
    codes, where a product with a rounded 1 / s falls on the other side.  (These
    widths are normed alike with and without an 8-bit output, so fp32's y is the y.)"""
    g = _gen(C)
    x = torch.ones(64, C, device="cuda") * (1 + torch.rand(64, 1, generator=g, device="cuda"))
    for turn in range(6):
        middle = 17.0 + 2 * torch.randint(0, 4, (C,), generator=g, device="cuda")
        middle *= torch.exp2(torch.randint(-6, 5, (C,), generator=g, device="cuda").float())
        middle[::16] = 448  # (every block's largest: s is about 1 times the factor below)
        gamma = middle * (1 + torch.rand(1, generator=g, device="cuda"))
        y = ops.rmsnorm(x, gamma, 1e-6)
        for group in (0, 128) if C > 256 or C < 128 else (0,):
            q, s = ops.rmsnorm(x, gamma, 1e-6, fp8=True, scale_group=group)
            full = s.repeat_interleave(group or C, 1)[:, :C]
            assert torch.equal(s[:, 0].cpu(), y[:, :group or C].abs().amax(1).cpu() / 448)
            assert torch.equal(q.cpu().view(torch.uint8), (y.cpu() / full.cpu()).to(torch.float8_e4m3fn).view(torch.uint8)), (C, turn, group)


def test_rmsnorm_e4m3_infinite_scale(ops):  # noqa: F811
    """A row whose y is infinite: its scale is, the finite values' codes are 0."""
    gamma = torch.ones(384, device="cuda")
    gamma[100] = math.inf
    for group, cols in ((0, 384), (128, 128)):
        q, s = ops.rmsnorm(torch.ones(3, 384, device="cuda"), gamma, fp8=True, scale_group=group)
        q, rest = q.float(), [i for i in range(cols) if i != 100]
        assert torch.isinf(s[:, 0]).all() and torch.isnan(q[:, 100]).all() and not q[:, rest].any()


# ------------------------------------------------------------------ sizes past 2^31
def _room(gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip("not enough free memory")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rmsnorm_more_rows_than_one_launch(ops, dt):  # noqa: F811
    """More than 2^23 rows: the same bits as each part alone, right at the seam."""
    _room(16)
    g = _gen(9)
    rows, C, seam = (1 << 23) + 133, 24, 1 << 23
    x, r = (torch.randn(rows, C, generator=g, device="cuda").to(_t(dt)) for _ in range(2))
    gamma = 1 + 0.1 * torch.randn(C, generator=g, device="cuda")
    for fp8 in (False, True):
        whole = ops.rmsnorm(x, gamma, 1e-6, resid=r, fp8=fp8)
        for a, b in ((0, 1000), (seam - 77, seam + 77), (seam, rows), (rows - 1, rows)):
            part = ops.rmsnorm(x[a:b], gamma, 1e-6, resid=r[a:b], fp8=fp8)
            for w, p in zip(whole, part):
                assert torch.equal(w[a:b].view(torch.uint8), p.view(torch.uint8)), (fp8, a)
        _check_norm(tuple(w[seam - 9:seam + 9] for w in whole), x[seam - 9:seam + 9], gamma, 1e-6, r[seam - 9:seam + 9], fp8, 0, dt, f"seam {fp8}")


@pytest.mark.parametrize("xt,M,K,N", [("bf16", 5, 32768, 140003), ("bf16", 20, 262400, 16400), ("f32", 3, 262400, 16383),
                                      ("f32", 2, 32768, 140003), ("e4m3", 3, 32768, 140003)])
def test_linear_rows_w4_codes_past_2_31_bytes(ops, xt, M, K, N):  # noqa: F811
    _room(16)
    g = _gen(K)
    w, scale, z, x = _w4(g, M, K, N, 128, True)
    assert w.numel() > 1 << 31
    x, xs = (x.to(_t(xt)), None) if xt != "e4m3" else (x.to(torch.float8_e4m3fn), torch.ones(M, 1, device="cuda"))
    got = ops.linear_rows_w4(x, w, scale, 128, zero=z, x_scale=xs)
    seam = (1 << 31) // (K // 2)
    for a in (0, seam - 20, N - 40):
        ref, size = _w4_bound(x, xs, w[a:a + 40], scale[a:a + 40], z[a:a + 40], 128)
        _w4_close(got[:, a:a + 40], ref, size, K, f"{(xt, M, K, N, a)}", 8 * U32 * size)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_cross_attention_keys_past_2_31_elements(ops, dt):  # noqa: F811
    """K and V rows behind 2^31 elements, for every form of the kernels."""
    rows, ld, d, L = 70000, 33024, 40, 200
    _room(16)
    store = torch.empty(rows * ld, device="cuda", dtype=_t(dt))
    k, v = store.as_strided((rows, 1, d), (ld, d, 1)), store.as_strided((rows, 1, d), (ld, d, 1), 64)
    a = rows - L
    g = _gen(3)
    for t in (k, v):
        t[a:].copy_(torch.randn(L, 1, d, generator=g, device="cuda"))
    q = torch.randn(1, 530, 1, d, generator=g, device="cuda").to(_t(dt))
    ints = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    for nq, most in ((1, L), (8, L), (40, L), (200, 90), (200, L), (530, L), (1, 5000), (40, 5000), (200, 5000)):
        n = min(most, L)
        got = ops.cross_attention(q[:, :nq], k, v, most, kv_start=ints(a), kv_len=ints(n))
        _check_attn(got, q[:, :nq], k[a:a + n], v[a:a + n], [range(n)], dt, f"far {(dt, nq, most)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("nq,most", [(300, 60), (300, 150), (300, 700), (128, 150)])
def test_cross_attention_queries_past_2_31_elements(ops, nq, most, dt):  # noqa: F811
    """Queries and results 2^23 elements apart, two images."""
    ld, d, heads = 1 << 23, 24, 2
    img = nq * ld + 64
    _room(64)
    qs, os = (torch.empty(2 * img, device="cuda", dtype=_t(dt)).as_strided((2, nq, heads, d), (img, ld, 32, 1)) for _ in range(2))
    g = _gen(nq)
    q = torch.randn(2, nq, heads, d, generator=g, device="cuda").to(_t(dt))
    k, v = (torch.randn(2, 60, 1, d, generator=g, device="cuda").to(_t(dt)) for _ in range(2))
    qs.copy_(q)
    pad = lambda t: torch.nn.functional.pad(t, (0, 0, 0, 0, 0, most - 60))  # noqa: E731
    kw = dict(kv_len=torch.tensor([60, 41], dtype=torch.int32, device="cuda"))
    ops.cross_attention(qs, pad(k), pad(v), most, out=os, **kw)
    assert torch.equal(os.contiguous(), ops.cross_attention(q, pad(k), pad(v), most, **kw))
    _check_attn(os, q, k, v, [range(60), range(60, 101)], dt, f"{(nq, most, dt)}")


# ------------------------------------------------------------------ together
def test_states_to_8_bits_to_4_bit_layer_to_attention(ops):  # noqa: F811
    """Encoder states -> norm to 8 bits -> 4-bit layer to K and V -> queries and
    pooled tokens over the ragged texts, every step against its own inputs."""
    g = _gen(21)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    lens = torch.tensor([77, 5, 300], dtype=torch.int32)
    start, tokens, b = (lens.cumsum(0).to(torch.int32) - lens), int(lens.sum()), torch.bfloat16
    states, resid, gamma = r(tokens, 384).to(b), r(tokens, 384).to(b), 1 + 0.1 * r(384)
    y8, sc, h = ops.rmsnorm(states, gamma, 1e-6, resid=resid, fp8=True, scale_group=128)
    _check_norm((y8, sc, h), states, gamma, 1e-6, resid, True, 128, "bf16", "states")
    w, ws, z, _ = _w4(g, 1, 384, 2 * 2 * 40, 64, True)
    kv = ops.linear_rows_w4(y8, w, ws, 64, zero=z, x_scale=sc, out_dtype=b)
    ref, size = _w4_bound(y8, sc, w, ws, z, 64)
    _w4_close(kv, ref, size, 384, "K and V", 8 * U32 * size + U16 * np.abs(ref) * (1 + 1e-3))
    k, v = kv.view(tokens, 2, 2, 40).unbind(1)
    k = k * 0.05  # (scores of order 1)
    texts = [range(int(s), int(s + n)) for s, n in zip(start, lens)]
    for nq in (1, 200):
        q = r(3, nq, 6, 40).to(b)
        got = ops.cross_attention(q, k, v, 300, kv_start=start.cuda(), kv_len=lens.cuda())
        _check_attn(got, q, k, v, texts, "bf16", f"attention {nq}")
