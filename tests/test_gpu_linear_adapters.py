"""Linear layers with a low-rank adapter per row (linear_adapters) on the GPU
against the oracle's float64 definition.  Tolerances count roundings."""
import math

import numpy as np
import pytest

from oracle import text as O
from tests.test_gpu_text_ops import NAN, U16, U32, _close, _gen, _np, _t, ops  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _case(seed, dt, M, K, N, rank, count):
    g = _gen(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, w = r(M, K).to(_t(dt)), (r(N, K) / math.sqrt(K)).to(_t(dt))
    down, up = (r(count, rank, K) / math.sqrt(K)).to(_t(dt)), r(count, N, rank).to(_t(dt))
    return x, w, down, up, 0.5 + torch.rand(count, generator=g, device="cuda"), r(N)


def _order(kind, M, count, seed):
    """Index of every row."""
    rng = np.random.default_rng(seed)
    if kind == "runs":  # runs of uneven length, some rows without an adapter
        out = []
        while len(out) < M:
            out += [int(rng.integers(-1, count))] * int(rng.integers(1, 90))
        return np.asarray(out[:M], np.int32)
    if kind == "mixed":  # every row its own, and indices outside the adapters
        return rng.integers(-3, count + 3, M).astype(np.int32)
    return np.full(M, {"none": -1, "one": count - 1}[kind], np.int32)


def _check(got, x, w, down, up, index, scale, bias, dt, what):
    K, rank = x.shape[-1], down.shape[1]
    y, s, t = O.linear_adapters(_np(x).reshape(-1, K), _np(w), _np(down), _np(up), index, None if scale is None else _np(scale),
                                None if bias is None else _np(bias))
    # Sums of K (and of K, then rank, products): below K, K + rank roundings of the
    # terms' sizes; scale and the parts of v (2^-16) three more; the result's own.
    tol = (K + 12) * U32 * s + ((K + rank + 12) * U32 + 2.0 ** -16) * t
    tol = tol + (U16 if dt == "bf16" else U32) * (np.abs(y) + tol)
    _close(_np(got).reshape(y.shape), y, tol + 1e-37, what)


SHAPES = [
    # M, K, N, rank, count
    (1, 8, 8, 8, 1),
    (1, 320, 1280, 16, 4),
    (7, 1280, 24, 8, 3),
    (17, 72, 168, 24, 40),
    (33, 200, 320, 40, 9),
    (64, 768, 72, 128, 70),
    (65, 64, 64, 8, 2),
    (100, 8, 320, 16, 5),
    (130, 320, 40, 136, 3),
    (200, 328, 648, 32, 7),
    (257, 1000, 328, 64, 4),
    (700, 640, 1288, 16, 6),
]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N,rank,count", SHAPES)
def test_linear_adapters(ops, M, K, N, rank, count, dt):  # noqa: F811
    x, w, down, up, scale, bias = _case(M + K + N, dt, M, K, N, rank, count)
    for at, kind in enumerate(("runs", "mixed", "none", "one")):
        index = _order(kind, M, count, M + at)
        sc, b = (scale, bias) if at % 2 == 0 else (None, None)
        got = ops.linear_adapters(x, w, down, up, torch.from_numpy(index).cuda(), scale=sc, bias=b)
        _check(got, x, w, down, up, index, sc, b, dt, f"{(M, K, N, rank, count, kind, dt)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N,rank", [(16384, 64, 320, 8), (20000, 320, 64, 16), (40000, 72, 136, 24), (3000, 256, 640, 32),
                                        (9000, 640, 256, 64)])
def test_linear_adapters_many_rows(ops, M, K, N, rank, dt):  # noqa: F811
    """All tiles of the product: a sample of rows, and the first and last ones, are checked."""
    x, w, down, up, scale, bias = _case(M, dt, M, K, N, rank, 5)
    index = _order("runs", M, 5, M)
    got = ops.linear_adapters(x, w, down, up, torch.from_numpy(index).cuda(), scale=scale, bias=bias)
    rows = np.unique(np.concatenate((np.arange(40), np.arange(M - 300, M), np.random.default_rng(1).integers(0, M, 400))))
    at = torch.from_numpy(rows).cuda()
    _check(got[at], x[at], w, down, up, index[rows], scale, bias, dt, f"{(M, K, N, rank, dt)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,t,K,N", [(3, 1, 64, 64), (5, 3, 40, 72), (6, 77, 128, 320), (3, 300, 320, 64)])
def test_linear_adapters_index_per_request(ops, n, t, K, N, dt):  # noqa: F811
    x, w, down, up, scale, bias = _case(n * t, dt, n * t, K, N, 16, 3)
    index = np.asarray([(2 * i) % 4 - (i == 1) for i in range(n)], np.int32)
    x3 = x.view(n, t, K)
    got = ops.linear_adapters(x3, w, down, up, torch.from_numpy(index).cuda(), scale=scale, bias=bias)
    assert got.shape == (n, t, N)
    _check(got, x, w, down, up, np.repeat(index, t), scale, bias, dt, f"{(n, t, K, N, dt)}")
    rows = torch.from_numpy(np.repeat(index, t)).cuda()
    assert torch.equal(ops.linear_adapters(x3, w, down, up, rows.view(n, t), scale=scale, bias=bias), got)
    assert torch.equal(ops.linear_adapters(x, w, down, up, rows, scale=scale, bias=bias), got.view(n * t, N))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M", [5, 40, 300])
def test_linear_adapters_other_rows_and_adapters_do_not_matter(ops, M, dt):  # noqa: F811
    """Infinities and NaN in another row or another row's adapter stay there."""
    K, N, rank, count = 136, 200, 24, 4
    x, w, down, up, scale, bias = _case(M, dt, M, K, N, rank, count)
    index = np.arange(M, dtype=np.int32) % 5 - 1
    ix = torch.from_numpy(index).cuda()
    clean = ops.linear_adapters(x, w, down, up, ix, scale=scale, bias=bias)
    for bad in (math.inf, NAN):
        d2, u2, s2, x2 = down.clone(), up.clone(), scale.clone(), x.clone()
        d2[2], u2[2], s2[2] = bad, -bad, bad
        x2[1] = bad
        got = ops.linear_adapters(x2, w, d2, u2, ix, scale=s2, bias=bias)
        keep = torch.from_numpy((index != 2) & (np.arange(M) != 1)).cuda()
        assert torch.equal(got[keep], clean[keep])
        assert not torch.isfinite(got[~keep]).any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 30, 200])
def test_linear_adapters_out_and_empty(ops, M, dt):  # noqa: F811
    K, N = 64, 72
    x, w, down, up, scale, bias = _case(M, dt, M, K, N, 8, 2)
    ix = torch.zeros(M, dtype=torch.int32, device="cuda")
    ref = ops.linear_adapters(x, w, down, up, ix)
    wide = torch.full((M, N + 24), 7.0, device="cuda", dtype=_t(dt))
    ops.linear_adapters(x, w, down, up, ix, out=wide[:, 8:8 + N])
    assert torch.equal(wide[:, 8:8 + N], ref) and (wide[:, :8] == 7).all() and (wide[:, 8 + N:] == 7).all()
    assert torch.equal(ops.linear_adapters(x, w, down, up, ix), ref)
    assert ops.linear_adapters(x[:0], w, down, up, ix[:0]).shape == (0, N)
    assert ops.linear_adapters(x, w[:0], down, up[:, :0], ix).shape == (M, 0)
    bare = ops.linear_adapters(x, w, down[:0], up[:0], ix)
    assert torch.equal(bare, ops.linear_adapters(x, w, down, up, ix - 1))


@pytest.mark.parametrize("dt", ["bf16"])
def test_linear_adapters_past_2_31_elements(ops, dt):  # noqa: F811
    """x and out past 2^31 elements: the product runs in parts, rows at their seams are checked."""
    K, N, M = 1024, 1032, (1 << 21) + 300
    g = _gen(3)
    x = torch.empty(M, K, device="cuda", dtype=_t(dt))
    rows = np.unique(np.concatenate([np.arange(a - 3, a + 3) for a in (3, 1048320, 1 << 20, 2096640, 1 << 21, M - 3)]))
    at = torch.from_numpy(rows).cuda()
    x.zero_()
    x[at] = torch.randn(len(rows), K, generator=g, device="cuda").to(_t(dt))
    _, w, down, up, scale, bias = _case(4, dt, 1, K, N, 8, 3)
    index = (torch.arange(M, device="cuda") // 100 % 4 - 1).to(torch.int32)
    got = ops.linear_adapters(x, w, down, up, index, scale=scale, bias=bias)
    _check(got[at], x[at], w, down, up, index[at].cpu().numpy(), scale, bias, dt, "parts")


def test_linear_adapters_streams_and_graphs(ops):  # noqa: F811
    for M in (20, 500):
        x, w, down, up, scale, bias = _case(M, "bf16", M, 192, 320, 16, 4)
        ix = torch.from_numpy(_order("runs", M, 4, 1)).cuda()
        ix2 = torch.from_numpy(_order("mixed", M, 4, 2)).cuda()
        x1, x2, i1 = x.clone(), x.flip(0).contiguous(), ix.clone()
        want = {0: ops.linear_adapters(x1, w, down, up, i1, scale=scale), 1: ops.linear_adapters(x2, w, down, up, ix2, scale=scale)}
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = ops.linear_adapters(x, w, down, up, ix, scale=scale)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want[0])
        graphs = []
        for _ in range(2):  # (two graphs, each with a workspace of its own)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = ops.linear_adapters(x, w, down, up, ix, scale=scale)
            graphs.append((graph, out))
        for turn in range(6):
            x.copy_((x1, x2)[turn % 2])
            ix.copy_((i1, ix2)[turn % 2])
            for graph, out in graphs:
                graph.replay()
                assert torch.equal(out, want[turn % 2])
            assert torch.equal(ops.linear_adapters(x, w, down, up, ix, scale=scale), want[turn % 2])
            torch.cuda.synchronize()


def _same(got, y, tol, what):
    """Infinities and NaN where the definition has them, the rest within `tol`."""
    got, on = _np(got).reshape(y.shape), np.isfinite(y)
    assert np.array_equal(got[~on], y[~on], equal_nan=True), what
    assert np.isfinite(got[on]).all() and (np.abs(got - np.where(on, y, 0))[on] <= tol[on]).all(), what


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(5, 136, 200), (40, 136, 200), (300, 136, 200), (9000, 72, 320)])
def test_linear_adapters_infinite_elements(ops, M, K, N, dt):  # noqa: F811
    """One infinity in an adapter or in x gives infinities where the definition does, of its sign, and NaN nowhere."""
    rank, count = 24, 3
    x, w, down, up, scale, bias = _case(M, dt, M, K, N, rank, count)
    x, w, down, up = (t.abs() + 0.25 for t in (x, w, down, up))  # (no sum has infinities of both signs)
    x[0] = 0
    x[0, 7] = 1  # (this row's v are single elements of `down`, so bf16 holds them)
    index = np.arange(M, dtype=np.int32) % (count + 1) - 1
    index[0] = 1
    for name in ("down", "up", "x"):
        for sign, sc in ((1, None), (-1, scale)):
            t = dict(x=x.clone(), down=down.clone(), up=up.clone())
            if name == "x":
                t["x"][M - 1, 5] = sign * math.inf
            else:
                t[name][1, 5, 7] = sign * math.inf
            got = ops.linear_adapters(t["x"], w, t["down"], t["up"], torch.from_numpy(index).cuda(), scale=sc, bias=bias)
            clean = O.linear_adapters(_np(x), _np(w), _np(down), _np(up), index, None if sc is None else _np(sc), _np(bias))
            with np.errstate(invalid="ignore"):
                y = O.linear_adapters(_np(t["x"]), _np(w), _np(t["down"]), _np(t["up"]), index, None if sc is None else _np(sc),
                                      _np(bias))[0]
            y[np.isnan(y)] = sign * math.inf if name == "x" else np.nan  # (x's zero row has none)
            tol = (K + 12) * U32 * clean[1] + ((K + rank + 12) * U32 + 2.0 ** -16) * clean[2]
            tol = tol + (U16 if dt == "bf16" else U32) * (np.abs(clean[0]) + tol)
            assert np.isinf(y).any()
            _same(got, y, tol, f"{(M, K, N, dt, name, sign)}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M", [8, 40, 300])
def test_linear_adapters_largest_v(ops, M, dt):  # noqa: F811
    """v between bf16's largest value and fp32's."""
    K, N, rank = 16, 64, 16
    x, w, down, up, _, _ = _case(M, dt, M, K, N, rank, 2)
    x[:, :2], down[:] = 1, 0
    down[0, 3, 0], down[0, 3, 1] = 3.3895e38, 1e36
    down[1] = -down[0]
    up /= 16
    index = np.arange(M, dtype=np.int32) % 2
    got = ops.linear_adapters(x, w, down, up, torch.from_numpy(index).cuda())
    assert torch.isfinite(got).all()
    _check(got, x, w, down, up, index, None, None, dt, f"{(M, dt)}")


def test_linear_adapters_v_past_2_28_values(ops):  # noqa: F811
    """fp32 rows times rank past 2^28, so that v is made in more than one turn of its grid."""
    M, K, N, rank = 262400, 8, 8, 1024
    x, w, down, up, scale, bias = _case(12, "f32", M, K, N, rank, 3)
    index = _order("runs", M, 3, 12)
    got = ops.linear_adapters(x, w, down, up, torch.from_numpy(index).cuda(), scale=scale, bias=bias)
    rows = np.unique(np.concatenate((np.arange(20), np.arange(M - 300, M), np.random.default_rng(2).integers(0, M, 300))))
    at = torch.from_numpy(rows).cuda()
    _check(got[at], x[at], w, down, up, index[rows], scale, bias, "f32", "v past 2^28")


@pytest.mark.parametrize("K,N,rank", [(1032, 8, 8), (8, 1032, 24)])
def test_linear_adapters_fp32_past_2_31_elements(ops, K, N, rank):  # noqa: F811
    """x, or out, past 2^31 elements in fp32, v made by the blocks that use it and by a launch of its own."""
    M, g = (1 << 21) + 300, _gen(5)
    rows = np.unique(np.concatenate([np.arange(a - 3, a + 3) for a in (3, 1 << 20, (1 << 31) // 1032, 1 << 21, M - 3)]))
    at = torch.from_numpy(rows).cuda()
    x = torch.zeros(M, K, device="cuda")
    x[at] = torch.randn(len(rows), K, generator=g, device="cuda")
    _, w, down, up, scale, bias = _case(6, "f32", 1, K, N, rank, 3)
    index = (torch.arange(M, device="cuda") // 100 % 4 - 1).to(torch.int32)
    got = ops.linear_adapters(x, w, down, up, index, scale=scale, bias=bias)
    _check(got[at], x[at], w, down, up, index[at].cpu().numpy(), scale, bias, "f32", f"{(K, N, rank)}")


@pytest.mark.parametrize("M,K,N,rank", [(4, 8, 64, 8), (9, 8, 64, 8), (60, 16, 40, 16), (65, 8, 64, 8), (700, 8, 320, 16),
                                        (3000, 8, 64, 8), (3000, 16, 64, 24)])
def test_linear_adapters_fp32_v(ops, M, K, N, rank):  # noqa: F811
    """fp32 layers keep v in fp32: the adapter's part is as near as its sums' roundings allow."""
    x, w, down, up, scale, _ = _case(M + rank, "f32", M, K, N, rank, 3)
    w.zero_()
    index = _order("runs", M, 3, M)
    got = _np(ops.linear_adapters(x, w, down, up, torch.from_numpy(index).cuda(), scale=scale))
    y, _, t = O.linear_adapters(_np(x), _np(w), _np(down), _np(up), index, _np(scale))
    # K, then rank, products and sums (fused or not, at most a rounding each), the scale, the sum with W x = 0 and the store
    tol = (K + rank + 4) * U32 * t
    _close(got, y, tol, f"{(M, K, N, rank)}")
    if K > 8 or M < 60:
        return
    # (two bf16 parts of v, off by up to 2^-17 of it, would not pass at these sizes: 28 U32 at most is below 2^-19)
    v = np.stack([_np(scale)[c] * (_np(down)[c] @ r) if c >= 0 else np.zeros(rank) for c, r in zip(index, _np(x))])
    hi = torch.from_numpy(v).float().bfloat16().double().numpy()
    parts = hi + torch.from_numpy(v - hi).float().bfloat16().double().numpy()
    z = np.stack([_np(up)[c] @ p if c >= 0 else np.zeros(N) for c, p in zip(index, parts)])
    assert (np.abs(z - y) > tol).any()
