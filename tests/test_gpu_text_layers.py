"""A text layer of requests with styles of their own, as it is used: states ->
norm -> q, k, v with each request's adapter -> attention inside the texts ->
projection with adapters -> residual, then the denoiser's tokens attend to the
states' keys and values.  Against float64 of the same chain; eager, and captured
with lengths and indices that change between replays."""
import numpy as np
import pytest

from oracle import text as O
from tests.test_gpu_text_ops import U16, _gen, _np, ops  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

H, KVH, D, C, RANK, COUNT = 4, 2, 40, 160, 16, 3


def _weights(dt):
    g = _gen(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    wide = (H + 2 * KVH) * D
    w = dict(gamma=1 + 0.1 * r(C), qkv=r(wide, C) / C ** 0.5, out=r(C, H * D) / C ** 0.5, kv=r(2 * KVH * D, C) / C ** 0.5,
             bias=r(H, 17), scale=0.5 + torch.rand(COUNT, generator=g, device="cuda"))
    for name, k, n in (("qkv", C, wide), ("out", H * D, C)):
        w[name + "_down"], w[name + "_up"] = r(COUNT, RANK, k) / k ** 0.5, 0.3 * r(COUNT, n, RANK)
    return {i: t if i in ("gamma", "bias", "scale") else t.to(dt) for i, t in w.items()}


def _run(ops, w, x, pixels, start, index, hi):  # noqa: F811
    y = ops.rmsnorm(x, w["gamma"])
    qkv = ops.linear_adapters(y, w["qkv"], w["qkv_down"], w["qkv_up"], index, scale=w["scale"]).view(-1, H + 2 * KVH, D)
    q, k, v = qkv.split([H, KVH, KVH], 1)
    o = ops.text_attention(q, k, v, hi, start=start, causal=True, cap=20.0, bias=w["bias"])
    o = ops.linear_adapters(o.view(-1, H * D), w["out"], w["out_down"], w["out_up"], index, scale=w["scale"])
    y, h = ops.rmsnorm(o, w["gamma"], resid=x)
    none = torch.full_like(index, -1)
    kv = ops.linear_adapters(y, w["kv"], w["qkv_down"], w["qkv_up"][:, :2 * KVH * D].contiguous(), none).view(-1, 2, KVH, D)
    image = ops.cross_attention(pixels, kv[:, 0], kv[:, 1], hi, kv_start=start[:-1].contiguous(), kv_len=start[1:] - start[:-1])
    return h, image


def _ref(w, x, pixels, lens, index, dt):
    """The chain in float64, rounded where a tensor is stored."""
    rnd = (lambda a: torch.from_numpy(np.asarray(a)).to(dt).double().numpy())  # noqa: E731
    W = {i: _np(t) for i, t in w.items()}
    ends = np.cumsum([0] + lens)
    texts = [(int(a), n) for a, n in zip(ends, lens)]
    y = rnd(O.rmsnorm(_np(x), W["gamma"])[0])
    qkv = rnd(O.linear_adapters(y, W["qkv"], W["qkv_down"], W["qkv_up"], index, W["scale"])[0]).reshape(-1, H + 2 * KVH, D)
    q, k, v = qkv[:, :H], qkv[:, H:H + KVH], qkv[:, H + KVH:]
    o = rnd(O.text_attention(q, k, v, texts, D ** -0.5, causal=True, cap=20.0, bias=W["bias"])[0])
    o = rnd(O.linear_adapters(o.reshape(-1, H * D), W["out"], W["out_down"], W["out_up"], index, W["scale"])[0])
    y, h = O.rmsnorm(o, W["gamma"], resid=_np(x))
    kv = rnd(rnd(y) @ W["kv"].T).reshape(-1, 2, KVH, D)
    image = O.cross_attention(_np(pixels), kv[:, 0], kv[:, 1], [list(range(a, a + n)) for a, n in texts], D ** -0.5)[0]
    return h, image


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_text_layer_with_adapters(ops, dt):  # noqa: F811
    w = _weights(dt)
    lens = [[77, 5, 40, 1, 30], [20, 33, 50, 49, 1]]
    styles = [[0, -1, 2, 1, 2], [2, 2, -1, 0, 1]]
    tokens, hi = sum(lens[0]), 77
    g = _gen(6)
    xs = [torch.randn(tokens, C, generator=g, device="cuda").to(dt) for _ in lens]
    pixels = torch.randn(5, 30, H, D, generator=g, device="cuda").to(dt)
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    starts = [ints(np.cumsum([0] + a)) for a in lens]
    rows = [ints(np.repeat(s, a)) for s, a in zip(styles, lens)]
    eager = [_run(ops, w, x, pixels, s, r, hi) for x, s, r in zip(xs, starts, rows)]
    # Errors of a chain of seven operators: each rounds its output once (U16, or fp32
    # sums, far below) and passes on what it is given, amplified at most a few times in
    # the mean (scores of size 1, rows of unit size); the mean square takes the mean.
    bound = 7 * 3 * (U16 if dt == torch.bfloat16 else 2.0 ** -20)
    for got, x, a, r in zip(eager, xs, lens, rows):
        for one, ref in zip(got, _ref(w, x, pixels, a, r.cpu().numpy(), dt)):
            err = np.linalg.norm(_np(one) - ref) / np.linalg.norm(ref)
            assert err < bound, err
    x, start, index = xs[0].clone(), starts[0].clone(), rows[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _run(ops, w, x, pixels, start, index, hi)
    for turn in (0, 1, 1, 0, 1):
        x.copy_(xs[turn])
        start.copy_(starts[turn])
        index.copy_(rows[turn])
        graph.replay()
        for one, ref in zip(out, eager[turn]):
            assert torch.equal(one, ref)
        again = _run(ops, w, xs[turn], pixels, starts[turn], rows[turn], hi)
        assert all(torch.equal(a, b) for a, b in zip(again, eager[turn]))
        torch.cuda.synchronize()
