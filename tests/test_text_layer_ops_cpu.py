"""text_attention and linear_adapters without a GPU: refusals of the C entry
points (made-up addresses, never dereferenced) and of the Python wrappers (CPU
and memoryless tensors), and pins of the oracle's definitions."""
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2605_08835_amd")
from oracle import text as O  # noqa: E402
from paper_2605_08835_amd import ops  # noqa: E402

F32, BF16 = 0, 1
A = [(i + 1) << 40 for i in range(12)]  # made-up, well-aligned addresses
NAN, INF = float("nan"), float("inf")
I32 = torch.int32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(P.binding.LIB_PATH):
        pytest.skip("libsynerdiff.so not built (run __graft_entry__.build())")
    return P.lib()


def _message(lib):
    return lib.synerdiff_last_error().decode()


TA = dict(dtype=BF16, q=A[0], q_ld=192, q_head=64, q_text=0, k=A[1], k_ld=192, k_head=64, k_text=0, v=A[2], v_ld=192, v_head=64,
          v_text=0, o=A[3], o_ld=128, o_head=64, o_text=0, tokens=500, n=0, max_len=77, start=A[4], length=None, mask=A[5],
          causal=1, prefix=A[6], cap=0.0, bias=A[7], reach=9, slope=A[8], heads=2, kv_heads=1, d=64, scale=0.125, zero=1,
          stream=None)
ON = dict(n=3)


@pytest.mark.parametrize("over,status,word", [
    (dict(), 0, ""), (dict(n=3, tokens=0), 0, ""), (dict(n=3, start=None, max_len=0), 0, ""),
    (dict(dtype=2), -1, "dtype"), (dict(n=-1), -1, "shape"), (dict(heads=0), -1, "shape"), (dict(kv_heads=0), -1, "shape"),
    (dict(heads=3, kv_heads=2), -1, "shape"), (dict(d=0), -1, "shape"), (dict(d=60), -1, "shape"), (dict(max_len=-1), -1, "shape"),
    (dict(d=264), -2, "256"), (dict(heads=1 << 17), -2, "2^16"), (dict(max_len=(1 << 30) + 1), -2, "2^30"),
    (dict(tokens=-1), -1, "token"), (dict(tokens=1 << 31), -1, "token"), (dict(length=A[9]), -1, "lengths"),
    (dict(causal=0), -1, "prefix"), (dict(scale=NAN), -1, "scale"), (dict(scale=-INF), -1, "scale"),
    (dict(scale=1e-30), -2, "scale"), (dict(scale=-1e30), -2, "scale"), (dict(cap=-1.0), -1, "cap"), (dict(cap=NAN), -1, "cap"),
    (dict(cap=INF), -1, "cap"), (dict(cap=1e-9), -2, "cap"), (dict(cap=4097.0), -2, "cap"), (dict(reach=-1), -1, "reach"), (dict(reach=(1 << 24) + 1), -1, "reach"),
    (dict(bias=None), -1, "reach"),
    (dict(ON, q_ld=(1 << 23) + 8), -2, "2^23"), (dict(ON, q=None), -1, "NULL"), (dict(ON, k=None), -1, "NULL"),
    (dict(ON, v=None), -1, "NULL"), (dict(ON, o=None), -1, "NULL"), (dict(ON, q_ld=196), -1, "16 bytes"),
    (dict(ON, q_head=-64), -1, "16 bytes"), (dict(ON, dtype=F32, v_ld=194), -1, "16 bytes"),
    (dict(ON, start=None, k_text=1001), -1, "16 bytes"), (dict(ON, k=A[1] + 8), -1, "aligned"), (dict(ON, o_ld=0), -1, "overlaps itself"),
    (dict(ON, o_head=0), -1, "overlaps itself"), (dict(ON, start=None), -1, "overlaps itself"),
    (dict(ON, start=A[4] + 2), -1, "aligned"), (dict(ON, bias=A[7] + 1), -1, "aligned"), (dict(ON, o=A[2]), -1, "overlap"),
    (dict(n=1 << 19), -2, "too many"), (dict(n=1 << 18, max_len=1 << 20), -2, "too many"),
])
def test_text_attention_refusals(lib, over, status, word):
    assert lib.synerdiff_op_text_attention(*dict(TA, **over).values()) == status
    assert word in _message(lib) or status == 0


LA = dict(dtype=BF16, x=A[0], M=0, K=64, w=A[1], N=48, down=A[2], up=A[3], rank=8, count=2, scale=A[4], index=A[5], group=1,
          bias=A[6], out=A[7], out_ld=48, scratch=A[8], floats=1 << 20, stream=None)
M9 = dict(M=9)


@pytest.mark.parametrize("over,status,word", [
    (dict(), 0, ""), (dict(M=9, N=0, out_ld=0), 0, ""),
    (dict(dtype=2), -1, "dtype"), (dict(M=-1), -1, "shape"), (dict(K=0), -1, "shape"), (dict(K=60), -1, "shape"),
    (dict(N=44), -1, "shape"), (dict(N=-8), -1, "shape"), (dict(rank=0), -1, "shape"), (dict(rank=12), -1, "shape"),
    (dict(count=-1), -1, "shape"), (dict(group=0), -1, "shape"),
    (dict(K=(1 << 20) + 8), -2, "2^20"), (dict(N=(1 << 20) + 8), -2, "2^20"), (dict(rank=1032), -2, "1024"),
    (dict(K=1 << 16, N=1 << 14), -2, "2^31"), (dict(dtype=F32, K=1 << 15, N=1 << 14), -2, "2^31"),
    (dict(M=(1 << 26) + 1), -2, "rows"), (dict(M=1 << 26, N=1 << 10), -2, "rows"), (dict(M=1 << 26, rank=128), -2, "rows"),
    (dict(M9, x=None), -1, "NULL"), (dict(M9, w=None), -1, "NULL"), (dict(M9, down=None), -1, "NULL"), (dict(M9, up=None), -1, "NULL"),
    (dict(M9, index=None), -1, "NULL"), (dict(M9, out=None), -1, "NULL"), (dict(M9, out_ld=40), -1, "stride"),
    (dict(M9, out_ld=52), -1, "aligned"), (dict(M9, dtype=F32, out_ld=50), -1, "aligned"), (dict(M9, x=A[0] + 8), -1, "aligned"),
    (dict(M9, up=A[3] + 2), -1, "aligned"), (dict(M9, bias=A[6] + 4), -1, "aligned"), (dict(M9, index=A[5] + 2), -1, "aligned"),
    (dict(M9, out=A[0]), -1, "overlap"), (dict(M9, out=A[3]), -1, "overlap"),
    (dict(M9, scratch=None), -4, "scratch"), (dict(M9, floats=71), -4, "scratch"), (dict(M9, scratch=A[8] + 4), -1, "scratch"),
])
def test_linear_adapters_refusals(lib, over, status, word):
    assert lib.synerdiff_op_linear_adapters(*dict(LA, **over).values()) == status
    assert word in _message(lib) or status == 0


def test_linear_adapters_scratch(lib):
    f = lib.synerdiff_op_linear_adapters_scratch_floats
    assert f(BF16, 8, 8) == 0 and f(BF16, 9, 8) == 72 and f(BF16, 100, 16) == 1600 and f(F32, 64, 8) == 512
    assert f(F32, 4, 16) == 0 and f(F32, 65, 8) == 520 and f(F32, 1 << 20, 8) == 0 and f(F32, 1 << 20, 24) == 24 << 20 and f(F32, 2047, 8) == 16376 and f(BF16, 1 << 20, 8) == 1 << 23
    assert f(BF16, 0, 8) == 0 and f(2, 10, 16) == 0 and f(BF16, -3, 8) == 0


def _z(*shape, t=torch.bfloat16):
    return torch.zeros(*shape, dtype=t)


def test_text_attention_wrapper_refusals():
    f = torch.float32
    q, k, start = _z(40, 4, 16), _z(40, 2, 16), _z(4, t=I32)
    qp, kp = _z(3, 11, 4, 16), _z(3, 11, 2, 16)
    packed, padded = dict(q=q, k=k, v=k, max_len=11, start=start), dict(q=qp, k=kp, v=kp, max_len=11)
    for base, kw in ((packed, dict(start=start.long())), (packed, dict(start=start[:0])), (packed, dict(start=start.view(2, 2))),
                     (packed, dict(length=start[:3])), (packed, dict(q=qp)), (packed, dict(k=kp)), (packed, dict(v=_z(39, 2, 16))),
                     (packed, dict(k=_z(39, 2, 16), v=_z(39, 2, 16))), (packed, dict(k=_z(40, 2, 24), v=_z(40, 2, 24))),
                     (packed, dict(q=_z(40, 16, 4).transpose(1, 2))), (packed, dict(mask=_z(39, t=torch.bool))),
                     (packed, dict(mask=_z(40, t=f))), (packed, dict(prefix=_z(4, t=I32))), (packed, dict(cap=0.0)),
                     (packed, dict(cap=-2.0)), (packed, dict(bias=_z(4, 8, t=f))), (packed, dict(bias=_z(2, 9, t=f))),
                     (packed, dict(bias=_z(4, 9))), (packed, dict(bias=_z(9, 4, t=f).t())), (packed, dict(slope=_z(2, t=f))),
                     (packed, dict(slope=_z(4))), (packed, dict(out=_z(40, 4, 16, t=f))), (packed, dict(out=_z(39, 4, 16))),
                     (packed, dict(out=_z(40, 16, 4).transpose(1, 2))), (packed, dict()),  # the last: not on a GPU
                     (padded, dict(max_len=12)), (padded, dict(length=_z(2, t=I32))), (padded, dict(mask=_z(33, t=torch.bool))),
                     (padded, dict(k=kp.float(), v=kp.float())), (padded, dict())):
        with pytest.raises(ValueError):
            ops.text_attention(**dict(base, **kw))
    with pytest.raises(TypeError):
        ops.text_attention(**dict(packed, q=q.half()))


def test_linear_adapters_wrapper_refusals():
    f = torch.float32
    x, w, down, up, index = _z(4, 64), _z(48, 64), _z(2, 8, 64), _z(2, 48, 8), _z(4, t=I32)
    for a in ((_z(64), w, down, up, index), (x, _z(48, 56), down, up, index), (x, w, _z(2, 8, 56), up, index),
              (x, w, down, _z(2, 8, 48), index), (x, w, down, _z(3, 48, 8), index), (x, w.float(), down, up, index),
              (x, w, down.float(), up, index), (_z(64, 4).t(), w, down, up, index), (x, _z(64, 48).t(), down, up, index),
              (x, w, _z(2, 64, 8).transpose(1, 2), up, index), (x, w, down, up, index.long()), (x, w, down, up, _z(3, t=I32)),
              (x, w, down, up, _z(8, t=I32)[::2]), (_z(2, 4, 64), w, down, up, _z(8, t=I32)),
              (_z(4, 0), _z(48, 0), _z(2, 8, 0), up, index), (x, w, down, up, index)):  # the last: not on a GPU
        with pytest.raises(ValueError):
            ops.linear_adapters(*a)
    for kw in (dict(scale=_z(2)), dict(scale=_z(3, t=f)), dict(bias=_z(48)), dict(bias=_z(47, t=f)), dict(out=_z(4, 47)),
               dict(out=_z(4, 48, t=f)), dict(out=_z(48, 4).t())):
        with pytest.raises(ValueError):
            ops.linear_adapters(x, w, down, up, index, **kw)
    with pytest.raises(TypeError):
        ops.linear_adapters(x.half(), w, down, up, index)


def _m(*shape, t=torch.bfloat16):
    return torch.empty(*shape, dtype=t, device="meta")


def test_sizes_past_31_bits():
    big = (1 << 32) + 8
    if not os.path.exists(P.binding.LIB_PATH):
        pytest.skip("libsynerdiff.so not built")
    for n, tokens, heads, max_len in ((2, 40, 4, big), (2, big, 4, 11), (big, 40, 4, 11), (2, 40, big, 11), (2, 40, 4, -big)):
        with pytest.raises(ValueError, match="2\\^31"):
            ops.text_attention(_m(tokens, heads, 16), _m(tokens, heads, 16), _m(tokens, heads, 16), max_len, start=_m(n + 1, t=I32))
    for M, K, N, count, rank in ((big, 64, 16, 2, 8), (4, big, 16, 2, 8), (4, 64, big, 2, 8), (4, 64, 16, big, 8), (4, 64, 16, 2, big)):
        with pytest.raises(ValueError, match="2\\^31"):
            ops.linear_adapters(_m(M, K), _m(N, K), _m(count, rank, K), _m(count, N, rank), _m(M, t=I32))


# ------------------------------------------------------------------ the oracle
def test_oracle_text_attention_closed_forms():
    rng = np.random.default_rng(0)
    q, k, v = (rng.standard_normal((7, h, 4)) for h in (4, 2, 2))
    texts = [(0, 3), (3, 4)]
    plain, _ = O.text_attention(q, k, v, texts, 0.5)
    # a text is dense attention on its own rows, as the other oracle has it
    for first, size in texts:
        rows = list(range(first, first + size))
        ref, _ = O.cross_attention(q[None, first:first + size], k, v, [rows], 0.5)
        assert np.allclose(plain[first:first + size], ref[0], atol=1e-13)
    causal, _ = O.text_attention(q, k, v, texts, 0.5, causal=True)
    for first, size in texts:
        assert np.allclose(causal[first], np.repeat(v[first], 2, 0)) and np.allclose(causal[first + size - 1], plain[first + size - 1])
    assert np.allclose(O.text_attention(q, k, v, texts, 0.5, causal=True, prefix=[3, 9])[0], plain)
    # -inf past a distance of 0 leaves each token itself; a constant changes nothing; a wide cap neither
    near = np.full((4, 3), -INF)
    near[:, 1] = 2.0
    assert np.allclose(O.text_attention(q, k, v, texts, 0.5, bias=near)[0], np.repeat(v, 2, 1))
    assert np.allclose(O.text_attention(q, k, v, texts, 0.5, bias=np.full((4, 1), 3.0))[0], plain)
    assert np.allclose(O.text_attention(q, k, v, texts, 0.5, cap=1e6)[0], plain, atol=1e-9)
    # a cap of nothing weighs all keys alike; a slope is a bias that falls by it
    flat, _ = O.text_attention(q, k, v, texts, 0.5, cap=1e-12)
    assert np.allclose(flat[0], np.repeat(v[:3].mean(0), 2, 0))
    fall = -np.abs(np.arange(-3, 4))[None] * np.arange(1, 5)[:, None] * 0.3
    assert np.allclose(O.text_attention(q, k, v, texts, 0.5, slope=0.3 * np.arange(1, 5))[0],
                       O.text_attention(q, k, v, texts, 0.5, bias=fall)[0])
    none = O.text_attention(q, k, v, texts, 0.5, mask=[0] * 7)[0]
    assert not none.any()


def test_oracle_linear_adapters_is_a_merged_weight():
    rng = np.random.default_rng(1)
    x, w, b = rng.standard_normal((5, 6)), rng.standard_normal((4, 6)), rng.standard_normal(4)
    down, up, scale = rng.standard_normal((2, 3, 6)), rng.standard_normal((2, 4, 3)), np.asarray([0.5, -2.0])
    y, s, t = O.linear_adapters(x, w, down, up, [0, 1, -1, 2, 1], scale, b)
    for m, c in enumerate((0, 1, None, None, 1)):
        merged = w if c is None else w + scale[c] * up[c] @ down[c]
        assert np.allclose(y[m], merged @ x[m] + b, atol=1e-13)
    assert (s + t >= np.abs(y) - 1e-12).all() and not t[2:4].any() and math.isclose(t[0, 0], 0.5 * (np.abs(up[0, 0]) @ (np.abs(down[0]) @ np.abs(x[0]))))
