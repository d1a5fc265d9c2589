"""Refusals of the text-side operators (rmsnorm, linear_rows_w4,
cross_attention): bad arguments are turned away before any GPU work, by the
C entry points (made-up addresses, never dereferenced) and by the Python
wrappers (CPU tensors).  CPU only."""
import os

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2605_08835_amd")
from paper_2605_08835_amd import ops  # noqa: E402

F32, BF16, E4M3 = 0, 1, 2
A = [(i + 1) << 40 for i in range(12)]  # made-up, well-aligned addresses


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(P.binding.LIB_PATH):
        pytest.skip("libsynerdiff.so not built (run __graft_entry__.build())")
    return P.lib()


def _message(lib):
    return lib.synerdiff_last_error().decode()


RMS = dict(dtype=BF16, x=A[0], x_ld=64, resid=A[1], resid_ld=64, sum=A[2], sum_ld=64, gamma=A[3], eps=1e-6, tokens=0,
           C=64, y_type=BF16, y=A[4], y_ld=64, scale=None, group=0, stream=None)


@pytest.mark.parametrize("over,status,word", [
    (dict(), 0, ""),
    (dict(dtype=2), -1, "dtype"), (dict(dtype=F32, y_type=BF16), -1, "y_type"), (dict(y_type=3), -1, "y_type"),
    (dict(tokens=-1), -1, "shape"), (dict(C=0), -1, "shape"), (dict(C=16385), -2, "16384"),
    (dict(tokens=1 << 31), -2, "2^31"), (dict(eps=-1e-6), -1, "eps"), (dict(eps=float("nan")), -1, "eps"),
    (dict(resid=None), -1, "sum without resid"),
    (dict(scale=A[5]), -1, "scale"), (dict(group=128), -1, "scale"),
    (dict(y_type=E4M3, scale=A[5], group=64), -1, "scale_group"),
    (dict(tokens=5, x=None), -1, "NULL"), (dict(tokens=5, y=None), -1, "NULL"),
    (dict(tokens=5, y_type=E4M3), -1, "NULL"),
    (dict(tokens=5, x_ld=63), -1, "stride"), (dict(tokens=5, resid_ld=1), -1, "stride"),
    (dict(tokens=5, sum_ld=0), -1, "stride"), (dict(tokens=5, y_ld=-64), -1, "stride"),
    (dict(tokens=5, x=A[0] + 1), -1, "aligned"), (dict(tokens=5, dtype=F32, y_type=F32, y=A[4] + 2), -1, "aligned"),
    (dict(tokens=5, gamma=A[3] + 2), -1, "aligned"),
    (dict(tokens=5, sum=A[0], sum_ld=72), -1, "overlap"), (dict(tokens=5, y=A[1], y_ld=80), -1, "overlap"),
    (dict(tokens=5, y=A[2]), -1, "overlap"), (dict(tokens=5, y_type=E4M3, scale=A[5], y=A[0]), -1, "overlap"),
])
def test_rmsnorm_refusals(lib, over, status, word):
    assert lib.synerdiff_op_rmsnorm(*dict(RMS, **over).values()) == status
    assert word in _message(lib) or status == 0


W4 = dict(x_type=BF16, x=A[0], x_ld=64, x_scale=None, x_group=0, M=0, K=64, w=A[1], group=32, scale_type=BF16,
          scale=A[2], zero=A[3], bias=A[4], add=A[5], silu_in=0, silu_out=0, out_type=F32, out=A[6], out_ld=48, N=48,
          stream=None)


@pytest.mark.parametrize("over,status,word", [
    (dict(), 0, ""), (dict(M=4, N=0), 0, ""),
    (dict(x_type=3), -1, "dtype"), (dict(scale_type=2), -1, "dtype"), (dict(out_type=2), -1, "dtype"),
    (dict(K=0), -1, "shape"), (dict(K=60), -1, "shape"), (dict(M=-1), -1, "shape"), (dict(N=-1), -1, "shape"),
    (dict(M=(1 << 19) + 1), -2, "2^19"), (dict(K=(1 << 24) + 8), -2, "2^24"), (dict(N=(1 << 24) + 1), -2, "2^24"),
    (dict(M=4, x_ld=(1 << 24) + 8), -2, "2^24"),
    (dict(group=0), -1, "group"), (dict(group=48), -1, "group"), (dict(group=256), -1, "group"),
    (dict(x_scale=A[7]), -1, "x_group"), (dict(x_group=128), -1, "x_group"),
    (dict(x_type=E4M3, x_scale=A[7], x_group=64), -1, "x_group"), (dict(x_type=E4M3, x_scale=A[7], silu_in=1), -2, "silu"),
    (dict(M=4, x=None), -1, "NULL"), (dict(M=4, w=None), -1, "NULL"), (dict(M=4, scale=None), -1, "NULL"),
    (dict(M=4, out=None), -1, "NULL"), (dict(M=4, x_type=E4M3), -1, "NULL"),
    (dict(M=4, x_ld=56), -1, "stride"), (dict(M=4, out_ld=47), -1, "stride"),
    (dict(M=4, x=A[0] + 8), -1, "aligned"), (dict(M=4, x_ld=68), -1, "aligned"), (dict(M=4, w=A[1] + 2), -1, "aligned"),
    (dict(M=4, x_type=E4M3, x_scale=A[7], x=A[0] + 4), -1, "aligned"), (dict(M=4, scale=A[2] + 1), -1, "aligned"),
    (dict(M=4, out=A[6] + 2), -1, "aligned"), (dict(M=4, bias=A[4] + 1), -1, "aligned"),
    (dict(M=4, add=A[6], out_ld=56), -1, "overlap"), (dict(M=4, add=A[6], out_type=BF16), -1, "overlap"),
    (dict(M=4, out=A[0]), -1, "overlap"),
])
def test_linear_rows_w4_refusals(lib, over, status, word):
    assert lib.synerdiff_op_linear_rows_w4(*dict(W4, **over).values()) == status
    assert word in _message(lib) or status == 0


XA = dict(dtype=BF16, q=A[0], q_ld=128, q_head=64, q_img=1280, k=A[1], k_ld=128, k_head=64, k_ctx=128 * 77, v=A[2],
          v_ld=128, v_head=64, v_ctx=128 * 77, kv_tokens=500, n_ctx=3, max_len=77, start=A[3], len=A[4], index=None,
          mask=A[5], o=A[6], o_ld=128, o_head=64, o_img=1280, n=3, heads=2, kv_heads=2, d=64, n_q=0, scale=0.125,
          scratch=None, floats=0, stream=None)


@pytest.mark.parametrize("over,status,word", [
    (dict(), 0, ""), (dict(n=0, n_q=5), 0, ""),
    (dict(dtype=2), -1, "dtype"), (dict(heads=3), -1, "shape"), (dict(d=60), -1, "shape"), (dict(d=0), -1, "shape"),
    (dict(d=264), -2, "shape"), (dict(heads=1 << 17), -2, "2^16"), (dict(max_len=(1 << 30) + 1), -2, "2^30"),
    (dict(n_q=9, k_ld=(1 << 23) + 8), -2, "2^23"), (dict(n_q=1 << 30), -2, "too many"),
    (dict(n=1 << 22, n_ctx=1 << 22, n_q=9), -2, "too many"), (dict(n=-1), -1, "shape"), (dict(n_q=-1), -1, "shape"), (dict(max_len=-1), -1, "shape"),
    (dict(kv_heads=0), -1, "shape"), (dict(n_ctx=-1), -1, "context"), (dict(kv_tokens=-1), -1, "context"),
    (dict(kv_tokens=1 << 31), -1, "context"), (dict(n_ctx=2), -1, "fewer contexts"),
    (dict(scale=float("nan")), -1, "scale"), (dict(scale=float("inf")), -1, "scale"),
    (dict(n_q=9, q=None), -1, "NULL"), (dict(n_q=9, v=None), -1, "NULL"), (dict(n_q=9, o=None), -1, "NULL"),
    (dict(n_q=9, q_ld=132), -1, "16 bytes"), (dict(n_q=9, k_head=-64), -1, "16 bytes"),
    (dict(n_q=9, start=None, v_ctx=1001), -1, "16 bytes"), (dict(n_q=9, dtype=F32, o_img=1282), -1, "16 bytes"),
    (dict(n_q=9, k=A[1] + 8), -1, "aligned"), (dict(n_q=9, o_head=0), -1, "overlaps itself"),
    (dict(n_q=9, len=A[4] + 2), -1, "aligned"), (dict(n_q=9, o=A[0]), -1, "overlap"),
])
def test_cross_attention_refusals(lib, over, status, word):
    assert lib.synerdiff_op_cross_attention(*dict(XA, **over).values()) == status
    assert word in _message(lib) or status == 0


def _z(*shape, t=torch.bfloat16):
    return torch.zeros(*shape, dtype=t)


def test_rmsnorm_wrapper_refusals():
    x = _z(4, 64)
    for kw in (dict(gamma=_z(64)), dict(gamma=_z(63, t=torch.float32)), dict(resid=_z(4, 63)),
               dict(resid=_z(4, 64, t=torch.float32)), dict(sum_out=x), dict(resid=x, sum_out=_z(4, 8)),
               dict(scale_group=128), dict(fp8=True, scale_group=64), dict(out=_z(4, 63)),
               dict(fp8=True, out=_z(4, 64)), dict(out=_z(4, 64, t=torch.float32)), dict()):  # the last: not on a GPU
        with pytest.raises(ValueError):
            ops.rmsnorm(x, **kw)
    for bad in (_z(4, 64).t(), _z(2, 4, 64)[:, :, ::2], _z(2, 4, 64).transpose(0, 1)):
        with pytest.raises(ValueError):
            ops.rmsnorm(bad)
    with pytest.raises(TypeError):
        ops.rmsnorm(_z(4, 64, t=torch.float16))


def test_linear_rows_w4_wrapper_refusals():
    f = torch.float32
    x, w, s = _z(4, 64), _z(48, 32, t=torch.uint8), _z(48, 2)
    for a in ((x, w, s, 48), (x, w, s, 64), (x, w, _z(2, 48).t(), 32), (x, _z(48, 31, t=torch.uint8), s, 32),
              (_z(4, 60), _z(48, 30, t=torch.uint8), s, 32), (_z(4), w, s, 32), (x, _z(48, 32, t=torch.int8), s, 32),
              (x, w, s, 32)):  # the last: not on a GPU
        with pytest.raises(ValueError):
            ops.linear_rows_w4(*a)
    for kw in (dict(zero=_z(48, 2, t=torch.int8)), dict(zero=_z(48, 1, t=torch.uint8)), dict(x_scale=_z(4, 1, t=f)),
               dict(bias=_z(48)), dict(bias=_z(47, t=f)), dict(add=_z(4, 48)), dict(add=_z(48, t=f)),
               dict(out=_z(4, 48)), dict(out=_z(4, 47, t=f))):
        with pytest.raises(ValueError):
            ops.linear_rows_w4(x, w, s, 32, **kw)
    x8 = x.to(torch.float8_e4m3fn)
    for xs in (None, _z(4, t=f), _z(4, 2, t=f), _z(3, 1, t=f), _z(4, 1)):
        with pytest.raises(ValueError):
            ops.linear_rows_w4(x8, w, s, 32, x_scale=xs)
    for a, kw in (((_z(4, 64, t=torch.float16), w, s, 32), {}), ((x, w, s.half(), 32), {}),
                  ((x, w, s, 32), dict(out_dtype=torch.float16))):
        with pytest.raises(TypeError):
            ops.linear_rows_w4(*a, **kw)


def test_cross_attention_wrapper_refusals():
    i32 = torch.int32
    q, kp, kv = _z(3, 5, 4, 16), _z(40, 2, 16), _z(3, 11, 2, 16)
    start, length = _z(3, t=i32), _z(3, t=i32)
    packed = dict(q=q, k=kp, v=kp, max_len=11, kv_start=start, kv_len=length)
    padded = dict(q=q, k=kv, v=kv, max_len=11)
    for base, kw in ((packed, dict(kv_len=None)), (packed, dict(k=kv)), (packed, dict(v=_z(39, 2, 16))),
                     (packed, dict(k=_z(40, 2, 24), v=_z(40, 2, 24))), (packed, dict(kv_start=start.long())),
                     (packed, dict(kv_len=length[:2])), (packed, dict(kv_index=_z(2, t=i32))),
                     (packed, dict(mask=_z(40, t=torch.float32))), (packed, dict(mask=_z(39, t=torch.bool))),
                     (packed, dict(out=_z(3, 5, 4, 16, t=torch.float32))), (packed, dict(q=_z(3, 5, 64))),
                     (packed, dict(q=_z(3, 5, 16, 4).transpose(2, 3))), (packed, dict()),  # the last: not on a GPU
                     (padded, dict(k=kp, v=kp)), (padded, dict(max_len=12)), (padded, dict(mask=_z(33, t=torch.bool))),
                     (padded, dict(k=kv.float(), v=kv.float())), (padded, dict())):
        with pytest.raises(ValueError):
            ops.cross_attention(**dict(base, **kw))
    with pytest.raises(TypeError):
        ops.cross_attention(**dict(padded, q=q.half()))
