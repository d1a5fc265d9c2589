"""Sizes past 31 bits, which the C entry points' arguments cannot hold, are
turned away by the Python wrappers of the text-side operators, not cut to
their low bits.  Tensors without memory; CPU only."""
import os

import pytest

torch = pytest.importorskip("torch")
P = pytest.importorskip("paper_2605_08835_amd")
from paper_2605_08835_amd import ops  # noqa: E402

pytestmark = pytest.mark.skipif(not os.path.exists(P.binding.LIB_PATH), reason="libsynerdiff.so not built")
BIG = (1 << 32) + 8


def _m(*shape, t=torch.bfloat16):
    return torch.empty(*shape, dtype=t, device="meta")


def test_rmsnorm_width():
    with pytest.raises(ValueError, match="2\\^31"):
        ops.rmsnorm(_m(2, BIG))


@pytest.mark.parametrize("M,K,N", [(BIG, 64, 16), (4, BIG, 16), (4, 64, BIG)])
def test_linear_rows_w4_sizes(M, K, N):
    with pytest.raises(ValueError, match="2\\^31"):
        ops.linear_rows_w4(_m(M, K), _m(N, K // 2, t=torch.uint8), _m(N, -(-K // 32)), 32)


def test_cross_attention_sizes():
    i32 = torch.int32
    for n, nq, heads, tokens, n_ctx, max_len in ((2, 5, 4, 40, 2, BIG), (2, 5, 4, 40, 2, -BIG), (2, 5, 4, 40, 2, 1 << 31),
                                                 (2, BIG, 4, 40, 2, 11), (BIG, 1, 4, 40, 2, 11), (2, 5, 4, 40, BIG, 11),
                                                 (2, 1, BIG, 40, 2, 11)):
        with pytest.raises(ValueError, match="2\\^31"):
            ops.cross_attention(_m(n, nq, heads, 16), _m(tokens, 4, 16), _m(tokens, 4, 16), max_len, kv_start=_m(n_ctx, t=i32),
                                kv_len=_m(n_ctx, t=i32), kv_index=_m(n, t=i32))
    with pytest.raises(ValueError, match="2\\^31"):
        ops.cross_attention(_m(2, 5, 4, 16), _m(2, BIG, 4, 16), _m(2, BIG, 4, 16), BIG)
