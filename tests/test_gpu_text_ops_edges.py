"""Edge values of the text-side operators on the GPU, against the oracle's
float64 definitions."""
import math

import pytest

from test_gpu_text_ops import _attn_case, _check_attn, ops  # noqa: F401

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
