"""Pins of the oracle's text-side operations against brute force, closed
forms and independent library routines (torch CPU).  CPU only."""
import math

import numpy as np
import pytest
import torch

from oracle import text as O

rng = np.random.default_rng(11)


def test_e4m3_is_the_nearest_value_of_the_format():
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    every = np.unique(every[np.isfinite(every)])
    assert np.array_equal(O.e4m3(every), every) and every.max() == 448
    v = np.concatenate([rng.standard_normal(2000) * s for s in (1e-3, 0.02, 1, 100)])
    v = v[np.abs(v) < 448]
    near = np.abs(v[:, None] - every[None]).min(1)
    assert np.array_equal(np.abs(O.e4m3(v) - v), near)
    f = v.astype(np.float32)  # torch rounds from fp32, ties to even
    assert np.array_equal(O.e4m3(f), torch.from_numpy(f).to(torch.float8_e4m3fn).double().numpy())
    mid = (every[1:] + every[:-1]) / 2  # ties
    assert np.array_equal(O.e4m3(mid), torch.from_numpy(mid).float().to(torch.float8_e4m3fn).double().numpy())


def test_rmsnorm_closed_forms_and_library():
    x, r, g = rng.standard_normal((5, 24)), rng.standard_normal((5, 24)), rng.standard_normal(24)
    y, h = O.rmsnorm(x, g, 1e-5, r)
    ref = torch.nn.functional.rms_norm(torch.from_numpy(x + r), (24,), torch.from_numpy(g), 1e-5).numpy()
    assert np.allclose(y, ref, rtol=1e-13) and np.array_equal(h, x + r)
    y, _ = O.rmsnorm(np.full((1, 7), -3.0), eps=0.0)
    assert np.allclose(y, -1)
    s = O.block_scales(np.arange(300.0)[None], 128)
    assert np.allclose(s, [[127 / 448, 255 / 448, 299 / 448]]) and O.block_scales(np.zeros((2, 5)), 0).shape == (2, 1)


def test_w4_weights_brute_force():
    codes = rng.integers(0, 256, (3, 20)).astype(np.uint8)
    scale, zero = rng.standard_normal((3, 2)), rng.integers(0, 16, (3, 2))
    w = O.w4_weights(codes, scale, zero, 32)
    for n in range(3):
        for k in range(40):
            c = (int(codes[n, k // 2]) >> (4 * (k % 2))) % 16
            assert w[n, k] == (c - zero[n, k // 32]) * scale[n, k // 32]
    assert np.array_equal(O.w4_weights(codes, scale, None, 32), O.w4_weights(codes, scale, np.full((3, 2), 8), 32))


@pytest.mark.parametrize("rep", [1, 3])
def test_cross_attention_matches_the_library_on_each_text(rep):
    q, k, v = rng.standard_normal((3, 4, 2 * rep, 8)), rng.standard_normal((20, 2, 8)), rng.standard_normal((20, 2, 8))
    texts = [range(0, 7), range(7, 8), []]
    o, w = O.cross_attention(q, k, v, texts, 0.3)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).transpose(0, 1)  # noqa: E731
    for i in range(2):
        rows = list(texts[i])
        ref = torch.nn.functional.scaled_dot_product_attention(
            t(q[i]), t(k[rows].repeat(rep, 1)), t(v[rows].repeat(rep, 1)), scale=0.3).transpose(0, 1).numpy()
        assert np.allclose(o[i], ref, atol=1e-13)
        assert (w[i] >= np.abs(o[i]) - 1e-15).all()
    assert not o[2].any()
    assert np.allclose(o[1], np.repeat(v[7], rep, 0)[None])  # one key: its value
    assert math.isfinite(w.sum())


def test_rmsnorm_unit_mean_square_and_scale():
    x = rng.standard_normal((4, 33))
    y, _ = O.rmsnorm(x, eps=0.0)
    assert np.allclose((y * y).mean(1), 1, rtol=1e-14)
    assert np.allclose(O.rmsnorm(x * np.array([[3.0], [1e-8], [1e12], [-2.0]]), eps=0.0)[0], y * np.array([[1], [1], [1], [-1]]), rtol=1e-13)


def test_w4_product_brute_force():
    codes, x = rng.integers(0, 256, (5, 36)).astype(np.uint8), rng.standard_normal((2, 72))
    scale, zero = rng.standard_normal((5, 2)), rng.integers(0, 16, (5, 2))
    y = x @ O.w4_weights(codes, scale, zero, 64).T
    for m in range(2):
        for n in range(5):
            s = 0.0
            for k in range(72):
                s += x[m, k] * scale[n, k // 64] * ((int(codes[n, k // 2]) >> (4 * (k % 2))) % 16 - int(zero[n, k // 64]))
            assert math.isclose(y[m, n], s, rel_tol=1e-12, abs_tol=1e-12)
