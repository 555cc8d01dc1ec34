"""Pins of the oracle's MXFP4 codec and head norms (CPU only)."""
import numpy as np
import pytest
import torch

from oracle import mxfp4
from oracle.qk_norm import norm_heads


def test_the_eight_magnitudes():
    assert mxfp4.e2m1_decode(np.arange(16)).tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]


def test_ties_saturation_and_signs():
    y = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 5.001, 7.99, -.25, -0.0, -5])
    assert mxfp4.e2m1_encode(y).tolist() == [0, 2, 2, 4, 4, 6, 6, 7, 7, 8, 8, 14]


def test_nearest_by_exhaustion():
    y = np.random.default_rng(0).uniform(-8, 8, 4000)
    v = mxfp4.e2m1_decode(mxfp4.e2m1_encode(y))
    assert np.array_equal(np.abs(v - y), np.abs(mxfp4.e2m1_decode(np.arange(16))[:, None] - y).min(0))


def test_scales_are_e8m0_of_the_block_maximum():
    x = np.zeros((1, 128))
    x[0, 3], x[0, 40], x[0, 64 + 31] = 5.9, -0.124, 1e-40
    codes, scales = mxfp4.quantise(x)
    # floor(log2): 2, -4 (0.124 2^6 = 7.9 saturates), below the range, none
    assert scales[0].tolist() == [127, 121, 2, 2]
    as_torch = torch.from_numpy(scales).view(torch.float8_e8m0fnu).double().numpy()
    assert np.array_equal(as_torch, np.ldexp(1.0, scales.astype(int) - 127))
    assert codes[0, 3] == 7 and codes[0, 40] == 15 and codes[0, 95] == 0


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_a_block_that_is_not_finite_is_nan(bad):
    x = np.ones((2, 128))
    x[1, 33] = bad
    codes, scales = mxfp4.quantise(x)
    v = mxfp4.dequantise(codes, scales)
    assert scales[1].tolist() == [125, 255, 125, 125] and not codes[1, 32:64].any()
    assert np.isnan(v[1, 32:64]).all() and np.array_equal(v[0], x[0]) and np.isfinite(v[1, 64:]).all()


def test_quantised_values_quantise_to_themselves():
    """At every size that bf16 has, and the relative error of what is not yet on the grid: the step
    below 2^(e + 2) is 2^(e + 1) at most, half of it to the nearest or 2^(e + 1) at saturation."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((512, 128)) * 2.0 ** rng.integers(-120, 126, (512, 1))
    v = mxfp4.dequantise(*mxfp4.quantise(x))
    codes, scales = mxfp4.quantise(v)
    assert np.array_equal(mxfp4.dequantise(codes, scales), v)
    top = np.abs(x).reshape(512, 4, 32).max(-1, keepdims=True)
    assert (np.abs(v - x).reshape(512, 4, 32) <= top / 4).all()


def test_pack_store_and_load():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((3, 2, 128))
    pool = np.full((2, 2, mxfp4.RUN), 0xA5, np.uint8)
    mxfp4.store(pool, [1, 0, 1], [0, 7, 15], x)
    data, v = mxfp4.load(pool, [1, 0, 1], [0, 7, 15])
    assert np.array_equal(v, mxfp4.dequantise(*mxfp4.quantise(x))) and data.shape == (3, 2, 68)
    assert int((pool != 0xA5).any(-1).sum()) == 4 and (pool[0, :, 1024:1024 + 28] == 0xA5).all()
    assert np.array_equal(mxfp4.unpack(mxfp4.pack(np.arange(128)[None] % 16)), np.arange(128)[None] % 16)
    whole = rng.standard_normal((2, 2, 16, 128))
    mxfp4.store(pool, [0] * 16 + [1] * 16, list(range(16)) * 2, whole.transpose(0, 2, 1, 3).reshape(32, 2, 128))
    assert np.array_equal(mxfp4.from_rows(whole), pool)


def test_norm_of_heads():
    x = np.arange(1, 129, dtype=np.float64).reshape(1, 1, 128)
    y = norm_heads(x, None, 1e-6)
    assert abs((y * y).mean() - 1) < 1e-9
    w = np.linspace(-1, 1, 128)
    assert np.allclose(norm_heads(x, w, 1e-6, 1.0), y * (w + 1))
    torch_y = torch.nn.functional.rms_norm(torch.from_numpy(x), (128,), torch.from_numpy(w), 0.5).numpy()
    assert np.allclose(norm_heads(x, w, 0.5), torch_y, rtol=1e-13)
