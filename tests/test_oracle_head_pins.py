"""Pins of the output head's oracle to the formats' definitions and to
mathematics (CPU): known codes, nearest-even rounding, the scale rule, the
gradients by differences, and the losses' identities."""
import numpy as np
import pytest
import torch

from oracle import head as H


@pytest.mark.parametrize("fmt,dtype", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_code_values_are_the_formats(fmt, dtype):
    want = torch.arange(256, dtype=torch.uint8).view(dtype).to(torch.float64).numpy()
    np.testing.assert_array_equal(H.code_values(fmt), want)
    assert np.nanmax(np.where(np.isinf(want), np.nan, want)) == H.MAX[fmt]


@pytest.mark.parametrize("fmt,dtype", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_encode_rounds_to_nearest_even(fmt, dtype):
    v = np.random.default_rng(0).standard_normal(20000) * np.exp2(
        np.random.default_rng(1).uniform(-20, 8, 20000))
    grid = np.sort(H.code_values(fmt)[np.isfinite(H.code_values(fmt))])
    mid = (grid[1:] + grid[:-1]) / 2        # every tie
    v = np.clip(np.concatenate([v, grid, mid]), -H.MAX[fmt], H.MAX[fmt]).astype(np.float32)
    want = torch.from_numpy(v).to(dtype).view(torch.uint8).numpy()
    np.testing.assert_array_equal(H.encode(v, fmt), want)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_exponent_is_the_smallest_that_fits(fmt):
    a = np.concatenate([np.exp2(np.random.default_rng(2).uniform(-140, 127, 500)),
                        H.MAX[fmt] * np.exp2(np.arange(-20.0, 20)), [0.0]])
    e = H.exponent(a, fmt)
    assert (a <= H.MAX[fmt] * np.exp2(e.astype(float))).all()
    low = (a > H.MAX[fmt] * np.exp2(e - 1.0)) | (e == -127) | (a == 0)
    assert low.all() and e[-1] == 0


def test_quantize_restores_what_the_grid_holds():
    rng = np.random.default_rng(3)
    v = H.code_values("e4m3")
    a = v[rng.integers(0, 0x7f, (200, 150))] * 4.0
    a[0, 0] = a[0, 140] = a[150, 0] = a[150, 140] = 448.0 * 4
    c, s = H.quantize(a, "e4m3")
    np.testing.assert_array_equal(H.dequantize(c, s, 200, 150, "e4m3"), a)
    assert (c[1, 1, 72:, :] == 0).all() and (c[1, 1, :, 22:] == 0).all()


def test_gradients_by_differences():
    rng = np.random.default_rng(4)
    x, t = rng.standard_normal((3, 11)), rng.standard_normal((3, 11))
    y, gl, gh, w = np.array([2, -1, 10]), rng.standard_normal(3), rng.standard_normal(3), rng.random(3)

    def loss(z):
        lp, h = H.token_logprobs(z, y, 1.3)
        return (gl * lp + gh * h).sum()

    def kl(z):
        return (w * H.distill_kl(z, t, 0.7)).sum()

    for f, g in ((loss, H.token_logprobs_backward(x, y, gl, gh, 1.3)),
                 (kl, H.distill_kl_backward(x, t, w, 0.7))):
        num = np.empty_like(x)
        for i in np.ndindex(x.shape):
            d = np.zeros_like(x)
            d[i] = 1e-6
            num[i] = (f(x + d) - f(x - d)) / 2e-6
        np.testing.assert_allclose(g, num, atol=1e-8)


def test_losses_identities():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4, 9))
    assert np.abs(H.distill_kl(x, x + 3.0)).max() < 1e-15
    assert (H.distill_kl(x, rng.standard_normal((4, 9))) > 0).all()
    np.testing.assert_allclose(H.token_logprobs(np.zeros((2, 8)), [0, 7])[1], np.log(8))
    np.testing.assert_allclose(H.lse(x, 2.0), np.log(np.exp(2 * x).sum(1)))
    m = np.full((1, 4), -np.inf)
    assert H.token_logprobs(m, [1])[0][0] == -np.inf and H.token_logprobs(m, [1])[1][0] == 0
    assert list(H.top(np.array([[1.0, 3.0, 3.0, np.nan]]), 5)[0]) == [3, 1, 2, 0, -1]
