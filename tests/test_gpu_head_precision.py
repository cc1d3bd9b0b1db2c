"""How many bits the 8-bit linear keeps, on sums whose large products cancel.

In eight columns of every block two products of 2^12 cancel and six of 2^-2 are
left, so what is lost beside the large ones shows in the result: a sum that
keeps 13 bits below the largest of the eight (units of 2^-1) loses all six,
fp32 none.  All values are on the 8-bit grids, so nothing else rounds but the
fp32 sums, which are off by at most (n/64 + 64) 2u S (u = 2^-24, S the sum of
the magnitudes: 8192 + 1.5 a block), and a bfloat16 output by half a step."""
import numpy as np
import pytest
import torch

from paper_2609_06161_amd import output as O

from test_gpu_head import DEV, HALF, U, f64

pytestmark = pytest.mark.gpu


def cancelling(T, m, n, fmt):
    """(x, layer, want, bound of the fp32 sums) with want > 4 bounds."""
    x, w = torch.zeros(T, n), torch.zeros(m, n)
    starts = range(0, n - 7, 128)
    for s in starts:
        x[:, s], x[:, s + 7] = 64.0, -64.0
        w[:, s], w[:, s + 7] = 64.0, 64.0
        x[:, s + 1:s + 7] = w[:, s + 1:s + 7] = 0.5
    # rows and tokens are told apart by powers of two
    x *= torch.exp2(torch.arange(T) % 5 - 2.0)[:, None]
    w *= torch.exp2(torch.arange(m) % 3 - 1.0)[:, None]
    want = x.double() @ w.double().T
    S = x.double().abs() @ w.double().abs().T
    bound = (n / 64 + 64) * 2 * U * S
    assert (want > 4 * bound).all()
    return x.to(DEV), O.Fp8Linear.from_dense(w.to(DEV), fmt), want.numpy(), bound.numpy()


def check(T, m, n, dtype, fmt="e4m3", xfmt="e4m3"):
    x, layer, want, bound = cancelling(T, m, n, fmt)
    got = f64(layer.forward(x, fmt=xfmt, dtype=dtype))
    over = np.abs(got - want) - (bound + HALF[dtype] * (np.abs(want) + bound))
    assert over.max() <= 0, f"off by {np.abs(got - want).max()} of {want.max()}"


@pytest.mark.parametrize("T,m,n", [(1, 300, 300), (5, 4099, 256), (16, 1000, 1030), (17, 300, 300),
                                   (32, 515, 1000)])
@pytest.mark.parametrize("fmt,xfmt", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_tokens_are_summed_in_fp32(T, m, n, fmt, xfmt, dtype):
    check(T, m, n, dtype, fmt, xfmt)


@pytest.mark.parametrize("T,m,n", [(33, 300, 300), (70, 515, 1000), (500, 8200, 600)])
def test_fp32_outputs_are_summed_in_fp32(T, m, n):
    check(T, m, n, torch.float32)
