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


def tile_bound(q, W, want):
    """What af1_fp8_linear allows a bfloat16 output of more than 16 tokens: (each
    entry's bound, the norm's).  Seven of eight products lose less than 2^-13
    of the largest of the eight each; fp32 sums and the output's rounding as
    above.  What is lost has the sign of a product, so for random signs it adds
    up in squares: the norm's bound takes twice that."""
    n = q.shape[1]
    cut, square, S = (torch.empty_like(want) for _ in range(3))
    pad = torch.nn.functional.pad
    Wg = pad(W, (0, -n % 8)).view(len(W), -1, 8).abs()
    for t, row in enumerate(pad(q, (0, -n % 8)).view(len(q), 1, -1, 8).abs()):
        p = Wg * row
        unit = p.amax(2) * 2.0 ** -13
        cut[t], square[t], S[t] = 7 * unit.sum(1), 7 * (unit ** 2).sum(1), p.sum((1, 2))
    acc = cut + (n / 64 + 64) * 2 * U * S
    half = HALF[torch.bfloat16]
    return acc + half * (want.abs() + acc), half * want.norm() + 2 * square.sum().sqrt()


@pytest.mark.parametrize("T,m,n", [(45, 300, 515), (45, 1000, 2000), (700, 3001, 4000),
                                   (130, 4100, 6000), (500, 8200, 600), (1030, 4100, 6000)])
@pytest.mark.parametrize("xfmt", ["e4m3", "e5m2"])
def test_bfloat16_tiles_keep_what_the_interface_says(T, m, n, xfmt):
    print(f"bfloat16 tiles T={T} m={m} n={n} {xfmt}", flush=True)
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.randn((T, n), generator=g, device=DEV).to(torch.bfloat16)
    w = torch.randn((m, n), generator=g, device=DEV) * n ** -0.5
    layer = O.Fp8Linear.from_dense(w)
    got = layer.forward(x, fmt=xfmt).double()
    W = layer.weight.dequantize(torch.float32).double()
    rows = torch.cat([O.Fp8Matrix.quantize(r[None].clone(), xfmt).dequantize(torch.float32) for r in x])
    q = rows.double()
    want = q @ W.T
    entry, norm = tile_bound(q, W, want)
    err = (got - want).abs()
    assert norm < 0.01 * want.norm()        # an output off by 1% does not pass
    assert (err <= entry).all(), (err - entry).max()
    assert err.norm() <= norm, (err.norm() / want.norm(), norm / want.norm())


@pytest.mark.parametrize("T,m,n", [(33, 300, 300), (500, 8200, 600)])
def test_bfloat16_tiles_where_products_cancel(T, m, n):
    """The six products of an eight beside two of 2^12 may be lost, no more."""
    x, layer, want, bound = cancelling(T, m, n, "e4m3")
    got = f64(layer.forward(x))
    bound = bound + HALF[torch.bfloat16] * (np.abs(want) + bound)
    assert (got <= want + bound).all() and (got >= -bound).all()
