"""The forms of the 8-bit linear for up to 16 tokens, at sizes that select each:
strips of one wave each over several rounds, shared by two, four and eight,
rows taken in chunks of columns, tokens rounded by the strips' workgroups or by
a launch in front; and the rounding of many tokens, four pieces a lane.  Against
the fp64 oracle of tests/test_gpu_head.py; up to 16 tokens are summed in fp32,
whose bound holds for both output types."""
import ctypes

import pytest
import torch

from oracle import head as H
from paper_2609_06161_amd import build_lib, output as O

from test_gpu_head import DEV, HALF, U, f64, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def plan():
    L = ctypes.CDLL(build_lib.HEAD_TEST_LIB)

    def of(m, n, T):
        out = (ctypes.c_int32 * 3)()
        assert L.af1_test_tokens_plan(*(ctypes.c_int64(v) for v in (m, n, T)), out) == 0
        return out[0], bool(out[1]), bool(out[2])
    return of


def units():
    return torch.cuda.get_device_properties(0).multi_processor_count


def weights(m, n, fmt, seed):
    """A matrix made on the GPU (some have 10^8 entries), and its values in fp64."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.randn((m, n), generator=g, device=DEV) * n ** -0.5
    w *= torch.exp2(2 * torch.randn((m, 1), generator=g, device=DEV))
    layer = O.Fp8Linear.from_dense(w, fmt)
    return layer, layer.weight.dequantize(torch.float32)


def check(layer, W, T, xfmt, dtype, seed, xdtype=torch.bfloat16):
    m, n = W.shape
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((T, n), generator=g, device=DEV)
    x *= torch.exp2(3 * torch.randn((T, 1), generator=g, device=DEV))
    x = x.to(xdtype)
    pad = 4096
    buf = torch.full((T * m + 2 * pad,), 3.0, dtype=dtype, device=DEV)
    y = layer.forward(x, buf[pad:pad + T * m].view(T, m), fmt=xfmt)
    assert (buf[:pad] == 3).all() and (buf[pad + T * m:] == 3).all()
    q = torch.from_numpy(H.round_rows(f64(x), xfmt)).to(DEV)
    want, S = torch.zeros((T, m), dtype=torch.float64, device=DEV), None
    S = want.clone()
    for i in range(0, m, 4096):       # fp64 copies of a part at a time
        part = W[i:i + 4096].double()
        want[:, i:i + 4096], S[:, i:i + 4096] = q @ part.T, q.abs() @ part.abs().T
    acc = (n / 64 + 64) * 2 * U * S
    within(f64(y), f64(want), f64(acc + HALF[dtype] * (want.abs() + acc)))
    return x, y


# waves a strip, sizes (rows past 4 strips of each unit, at them, and so on)
SIZES = [(1, lambda u: 64 * u + 17, 300), (1, lambda u: 4 * 64 * u + 40, 515),
         (1, lambda u: 64 * u + 1003, 9216), (2, lambda u: 64 * u, 700),
         (4, lambda u: 32 * u + 5, 1030), (4, lambda u: 64 * u - 16, 4096),
         (8, lambda u: 32 * u - 40, 2000)]


@pytest.mark.parametrize("share,rows,n", SIZES)
def test_strips(plan, share, rows, n):
    m = rows(units())
    layer, W = weights(m, n, "e4m3", n)
    for T, own in ((1, True), (13, 13 * -(-n // 128) <= 128), (16, 16 * -(-n // 128) <= 128)):
        print(f"strips m={m} n={n} T={T} by {share}", flush=True)
        assert plan(m, n, T) == (share, False, not own)
        for dtype in (torch.float32, torch.bfloat16):
            x, y = check(layer, W, T, "e4m3", dtype, T)
            assert torch.equal(layer.forward(x, dtype=dtype), y)


@pytest.mark.parametrize("share,rows", [(2, lambda u: 64 * u + 17), (4, lambda u: 32 * u + 5),
                                        (8, lambda u: 77)])
@pytest.mark.parametrize("n", [9217, 9300, 16384, 20000])
def test_strips_of_long_rows(plan, share, rows, n):
    """Chunks of 64 column blocks: 73 blocks, 128 (whole chunks) and 157."""
    m = rows(units())
    layer, W = weights(m, n, "e4m3", n + share)
    for T in (1, 13):
        print(f"long strips m={m} n={n} T={T} by {share}", flush=True)
        assert plan(m, n, T) == (share, True, True)
        for dtype in (torch.float32, torch.bfloat16):
            check(layer, W, T, "e4m3", dtype, T)


@pytest.mark.parametrize("wfmt,xfmt,xdtype", [("e5m2", "e4m3", torch.float32),
                                              ("e4m3", "e5m2", torch.float16),
                                              ("e5m2", "e5m2", torch.bfloat16)])
def test_strips_of_other_types(plan, wfmt, xfmt, xdtype):
    for m, n in ((64 * units() + 17, 600), (64 * units() + 17, 9300), (32 * units() + 5, 1030)):
        layer, W = weights(m, n, wfmt, m)
        for T in (1, 16):
            print(f"strips m={m} n={n} T={T} {wfmt} {xfmt} {xdtype}", flush=True)
            for dtype in (torch.float32, torch.bfloat16):
                check(layer, W, T, xfmt, dtype, T, xdtype)


@pytest.mark.parametrize("T,n", [(1030, 17000), (1100, 16400), (2049, 8200)])
@pytest.mark.parametrize("xfmt,xdtype", [("e4m3", torch.bfloat16), ("e5m2", torch.float32),
                                         ("e4m3", torch.float16)])
def test_many_tokens_are_rounded_by_four(plan, T, n, xfmt, xdtype):
    assert plan(100, n, T)[0] == 4
    layer, W = weights(100, n, "e4m3", T)
    check(layer, W, T, xfmt, torch.float32, T, xdtype)


def test_the_rounding_changes_with_the_tokens(plan):
    """Both roundings of many tokens give the same codes."""
    n, T = 17000, 1030
    assert plan(100, n, 300)[0] == 1 and plan(100, n, T)[0] == 4
    layer, W = weights(100, n, "e4m3", 1)
    x = torch.randn((T, n), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    x[:300, :128] *= 2.0 ** 20
    whole = layer.forward(x, dtype=torch.float32)
    part = layer.forward(x[:300].clone(), dtype=torch.float32)
    S = H.round_rows(f64(x[:300]), "e4m3")
    bound = 2 * (n / 64 + 64) * 2 * U * (torch.from_numpy(S).abs().to(DEV) @ W.double().abs().T)
    assert ((whole[:300].double() - part.double()).abs() <= bound).all()
