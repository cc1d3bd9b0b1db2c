"""Every form of the 8-bit linear, over one range of columns and over several,
at sizes that fit none of its tiles, against the fp64 oracle with the bounds of
tests/test_gpu_head.py; and the KL divergence when the blocks of a row do not
wait for each other's statistics (the test build: every other part publishes
late, nothing waits), so that they compute what they miss."""
import ctypes
import importlib.util

import numpy as np
import pytest
import torch

from paper_2609_06161_amd import af1, build_lib, head, output as O

from test_gpu_head import check_linear, check_kl, logits, randn

pytestmark = pytest.mark.gpu

FEW, SHORT_TILES, TILES, LARGE_TILES = range(4)


@pytest.fixture(scope="module")
def plan():
    L = ctypes.CDLL(build_lib.HEAD_TEST_LIB)
    L.af1_test_linear_plan.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int32,
                                                             ctypes.POINTER(ctypes.c_int32)]

    def of(m, n, T, y):
        out = (ctypes.c_int32 * 2)()
        assert L.af1_test_linear_plan(m, n, T, y, out) == 0
        return out[0], out[1] > 1
    return of


CASES = [
    (torch.bfloat16, FEW, False, 20, 1000, 1030), (torch.float32, FEW, False, 32, 515, 129),
    (torch.bfloat16, SHORT_TILES, False, 45, 300, 515), (torch.float32, SHORT_TILES, False, 64, 2049, 260),
    (torch.bfloat16, SHORT_TILES, True, 45, 1000, 2000), (torch.float32, SHORT_TILES, True, 100, 129, 2000),
    (torch.bfloat16, TILES, False, 700, 3001, 4000), (torch.float32, TILES, False, 500, 8200, 600),
    (torch.bfloat16, TILES, True, 130, 4100, 6000), (torch.float32, TILES, True, 200, 4100, 4000),
    (torch.bfloat16, LARGE_TILES, False, 500, 8200, 600),
    (torch.bfloat16, LARGE_TILES, True, 1030, 4100, 6000)]


@pytest.mark.parametrize("ydtype,form,split,T,m,n", CASES)
def test_form(plan, ydtype, form, split, T, m, n):
    print(f"form {form} split={split} T={T} m={m} n={n} {ydtype}", flush=True)
    y = af1.AF1_SRC_F32 if ydtype == torch.float32 else af1.AF1_SRC_BF16
    assert plan(m, n, T, y) == (form, split)
    layer, x, _, out = check_linear(T, m, n, ydtype=ydtype)
    assert torch.equal(layer.forward(x.to("cuda"), dtype=ydtype), out)


@pytest.mark.parametrize("n", [1, 130, 300, 400, 520])
def test_fewer_column_blocks_than_the_ring(plan, n):
    assert plan(8200, n, 500, af1.AF1_SRC_BF16) == (LARGE_TILES, False)
    check_linear(500, 8200, n)
    check_linear(45, 300, n)
    check_linear(140, 777, n, ydtype=torch.float32)


def test_mixed_formats_in_tiles(plan):
    assert plan(8200, 600, 500, af1.AF1_SRC_BF16)[0] == LARGE_TILES
    check_linear(500, 8200, 600, "e4m3", "e5m2", torch.float32, torch.bfloat16)
    check_linear(300, 3001, 3000, "e5m2", "e4m3", torch.float16, torch.float32)


def test_rows_and_neighbours_are_left_alone():
    """Outputs stay inside y: the entries around it keep their values, for odd
    row lengths and tiles that reach past the last row and token."""
    for T, m, n, dtype in ((3, 77, 300, torch.bfloat16), (20, 1001, 515, torch.float32),
                           (45, 301, 515, torch.bfloat16), (130, 4101, 700, torch.float32),
                           (510, 8201, 300, torch.bfloat16)):
        layer = O.Fp8Linear.from_dense(randn(T, m, n).to("cuda"))
        pad = 4096
        buf = torch.full((T * m + 2 * pad,), 3.0, dtype=dtype, device="cuda")
        layer.forward(randn(T + 1, T, n).to("cuda"), buf[pad:pad + T * m].view(T, m))
        assert (buf[:pad] == 3).all() and (buf[pad + T * m:] == 3).all()


@pytest.fixture(scope="module")
def late():
    """The tensor calls on the test build."""
    def load(name, path):
        spec = importlib.util.spec_from_file_location(name, path)
        mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(mod)
        return mod
    lib = load("paper_2609_06161_amd.head_late", head.__file__)
    lib.LIB_PATH = build_lib.HEAD_TEST_LIB
    lib.lib()
    calls = load("paper_2609_06161_amd.output_late", O.__file__)
    calls.head = lib
    return calls


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(1, 2049), (3, 20011), (2, 130000), (130, 20011)])
def test_kl_statistics_computed_instead(late, T, V, dtype):
    print(f"late statistics T={T} V={V} {dtype}", flush=True)
    s = logits(T + V, T, V, dtype).to("cuda")
    t = (s.float() + 0.5 * randn(V, T, V).to("cuda")).to(dtype)
    kl, d = check_kl(s, t)
    for _ in range(2):
        k2, d2 = late.distill_kl(s, t)
        assert torch.equal(k2, kl) and torch.equal(d2, d)
    # written over the student: what is missing is read before it is written
    own = s.clone()
    k3, d3 = late.distill_kl(own, t, dstudent=own)
    assert torch.equal(k3, kl) and torch.equal(d3, d)


def test_kl_beyond_64_parts():
    """A vocabulary of more parts than a wave has lanes."""
    T, V = 2, 140001
    s = logits(9, T, V, torch.float32).to("cuda")
    check_kl(s, s + 0.3 * randn(10, T, V).to("cuda"))
    np.testing.assert_array_equal(
        O.distill_kl(s, s.clone())[0].cpu().numpy(), np.zeros(T, np.float32))
