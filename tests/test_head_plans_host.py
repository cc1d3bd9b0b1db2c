"""Launch plans of the output head's kernels, as the test build tells them
(host code; 256 compute units are assumed where there is no device)."""
import ctypes

import pytest

from paper_2609_06161_amd import af1, build_lib, head


@pytest.fixture(scope="module")
def lib():
    return ctypes.CDLL(build_lib.HEAD_TEST_LIB)


@pytest.mark.parametrize("dtype,piece", [(af1.AF1_SRC_F32, 8192), (af1.AF1_SRC_BF16, 16384),
                                         (af1.AF1_SRC_F16, 16384)])
def test_kl_rows_wait_for_no_more_parts_than_run_at_once(lib, dtype, piece):
    """Four workgroups a compute unit run at once; a row's parts wait for each
    other only where they are at most half of these."""
    def plan(T, V):
        out = (ctypes.c_int32 * 2)()
        assert lib.af1_test_kl_plan(dtype, ctypes.c_int64(T), ctypes.c_int64(V), out) == 0
        return out[0], bool(out[1])

    for T in (1, 2, 33, 3000):
        for V in (1, 100, 5000, 128256, 1 << 20, 512 * piece, 512 * piece + 8, 3 << 21, 10 ** 7,
                  head.AF1_HEAD_MAX_VOCAB):
            parts, first = plan(T, V)
            assert first == (parts > 512), (T, V, parts)
            assert parts <= 1 or parts <= -(-V // 2048)
    assert plan(1, 512 * piece) == (512, False) and plan(1, head.AF1_HEAD_MAX_VOCAB)[1]
