"""Refusals of the output head's C ABI beyond tests/test_head_abi_host.py, whose
calls with fake addresses are used here (none passes validation)."""
import pytest

from test_head_abi_host import BATCH, SHAPE, backward, kl, logprobs


@pytest.mark.parametrize("call", [logprobs, backward, kl])
def test_scales_that_overflow_inside_are_refused(call):
    """scale times log2(e) would be infinite, and every result NaN."""
    assert call(scale=2.4e38) == SHAPE and call(scale=3.4e38) == SHAPE
    assert call(scale=2.29e38, T=-1) == BATCH and call(scale=1e-45, T=-1) == BATCH
