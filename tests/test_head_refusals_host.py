"""Refusals of the output head's C ABI beyond tests/test_head_abi_host.py, whose
calls with fake addresses are used here (none passes validation)."""
import pytest

from paper_2609_06161_amd import head

from test_head_abi_host import ALIAS, BATCH, P, SHAPE, WS, backward, kl, linear, logprobs, matrix


@pytest.mark.parametrize("call", [logprobs, backward, kl])
def test_scales_that_overflow_inside_are_refused(call):
    """scale times log2(e) would be infinite, and every result NaN."""
    assert call(scale=2.4e38) == SHAPE and call(scale=3.4e38) == SHAPE
    assert call(scale=2.29e38, T=-1) == BATCH and call(scale=1e-45, T=-1) == BATCH


WIDE = 128256      # a few rows of it are several workgroups' work


def test_logprobs_workspace_refusals():
    need = head.af1_token_logprobs_workspace_bytes(6, WIDE, 3)
    assert need > 0

    def call(**kw):
        return logprobs(V=WIDE, ld=WIDE, T=6, **kw)

    assert call(ws=None) == WS and call(ws_bytes=need - 1) == WS and call(ws=P[8] + 8) != WS
    last = 6 * WIDE * 2 - 16                      # the last bytes of the logits
    for p in (P[0], P[0] + last, P[1], P[2], P[3], P[4], P[5], P[6], P[7]):
        assert call(ws=p) == ALIAS
    for k in ("lp", "ent", "lse", "top", "idx", "saved"):
        assert call(**{k: P[8] + need // 16 * 16 - 16}) == ALIAS, k


def test_distill_kl_workspace_refusals():
    need = head.af1_distill_kl_workspace_bytes(6, WIDE)
    assert need > 0

    def call(**kw):
        return kl(V=WIDE, ld_s=WIDE, ld_t=WIDE, T=6, **{"ldd": WIDE, **kw})

    assert call(ws=None) == WS and call(ws_bytes=0) == WS
    # what the call itself needs is at most what is asked for, for any type
    assert call(ws_bytes=need, out=P[0]) == ALIAS
    for p in (P[0], P[1], P[2], P[3], P[4], P[0] + 6 * WIDE * 2 - 16, P[4] + 6 * WIDE * 2 - 16):
        assert call(ws=p) == ALIAS
    for k in ("w", "out", "ds"):
        assert call(**{k: P[5]}) == ALIAS, k
    # the loss alone: no gradient to overlap, and its stride is not looked at
    assert call(ds=None, ldd=0, ws=None) == WS and call(ds=None, ldd=0, out=P[1]) == ALIAS


@pytest.mark.parametrize("T", [4, 16, 24, 70, 500])
def test_linear_workspace_refusals(T):
    W = matrix(rows=4096, cols=4096)
    need = head.af1_fp8_linear_workspace_bytes(4096, 4096, T)
    if T == 4:
        assert need == 0                          # the tokens stay in the workgroups
        return
    assert linear(W, T=T, ws=None) == WS and linear(W, T=T, ws_bytes=need - 1) == WS
    for p in (P[0], P[1], P[2], P[3]):
        assert linear(W, T=T, ws=p) == ALIAS
    assert linear(W, T=T, y=P[4] + need - 16) == ALIAS
