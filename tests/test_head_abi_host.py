"""Host-only checks of the output head's C ABI and binding: exports, sizes,
and every refusal, returned before anything is enqueued (fake device addresses
are safe because no call below passes validation)."""
import os
import re
import subprocess

import pytest
import torch

from paper_2609_06161_amd import af1, head, output

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BASE, MB = 0x7F00_0000_0000, 1 << 20
P = [BASE + 4096 * MB * i for i in range(12)]      # arrays 4 GiB apart
OK, NULL, SHAPE, BATCH, ALIGN, WS, ALIAS, DTYPE = (
    af1.AF1_OK, af1.AF1_ERR_NULL, af1.AF1_ERR_SHAPE, af1.AF1_ERR_BATCH, af1.AF1_ERR_ALIGN,
    af1.AF1_ERR_WORKSPACE, af1.AF1_ERR_ALIAS, af1.AF1_ERR_DTYPE)
BIG = 1 << 31


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "af1_head.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(af1_[a-z0-9_]+)\s*\(", text))
    assert len(names) == 12
    out = subprocess.run(["nm", "-D", "--defined-only", head.LIB_PATH], capture_output=True,
                         text=True, check=True).stdout
    assert set(re.findall(r"\bT (af1_\w+)", out)) == names
    for name in names:
        assert hasattr(head.lib(), name)


def test_storage_sizes():
    assert head.af1_fp8_code_bytes(1, 1) == 128 * 128
    assert head.af1_fp8_code_bytes(129, 256) == 2 * 2 * 128 * 128
    assert head.af1_fp8_scale_bytes(50257, 4096) == 393 * 32
    for rows, cols in ((0, 1), (1, 0), (-1, 5), (af1.AF1_MAX_DIM + 1, 1)):
        assert head.af1_fp8_code_bytes(rows, cols) == 0
        assert head.af1_fp8_scale_bytes(rows, cols) == 0
        assert head.af1_fp8_linear_workspace_bytes(rows, cols, 4) == 0
    assert head.af1_fp8_linear_workspace_bytes(128, 128, 0) == 0
    assert head.af1_fp8_linear_workspace_bytes(128, 128, head.AF1_HEAD_MAX_TOKENS + 1) == 0
    assert head.af1_token_logprobs_workspace_bytes(4, 0, 0) == 0
    assert head.af1_distill_kl_workspace_bytes(0, 100) == 0


def quantize(src=P[0], dt=af1.AF1_SRC_BF16, rows=256, cols=300, fmt=0, codes=P[1], scales=P[2]):
    return head.af1_fp8_quantize(src, dt, rows, cols, fmt, codes, scales, stream=0, check=False)


def test_quantize_refusals():
    assert quantize(dt=af1.AF1_SRC_I8) == DTYPE and quantize(dt=9) == DTYPE
    assert quantize(fmt=2) == DTYPE
    assert quantize(rows=0) == SHAPE and quantize(cols=af1.AF1_MAX_DIM + 1) == SHAPE
    for k in ("src", "codes", "scales"):
        assert quantize(**{k: None}) == NULL
        assert quantize(**{k: P[3] + 8}) == ALIGN
    assert quantize(codes=P[0] + 16) == ALIAS
    assert quantize(scales=P[1] + 2 * 3 * 128 * 128 - 16) == ALIAS
    assert quantize(scales=P[0]) == ALIAS


def matrix(rows=256, cols=300, fmt=0, codes=P[0], scales=P[1]):
    return head.make_matrix(rows, cols, fmt, codes, scales)


def test_dequantize_and_transpose_refusals():
    def deq(W=matrix(), dst=P[3], dt=af1.AF1_SRC_F32):
        return head.af1_fp8_dequantize(W, dst, dt, stream=0, check=False)

    def tr(W=matrix(), codes=P[3], scales=P[4]):
        return head.af1_fp8_transpose(W, codes, scales, stream=0, check=False)

    for f in (deq, tr):
        assert f(None) == NULL
        assert f(matrix(fmt=7)) == DTYPE
        assert f(matrix(rows=0)) == SHAPE
        assert f(matrix(codes=None)) == NULL
        assert f(matrix(scales=P[1] + 4)) == ALIGN
    assert deq(dt=af1.AF1_SRC_I8) == DTYPE
    assert deq(dst=None) == NULL and deq(dst=P[3] + 2) == ALIGN
    assert deq(dst=P[0] + 64) == ALIAS and deq(dst=P[1]) == ALIAS
    assert tr(codes=None) == NULL and tr(scales=None) == NULL
    assert tr(codes=P[0]) == ALIAS and tr(scales=P[3]) == ALIAS and tr(scales=P[1]) == ALIAS


def linear(W=matrix(), x=P[2], xd=af1.AF1_SRC_BF16, xf=0, T=70, y=P[3], yd=af1.AF1_SRC_F32,
           ws=P[4], ws_bytes=BIG):
    return head.af1_fp8_linear(W, x, xd, xf, T, y, yd, ws, ws_bytes, stream=0, check=False)


def test_linear_refusals():
    assert linear(None) == NULL
    assert linear(xd=af1.AF1_SRC_I8) == DTYPE and linear(xf=5) == DTYPE
    assert linear(yd=af1.AF1_SRC_F16) == DTYPE and linear(matrix(fmt=-1)) == DTYPE
    assert linear(matrix(cols=0)) == SHAPE
    assert linear(T=-1) == BATCH and linear(T=head.AF1_HEAD_MAX_TOKENS + 1) == BATCH
    assert linear(x=None) == NULL and linear(y=None) == NULL
    assert linear(matrix(codes=None)) == NULL
    for k in ("x", "y", "ws"):
        assert linear(**{k: P[5] + 2}) == ALIGN
    need = head.af1_fp8_linear_workspace_bytes(256, 300, 70)
    assert linear(ws=None) == WS and linear(ws_bytes=need - 1) == WS
    for y in (P[0], P[1], P[2], P[4]):
        assert linear(y=y) == ALIAS
    assert linear(ws=P[2]) == ALIAS and linear(ws=P[0]) == ALIAS
    assert linear(T=0, x=None, y=None, ws=None) == OK


def logprobs(z=P[0], dt=af1.AF1_SRC_BF16, T=6, V=1000, ld=1000, scale=1.0, y=P[1], lp=P[2],
             ent=P[3], lse=P[4], k=3, top=P[5], idx=P[6], saved=P[7], ws=P[8], ws_bytes=BIG):
    return head.af1_token_logprobs(z, dt, T, V, ld, scale, y, lp, ent, lse, k, top, idx, saved, ws,
                                   ws_bytes, stream=0, check=False)


def test_logprobs_refusals():
    assert logprobs(dt=af1.AF1_SRC_I8) == DTYPE
    for bad in (dict(V=0, ld=0), dict(ld=999), dict(V=head.AF1_HEAD_MAX_VOCAB + 1, ld=1 << 25),
                dict(k=-1), dict(k=33), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("inf")), dict(scale=float("nan"))):
        assert logprobs(**bad) == SHAPE, bad
    assert logprobs(T=-1) == BATCH and logprobs(T=head.AF1_HEAD_MAX_TOKENS + 1) == BATCH
    assert logprobs(z=None) == NULL and logprobs(y=None) == NULL
    assert logprobs(top=None) == NULL and logprobs(idx=None) == NULL
    for bad in (dict(z=P[0] + 1), dict(dt=af1.AF1_SRC_F32, z=P[0] + 2), dict(y=P[1] + 4),
                dict(lp=P[2] + 2), dict(ent=P[3] + 1), dict(lse=P[4] + 2), dict(top=P[5] + 2),
                dict(idx=P[6] + 4), dict(saved=P[7] + 8), dict(ws=P[8] + 4)):
        assert logprobs(**bad) == ALIGN, bad
    for bad in (dict(lp=P[0]), dict(ent=P[2] + 8), dict(lse=P[1]), dict(top=P[0] + 1000),
                dict(idx=P[5]), dict(saved=P[0] + 11984)):
        assert logprobs(**bad) == ALIAS, bad
    need = head.af1_token_logprobs_workspace_bytes(6, 1000, 3)
    if need:
        assert logprobs(ws=None) == WS and logprobs(ws_bytes=need - 1) == WS
        assert logprobs(ws=P[0]) == ALIAS
    assert logprobs(T=0, z=None, y=None, ws=None) == OK


def backward(z=P[0], dt=af1.AF1_SRC_BF16, T=6, V=1000, ld=1000, scale=1.0, y=P[1], saved=P[2],
             gl=P[3], gh=P[4], dz=P[5], ldd=1000):
    return head.af1_token_logprobs_backward(z, dt, T, V, ld, scale, y, saved, gl, gh, dz, ldd,
                                            stream=0, check=False)


def test_logprobs_backward_refusals():
    assert backward(dt=5) == DTYPE
    for bad in (dict(ldd=999), dict(ld=10), dict(V=0), dict(scale=0.0)):
        assert backward(**bad) == SHAPE, bad
    assert backward(T=-2) == BATCH
    for k in ("z", "saved", "dz", "y"):
        assert backward(**{k: None}) == NULL, k
    for bad in (dict(z=P[0] + 1), dict(dz=P[5] + 1), dict(y=P[1] + 4), dict(saved=P[2] + 8),
                dict(gl=P[3] + 2), dict(gh=P[4] + 2)):
        assert backward(**bad) == ALIGN, bad
    # only the logits' own array, with the same stride, may be written over
    assert backward(dz=P[0], ldd=1008) == ALIAS and backward(dz=P[0] + 2) == ALIAS
    for p in (P[1], P[2], P[3], P[4]):
        assert backward(dz=p) == ALIAS
    assert backward(T=0, z=None, dz=None) == OK


def kl(s=P[0], t=P[1], dt=af1.AF1_SRC_BF16, T=6, V=1000, ld_s=1000, ld_t=1000, scale=1.0, w=P[2],
       out=P[3], ds=P[4], ldd=1000, ws=P[5], ws_bytes=BIG):
    return head.af1_distill_kl(s, t, dt, T, V, ld_s, ld_t, scale, w, out, ds, ldd, ws, ws_bytes,
                               stream=0, check=False)


def test_distill_kl_refusals():
    assert kl(dt=af1.AF1_SRC_I8) == DTYPE
    for bad in (dict(ld_s=999), dict(ld_t=1), dict(ldd=0), dict(V=0), dict(scale=float("nan"))):
        assert kl(**bad) == SHAPE, bad
    assert kl(T=-1) == BATCH
    for k in ("s", "t", "out"):
        assert kl(**{k: None}) == NULL, k
    for bad in (dict(s=P[0] + 1), dict(t=P[1] + 1), dict(ds=P[4] + 1), dict(w=P[2] + 2),
                dict(out=P[3] + 1), dict(ws=P[5] + 8)):
        assert kl(**bad) == ALIGN, bad
    for bad in (dict(ds=P[1]), dict(ds=P[0] + 2), dict(ds=P[0], ldd=1001), dict(out=P[0]),
                dict(out=P[1]), dict(out=P[2]), dict(out=P[4]), dict(ds=P[2])):
        assert kl(**bad) == ALIAS, bad
    need = head.af1_distill_kl_workspace_bytes(6, 1000)
    if need:
        assert kl(ws=None) == WS and kl(ws_bytes=need - 1) == WS
        assert kl(ws=P[0]) == ALIAS and kl(ws=P[1]) == ALIAS
    assert kl(T=0, s=None, t=None, out=None) == OK


def test_tensor_checks():
    z = torch.zeros(3, 8)
    for call in (lambda: output.token_logprobs(z), lambda: output.distill_kl(z, z),
                 lambda: output.Fp8Matrix.quantize(z),
                 lambda: output.Fp8Matrix(8, 8, "e4m3", z, z),
                 lambda: output.Fp8Matrix(8, 8, "int8", z, z)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("m,n", [(4096, 4096), (8192, 8192), (1024, 50257), (50257, 4096),
                                 (14336, 4096), (129, 2000), (20, 70)])
def test_one_workspace_for_fewer_tokens(m, n):
    need = [head.af1_fp8_linear_workspace_bytes(m, n, t) for t in range(1, 1101)]
    for T in (1, 5, 16, 17, 32, 33, 40, 64, 65, 100, 128, 129, 200, 257, 500, 640, 1000, 1100):
        assert output.workspace_up_to(m, n, T) >= max(need[:T])
    assert output.workspace_up_to(m, n, 0) == 0
