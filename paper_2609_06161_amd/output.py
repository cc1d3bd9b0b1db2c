"""The output head on torch tensors: the 8-bit block-scaled linear, the log
probabilities of given tokens and the KL divergence to a teacher, as plain
calls that check their tensors, provide outputs and workspaces where none are
given, and forward to the C entry points (include/af1_head.h).

Every call runs on the device of its tensors, on `stream` (a torch stream or the
handle of one) or that device's current stream, and what it allocates belongs to
that stream.  bfloat16 tensors may also be given as int16 bit patterns, the
form in which DeviceLayer returns its outputs.  Workspaces (`ws`) are optional;
one that is passed in must not be used by another call at the same time, which
two captured graphs that share it would do if they were replayed together.
"""
import contextlib
from typing import NamedTuple, Optional

import torch

from . import af1, head
from .layer import on_stream

FORMATS = {"e4m3": head.AF1_FP8_E4M3, "e5m2": head.AF1_FP8_E5M2}
DENSE = {torch.float32: af1.AF1_SRC_F32, torch.bfloat16: af1.AF1_SRC_BF16,
         torch.float16: af1.AF1_SRC_F16, torch.int16: af1.AF1_SRC_BF16}


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _dense(t, name):
    """af1's type code of a dense GPU tensor."""
    code = DENSE.get(t.dtype) if isinstance(t, torch.Tensor) and t.is_cuda else None
    if code is None:
        raise ValueError(f"{name} must be a GPU tensor of float32, bfloat16, float16 or int16 "
                         "(bfloat16 patterns)")
    return code


def _array(t, name, device, dtype, shape):
    """Checks an optional contiguous array of a call."""
    if t is None or (t.dtype is dtype and t.shape == shape and t.device == device
                     and t.is_contiguous()):
        return
    raise ValueError(f"{name} must be {dtype}, contiguous, of shape {tuple(shape)}, on {device}, not "
                     f"{t.dtype} of shape {tuple(t.shape)} on {t.device}")


def _workspace(ws, need, device):
    """(workspace, its bytes)."""
    if ws is None:
        return (torch.empty(need, dtype=torch.uint8, device=device), need) if need else (None, 0)
    _need(ws.device == device and ws.is_contiguous(), f"ws must be contiguous on {device}")
    return ws, ws.numel() * ws.element_size()


@contextlib.contextmanager
def _on(device, stream):
    """The device of the tensors and the stream that the kernels run on."""
    with torch.cuda.device(device), on_stream(stream, device):
        yield


def _run(call, device, stream, *args):
    """call(*args, stream) on the tensors' device and the given stream, or that
    device's current one.  Entering a device and a stream costs as much as the
    smallest kernels, so it is left out where both are current already."""
    if stream is None or isinstance(stream, int):
        index = device.index
        if index == torch._C._cuda_getDevice():
            current = torch._C._cuda_getCurrentRawStream(index)
            if stream is None or stream == current:
                return call(*args, current)
    with _on(device, stream):
        return call(*args, stream)


class Fp8Matrix:
    """A rows x cols matrix in 8-bit floating point ("e4m3" or "e5m2") with a
    power-of-two scale for each block of 128 x 128: codes and scales as uint8
    tensors in the storage of af1_fp8_matrix."""

    def __init__(self, rows, cols, fmt, codes, scales):
        _need(fmt in FORMATS, f"fmt must be one of {tuple(FORMATS)}, not {fmt!r}")
        self.rows, self.cols, self.fmt = int(rows), int(cols), fmt
        _need(head.af1_fp8_code_bytes(self.rows, self.cols) > 0,
              f"rows and cols must be in 1..{af1.AF1_MAX_DIM}, not {rows} x {cols}")
        for t, need, name in ((codes, head.af1_fp8_code_bytes(self.rows, self.cols), "codes"),
                              (scales, head.af1_fp8_scale_bytes(self.rows, self.cols), "scales")):
            _need(isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.uint8
                  and t.is_contiguous() and t.numel() == need,
                  f"{name} must be a contiguous GPU tensor of {need} uint8")
        _need(codes.device == scales.device, "codes and scales must be on one device")
        self.codes, self.scales = codes, scales
        self.desc = head.make_matrix(self.rows, self.cols, FORMATS[fmt], codes, scales)

    @property
    def device(self):
        return self.codes.device

    @classmethod
    def empty(cls, rows, cols, fmt="e4m3", device="cuda"):
        code, scale = head.af1_fp8_code_bytes(rows, cols), head.af1_fp8_scale_bytes(rows, cols)
        return cls(rows, cols, fmt, torch.empty(code, dtype=torch.uint8, device=device),
                   torch.empty(scale, dtype=torch.uint8, device=device))

    @classmethod
    def quantize(cls, src, fmt="e4m3", out=None, stream=None):
        """The 8-bit form of a dense contiguous matrix."""
        dtype = _dense(src, "src")
        _need(src.dim() == 2 and src.is_contiguous(), "src must be a contiguous matrix")
        _need(fmt in FORMATS, f"fmt must be one of {tuple(FORMATS)}, not {fmt!r}")
        rows, cols = src.shape
        _need(out is None or ((out.rows, out.cols, out.fmt) == (rows, cols, fmt)
                              and out.device == src.device),
              f"out must be a {rows} x {cols} {fmt} matrix on {src.device}")

        def call(stream):
            M = cls.empty(rows, cols, fmt, src.device) if out is None else out
            head.af1_fp8_quantize(src, dtype, rows, cols, FORMATS[fmt], M.codes, M.scales, stream)
            return M

        return _run(call, src.device, stream)

    def dequantize(self, dtype=torch.bfloat16, out=None, stream=None):
        """The values that the matrix stands for."""
        _need(dtype in DENSE, f"dtype must be one of {tuple(DENSE)}, not {dtype}")
        _array(out, "out", self.device, dtype, (self.rows, self.cols))

        def call(stream):
            dst = out
            if dst is None:
                dst = torch.empty((self.rows, self.cols), dtype=dtype, device=self.device)
            head.af1_fp8_dequantize(self.desc, dst, DENSE[dtype], stream)
            return dst

        return _run(call, self.device, stream)

    def transpose(self, stream=None):
        """The transposed matrix; codes and scales are moved, nothing rounds."""
        def call(stream):
            T = Fp8Matrix.empty(self.cols, self.rows, self.fmt, self.device)
            head.af1_fp8_transpose(self.desc, T.codes, T.scales, stream)
            return T

        return _run(call, self.device, stream)


class Fp8Linear:
    """y = x W^T with W an Fp8Matrix of m = rows by n = cols.  Activations are
    rounded to 8 bits inside the call, each token's 128 columns at a scale of
    their own.  Sums are fp32 for outputs in fp32 and for up to 16 tokens; for
    more tokens with outputs in bfloat16 (the default) each eight columns'
    products are cut below 2^-13 of their largest before that (af1_fp8_linear)."""

    def __init__(self, weight, transposed=None):
        self.weight = weight
        self.m, self.n = weight.rows, weight.cols
        if transposed is not None:
            _need((transposed.rows, transposed.cols) == (self.n, self.m),
                  f"transposed must be {self.n} x {self.m}")
        self._T = transposed

    @classmethod
    def from_dense(cls, w, fmt="e4m3", stream=None):
        return cls(Fp8Matrix.quantize(w, fmt, stream=stream))

    def transposed(self, stream=None):
        """The weight transposed, made once (the weight is frozen) and complete
        when this returns, since calls on any stream use it from then on.  The
        first call, or the first input_grad, cannot be captured into a graph:
        the copy would exist only after a replay."""
        if self._T is None:
            dev = self.weight.device
            with _on(dev, stream):
                _need(not torch.cuda.is_current_stream_capturing(),
                      "call transposed() before input_grad is captured into a graph")
                T = self.weight.transpose()
                torch.cuda.current_stream().synchronize()
            self._T = T
        return self._T

    def workspace(self, T, grad=False):
        """A workspace for calls of up to T tokens."""
        m, n = (self.n, self.m) if grad else (self.m, self.n)
        _need(0 <= T <= head.AF1_HEAD_MAX_TOKENS, f"T must be at most {head.AF1_HEAD_MAX_TOKENS}")
        return torch.empty(max(workspace_up_to(m, n, T), 16), dtype=torch.uint8,
                           device=self.weight.device)

    def forward(self, x, y=None, ws=None, fmt="e4m3", dtype=torch.bfloat16, stream=None):
        """[T, n] -> [T, m] of y's type, or of `dtype` (float32, bfloat16)."""
        return _linear(self.weight, x, y, ws, fmt, dtype, stream)

    def input_grad(self, dy, dx=None, ws=None, fmt="e5m2", dtype=torch.bfloat16, stream=None):
        """dx = dy W, [T, m] -> [T, n]."""
        return _linear(self.transposed(stream), dy, dx, ws, fmt, dtype, stream)


def workspace_up_to(m, n, T):
    """Bytes that cover every 8-bit linear of 1 to T tokens.  Fewer tokens may
    need more: they are split over more ranges of columns.  Between these steps
    the ranges only become fewer, so a step's need grows at most as its tokens."""
    need = head.af1_fp8_linear_workspace_bytes(m, n, min(T, 16))
    for first, last in [(17, 32), (33, 64)] + [(t, t + 63) for t in range(65, T + 1, 64)]:
        if first <= T:
            here = head.af1_fp8_linear_workspace_bytes(m, n, first)
            need = max(need, -(-here * min(last, T) // first))
    return need


def _linear(W, x, y, ws, fmt, dtype, stream):
    x_dtype, dev = _dense(x, "x"), W.codes.device
    if fmt not in FORMATS:
        raise ValueError(f"fmt must be one of {tuple(FORMATS)}, not {fmt!r}")
    if x.dim() != 2 or x.shape[1] != W.cols or not x.is_contiguous() or x.device != dev:
        raise ValueError(f"x must be contiguous of shape [T, {W.cols}] on {dev}")
    if y is not None:
        _array(y, "y", dev, y.dtype, (x.shape[0], W.rows))
    return _run(_linear_call, dev, stream, W, x, x_dtype, FORMATS[fmt], y, dtype, ws)


def _linear_call(W, x, x_dtype, fmt, y, dtype, ws, stream):
    T, dev = x.shape[0], x.device
    if y is None:
        y = torch.empty((T, W.rows), dtype=dtype, device=dev)
    ws, size = _workspace(ws, head.af1_fp8_linear_workspace_bytes(W.rows, W.cols, T)
                          if ws is None else 0, dev)
    head.af1_fp8_linear(W.desc, x, x_dtype, fmt, T, y, _dense(y, "y"), ws, size, stream)
    return y


def _logits(t, name):
    """(dtype code, T, V, row stride) of a [T, V] tensor whose rows may be apart."""
    dtype, shape = _dense(t, name), t.shape
    if len(shape) != 2 or shape[1] < 1:
        raise ValueError(f"{name} must be [T, V]")
    T, V = shape
    ld, step = t.stride()
    if V > 1 and step != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    if T <= 1:
        ld = V
    elif ld < V:
        raise ValueError(f"{name}'s rows must not overlap")
    return dtype, T, V, ld


class TokenLogprobs(NamedTuple):
    """What token_logprobs gives: fp32[T] each, the alternatives [T, k], and
    `saved` for its backward."""
    logprob: Optional[torch.Tensor]
    entropy: torch.Tensor
    lse: torch.Tensor
    top_logprob: Optional[torch.Tensor]
    top_index: Optional[torch.Tensor]
    saved: torch.Tensor


def token_logprobs(logits, targets=None, k=0, scale=1.0, ws=None, stream=None):
    """Log probabilities of the given tokens under softmax(scale * logits), the
    entropy, and the k most likely tokens (af1_token_logprobs)."""
    rows, dev = _logits(logits, "logits"), logits.device
    T = rows[1]
    _array(targets, "targets", dev, torch.int64, (T,))
    if not 0 <= k <= head.AF1_HEAD_MAX_TOP:
        raise ValueError(f"k must be in 0..{head.AF1_HEAD_MAX_TOP}, not {k}")
    return _run(_logprobs_call, dev, stream, logits, rows, targets, k, scale, ws)


def _logprobs_call(logits, rows, targets, k, scale, ws, stream):
    dtype, T, V, ld = rows
    dev = logits.device
    need = head.af1_token_logprobs_workspace_bytes(T, V, k) if ws is None else 0
    # one block: the saved rows and the workspace first, which are aligned to 16
    # bytes, then what belongs to tokens
    saved, own, entropy, lse, logprob, top = torch.empty(
        (7 + k) * T + need // 4, dtype=torch.float32, device=dev).split_with_sizes(
            (4 * T, need // 4, T, T, T, k * T))
    index = None
    if targets is None:
        logprob = None
    if k:
        top, index = top.view(T, k), torch.empty((T, k), dtype=torch.int64, device=dev)
    else:
        top = None
    ws, size = (own, need) if ws is None else _workspace(ws, 0, dev)
    head.af1_token_logprobs(logits, dtype, T, V, ld, scale, targets, logprob, entropy, lse, k, top,
                            index, saved, ws, size, stream)
    return TokenLogprobs(logprob, entropy, lse, top, index, saved.view(T, 4))


def token_logprobs_backward(logits, targets, result, g_logprob=None, g_entropy=None, scale=1.0,
                            dlogits=None, stream=None):
    """The logits' gradient for the gradients of token_logprobs' logprob and
    entropy (either may be None); `result` is what it returned.  dlogits may be
    the logits themselves."""
    dtype, T, V, ld = _logits(logits, "logits")
    dev = logits.device
    _array(targets, "targets", dev, torch.int64, (T,))
    _array(g_logprob, "g_logprob", dev, torch.float32, (T,))
    _array(g_entropy, "g_entropy", dev, torch.float32, (T,))
    _array(result.saved, "result.saved", dev, torch.float32, (T, 4))
    _need(g_logprob is None or targets is not None, "g_logprob needs targets")

    def call(stream):
        out, ldd = _gradient(dlogits, logits)
        head.af1_token_logprobs_backward(logits, dtype, T, V, ld, scale, targets, result.saved,
                                         g_logprob, g_entropy, out, ldd, stream)
        return out

    return _run(call, dev, stream)


def _gradient(out, logits):
    """(gradient, its row stride)."""
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        return out, logits.shape[1]
    _need(out.dtype == logits.dtype and out.shape == logits.shape
          and out.device == logits.device, "the gradient must match the logits")
    return out, _logits(out, "the gradient")[3]


def distill_kl(student, teacher, scale=1.0, weight=None, grad=True, dstudent=None, ws=None,
               stream=None):
    """(kl, dstudent): each token's KL divergence from softmax(scale * teacher)
    to softmax(scale * student), and the student logits' gradient of
    sum_t weight[t] kl[t] (weight None: ones; grad False: None).  dstudent may
    be the student itself."""
    dtype, T, V, ld_s = _logits(student, "student")
    t_dtype, _, _, ld_t = _logits(teacher, "teacher")
    dev = student.device
    _need(teacher.shape == student.shape and t_dtype == dtype and teacher.device == dev,
          "student and teacher must have one shape, type and device")
    _array(weight, "weight", dev, torch.float32, (T,))

    def call(stream):
        out, ldd = None, 0
        if grad or dstudent is not None:
            out, ldd = _gradient(dstudent, student)
        need = head.af1_distill_kl_workspace_bytes(T, V) if ws is None else 0
        # one block, the workspace first for its alignment
        wk, kl = torch.empty(need // 4 + T, dtype=torch.float32, device=dev).split_with_sizes(
            (need // 4, T))
        wk, size = (wk, need) if ws is None else _workspace(ws, 0, dev)
        head.af1_distill_kl(student, teacher, dtype, T, V, ld_s, ld_t, scale, weight, kl, out, ldd,
                            wk, size, stream)
        return kl, out

    return _run(call, dev, stream)


def reconstruction_step(layer, output, x, teacher, weight=None, scale=1.0, grads=None,
                        accumulate=False, want_dx=True, stream=None):
    """One step of the scale-only reconstruction (Sec. 4.1, label
    eq:scale_only_kl) for a factorized linear below an 8-bit output head: the
    student logits head(layer(x)), their KL divergence to the teacher's, and
    the gradients of the layer's three scale vectors and of x.

    layer: DeviceLayer; output: Fp8Linear with n = layer.m; x: [T, layer.n]
    bfloat16; teacher: [T, V] logits (float32 or bfloat16).  Returns (kl [T],
    dx or None, (ds_out, ds_mid, ds_in)); the sum of weight * kl is the loss.
    A padding token (weight 0) may have any teacher row, its x has to be finite;
    a kl of it that is not finite is returned as 0."""
    _need(output.n == layer.m, f"the head reads {output.n} features, the layer gives {layer.m}")
    _need(teacher.dtype in (torch.float32, torch.bfloat16), "teacher must be float32 or bfloat16")
    xb = x.view(torch.int16) if x.dtype == torch.bfloat16 else x
    with _on(x.device, stream):     # the layer's own calls stay on the current device
        hidden, saved = layer.forward_train(xb)
        logits = output.forward(hidden, dtype=teacher.dtype)
        # the gradient takes the logits' place
        kl, dlogits = distill_kl(logits, teacher, scale, weight, dstudent=logits)
        dh = output.input_grad(dlogits)
        dx, grads = layer.backward(xb, dh.view(torch.int16), saved, grads=grads,
                                   accumulate=accumulate, want_dx=want_dx)
        if weight is not None:
            kl = torch.where(weight == 0, kl.nan_to_num(0.0, 0.0), kl)
    return kl, dx, grads
