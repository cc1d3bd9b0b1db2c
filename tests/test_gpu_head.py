"""GPU tests of the output head and its losses against the fp64 oracle.

Tolerances are counted, not fitted.  u = 2^-24 is half a step of fp32.

Linear: products of two 8-bit values are exact and the scales powers of two.
Each of the (n/64) matrix instructions adds 64 products to the accumulator;
allowing every one of its additions a full step of what is in flight, which is
at most S = sum |x_j w_j|, bounds the error by (n/64 + 64) 2u S.  That holds for
outputs in fp32.  For outputs in bfloat16 the 8-bit instructions cut each
product 13 bits below the largest of the instruction: an error of less than
2^-13 of it for each of a block's 128 products, and the largest is at most
max_J |x| max_J |w| of the block J; the sum over the blocks is added.

Softmax: a term 2^t has a relative error of |t| ln2 2u (two roundings of t) and
2u (the exponential), the sum of V terms in any order at most V u more; t
beyond 40 contributes nothing at this accuracy.  So ln Z is within
eps = (60 + V) u of the truth when sums are sequential, and log probabilities,
entropies (whose terms are weighted by |t|) within eps (1 + |value|) (times 40
for the weights).  The bound holds for every order of summation."""
import numpy as np
import pytest
import torch

from oracle import head as H
from paper_2609_06161_amd import head, output as O, synth
from paper_2609_06161_amd.layer import DeviceLayer, to_device

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: U}
FLOOR = {torch.bfloat16: 2.0 ** -127, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -127}
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
DEV = "cuda"


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float32)


def within(got, want, bound):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    fin = np.isfinite(want)
    np.testing.assert_array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    bound = np.broadcast_to(bound, want.shape)
    over = np.abs(got - want)[fin] - bound[fin]
    worst = over.max() if over.size else -1.0
    assert worst <= 0, f"{(over > 0).sum()} of {over.size} beyond the bound, worst by {worst:.3g}"


# --------------------------------------------------------------------------
# the 8-bit matrix
# --------------------------------------------------------------------------

def wide(seed, rows, cols, dtype):
    """Entries over many binades, a block of zeros, and tiny and huge blocks."""
    width = 1 if dtype == torch.float16 else 4
    a = randn(seed, rows, cols) * torch.exp2(width * randn(seed + 1, rows, 1))
    a[:128, :128] = 0
    if cols > 128:
        a[:128, 128:256] *= 2.0 ** (-12 if dtype == torch.float16 else -126)
    if rows > 128:
        a[128:256, :128] *= 2.0 ** (4 if dtype == torch.float16 else 110)
    return a.to(dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (128, 128), (129, 127), (300, 515), (57, 1030)])
def test_quantize_bit_exact(rows, cols, fmt, dtype):
    a = wide(11, rows, cols, dtype)
    M = O.Fp8Matrix.quantize(a.to(DEV), fmt)
    codes, scales = H.quantize(f64(a), fmt)
    np.testing.assert_array_equal(M.scales.cpu().numpy(), scales.ravel())
    np.testing.assert_array_equal(M.codes.cpu().numpy(), codes.ravel())
    want = H.dequantize(codes, scales, rows, cols, fmt)
    np.testing.assert_array_equal(f64(M.dequantize(torch.float32)), want.astype(np.float32))
    np.testing.assert_array_equal(f64(M.dequantize(torch.bfloat16)),
                                  f64(torch.from_numpy(want).to(torch.float32).to(torch.bfloat16)))
    np.testing.assert_array_equal(f64(M.dequantize(torch.float16)),
                                  f64(torch.from_numpy(want).to(torch.float32).to(torch.float16)))


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantize_of_what_is_not_finite(fmt):
    a = randn(12, 40, 140)
    a[3, 5], a[3, 6], a[7, 130], a[20, 20] = np.nan, np.inf, -np.inf, -0.0
    M = O.Fp8Matrix.quantize(a.to(DEV), fmt)
    v = f64(M.dequantize(torch.float32))
    codes, scales = H.quantize(f64(a), fmt)
    np.testing.assert_array_equal(M.scales.cpu().numpy(), scales.ravel())
    np.testing.assert_array_equal(v, H.dequantize(codes, scales, 40, 140, fmt))
    assert np.isnan(v[3, 5]) and np.signbit(v[20, 20])
    assert (np.isnan if fmt == "e4m3" else np.isposinf)(v[3, 6])
    assert (np.isnan if fmt == "e4m3" else np.isneginf)(v[7, 130])


@pytest.mark.parametrize("rows,cols", [(1, 1), (128, 256), (300, 515), (129, 1000)])
def test_transpose_moves_codes(rows, cols):
    a = wide(13, rows, cols, torch.bfloat16).to(DEV)
    M, MT = O.Fp8Matrix.quantize(a), O.Fp8Matrix.quantize(a.T.contiguous())
    T = M.transpose()
    assert (T.rows, T.cols) == (cols, rows)
    assert torch.equal(T.codes, MT.codes) and torch.equal(T.scales, MT.scales)


# --------------------------------------------------------------------------
# the linear
# --------------------------------------------------------------------------

LINEAR = [(1, 1, 1), (1, 128, 128), (2, 129, 127), (3, 1000, 4096), (8, 300, 2080), (15, 64, 130),
          (16, 515, 256), (17, 200, 300), (31, 1030, 384), (32, 96, 1000), (33, 257, 128),
          (64, 512, 512), (65, 1000, 640), (100, 129, 2000), (128, 256, 1024), (129, 300, 515),
          (200, 2000, 260), (257, 513, 700), (500, 1024, 1024)]


def linear_bound(ydtype, x, codes, scales, m, n, wfmt, xfmt, want, S):
    acc = (n / 64 + 64) * 2 * U * S
    if ydtype == torch.float32:
        return acc
    W, q = H.dequantize(codes, scales, m, n, wfmt), H.round_rows(x, xfmt)
    for j in range(0, n, 128):
        acc = acc + 128 * 2.0 ** -13 * np.outer(np.abs(q[:, j:j + 128]).max(1),
                                                np.abs(W[:, j:j + 128]).max(1))
    return acc + HALF[ydtype] * (np.abs(want) + acc)


def check_linear(T, m, n, wfmt="e4m3", xfmt="e4m3", xdtype=torch.bfloat16, ydtype=torch.float32,
                 xscale=1.0, layer=None, x=None):
    x = randn(21, T, n) * torch.exp2(2 * randn(22, T, 1)) * xscale if x is None else x
    x = x.to(xdtype)
    w = randn(23, m, n) * torch.exp2(2 * randn(24, m, 1)) * n ** -0.5
    layer = O.Fp8Linear.from_dense(w.to(DEV), wfmt) if layer is None else layer
    y = layer.forward(x.to(DEV), fmt=xfmt, dtype=ydtype)
    assert y.shape == (T, m) and y.dtype == ydtype
    codes, scales = H.quantize(f64(w), wfmt)
    want, S = H.linear(f64(x), codes, scales, m, n, wfmt, xfmt)
    within(f64(y), want, linear_bound(ydtype, f64(x), codes, scales, m, n, wfmt, xfmt, want, S))
    return layer, x, w, y


@pytest.mark.parametrize("T,m,n", LINEAR)
def test_linear(T, m, n):
    print(f"linear T={T} m={m} n={n}", flush=True)
    check_linear(T, m, n)


@pytest.mark.parametrize("T,m,n", [(1, 300, 515), (13, 1000, 256), (40, 129, 2000), (300, 520, 515)])
@pytest.mark.parametrize("wfmt,xfmt,xdtype,ydtype", [
    ("e4m3", "e4m3", torch.float32, torch.bfloat16), ("e5m2", "e4m3", torch.float16, torch.float32),
    ("e4m3", "e5m2", torch.bfloat16, torch.bfloat16), ("e5m2", "e5m2", torch.float32, torch.bfloat16)])
def test_linear_types(T, m, n, wfmt, xfmt, xdtype, ydtype):
    check_linear(T, m, n, wfmt, xfmt, xdtype, ydtype)


def test_linear_int16_patterns_and_given_arrays():
    layer, x, _, y = check_linear(20, 300, 640, ydtype=torch.bfloat16)
    out = torch.full((20, 300), -1, dtype=torch.int16, device=DEV)
    ws = layer.workspace(64).fill_(255)        # what is in it does not matter
    got = layer.forward(x.to(DEV).view(torch.int16), out, ws)
    assert got is out and torch.equal(out.view(torch.bfloat16), y)


@pytest.mark.parametrize("T", [1, 5, 16, 40, 200])
def test_linear_extreme_rows(T):
    """Rows of zeros, tiny and huge rows, NaN and infinity in some; a row's
    result depends on that row only."""
    n, m = 400, 300
    x = randn(31, T, n)
    x[0] *= 2.0 ** -120
    if T > 1:
        x[1] *= 2.0 ** 100
        x[2] = 0
        x[3, 7] = float("nan")
        x[4, 390] = float("inf")
    layer, _, _, y = check_linear(T, m, n, x=x, xdtype=torch.float32)
    if T > 1:
        assert (y[2] == 0).all() and torch.isnan(y[3]).all() and torch.isnan(y[4]).all()


@pytest.mark.parametrize("T,m,n", [(1, 300, 515), (7, 1000, 257), (50, 129, 640), (260, 515, 300)])
def test_linear_input_gradient(T, m, n):
    """dx = dy W through the transposed copy, gradients of a small magnitude."""
    w, dy = randn(41, m, n) * n ** -0.5, randn(42, T, m) * torch.exp2(-20 + 3 * randn(43, T, m))
    dy = dy.to(torch.bfloat16)
    layer = O.Fp8Linear.from_dense(w.to(DEV))
    dx = layer.input_grad(dy.to(DEV), dtype=torch.float32)
    codes, scales = H.quantize(f64(w).T, "e4m3")
    want, S = H.linear(f64(dy), codes, scales, n, m, "e4m3", "e5m2")
    within(f64(dx), want, (m / 64 + 64) * 2 * U * S)


def test_linear_zero_tokens():
    layer = O.Fp8Linear.from_dense(randn(44, 130, 70).to(DEV))
    assert layer.forward(torch.empty((0, 70), device=DEV)).shape == (0, 130)


def test_linear_repeats_bit_for_bit():
    for T, m, n in ((1, 1000, 4096), (16, 4096, 1000), (70, 700, 4096), (300, 640, 2000)):
        layer = O.Fp8Linear.from_dense(randn(45, m, n).to(DEV))
        x = randn(46, T, n).to(DEV)
        first = layer.forward(x)
        for _ in range(3):
            assert torch.equal(layer.forward(x), first)


# --------------------------------------------------------------------------
# log probabilities
# --------------------------------------------------------------------------

def logits(seed, T, V, dtype, width=3.0):
    z = randn(seed, T, V) * width
    z[:, V // 2] += 6.0
    return z.to(dtype)


def softmax_eps(V):
    return (60 + V) * U


def gradient_bound(x, scale, gl, gh, dtype, want):
    """A probability is within softmax_eps and |log p| 4u of the truth; the
    gradient's factors multiply that; the result rounds to its type."""
    V = x.shape[1]
    lp = np.maximum(H.log_softmax(x, scale), -200.0)
    p, Hh = np.exp(lp), -H.xlogx(np.exp(lp), lp).sum(1, keepdims=True)
    rel = softmax_eps(V) + 4 * U * np.abs(lp) + 8 * U
    size = np.abs(gl)[:, None] + np.abs(gh)[:, None] * (np.abs(lp) + np.abs(Hh) + 40)
    acc = scale * (p * size * rel + 4 * U * (np.abs(want) / scale + np.abs(gl)[:, None] * (p > 1e-3)))
    return np.nan_to_num(acc + HALF[dtype] * (np.abs(want) + acc) + FLOOR[dtype], nan=0.0)


def check_logprobs(z, y, k, scale, top_only_index=False):
    got = O.token_logprobs(z, y, k, scale)
    x = f64(z)
    V = x.shape[1]
    eps = softmax_eps(V)
    yy = y.cpu().numpy() if y is not None else np.zeros(len(x), np.int64)
    with np.errstate(all="ignore"):
        lp, ent = H.token_logprobs(x, yy, scale)
        lse = H.lse(x, scale)
        if y is not None:
            within(got.logprob.cpu(), lp, eps + 4 * U * (np.abs(lp) + 1))
        within(got.entropy.cpu(), ent, 40 * eps + 4 * U * np.abs(ent))
        within(got.lse.cpu(), lse, eps + 4 * U * (np.abs(lse) + 1))
    if k:
        idx = H.top(x, k)
        np.testing.assert_array_equal(got.top_index.cpu().numpy(), idx)
        with np.errstate(all="ignore"):
            want = np.where(idx < 0, -np.inf,
                            np.take_along_axis(H.log_softmax(x, scale), np.maximum(idx, 0), 1))
            within(got.top_logprob.cpu(), want, eps + 4 * U * (np.abs(want) + 1))
    return got


VOCABS = [1, 2, 7, 8, 9, 63, 64, 65, 255, 1000, 4097, 20011]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", VOCABS)
def test_logprobs(V, dtype):
    for T, k, scale in ((1, 20, 1.0), (5, 0, 0.5), (3, 32, 1.25)):
        print(f"logprobs T={T} V={V} {dtype} k={k}", flush=True)
        z = logits(V + T, T, V, dtype).to(DEV)
        y = torch.arange(T, device=DEV) * 7919 % V
        check_logprobs(z, y, k, scale)


@pytest.mark.parametrize("T,V,k", [(1, 128256, 20), (2, 150001, 1), (70, 33000, 5), (600, 5003, 7),
                                   (1500, 301, 3)])
def test_logprobs_sizes(T, V, k):
    z = logits(V, T, V, torch.bfloat16).to(DEV)
    check_logprobs(z, torch.arange(T, device=DEV) % V, k, 1.0)


@pytest.mark.parametrize("T", [1, 4, 300])
def test_logprobs_ties_and_order(T):
    """Equal logits come in the order of their indices: constant rows, rows of
    few values, ascending and descending rows."""
    V = 9000
    rows = [torch.zeros(V), (torch.arange(V) % 3).float(), torch.arange(V).float() * 2.0 ** -9,
            -torch.arange(V).float() * 2.0 ** -9]
    z = torch.stack([rows[i % 4] for i in range(T)])
    z[-1, 17], z[-1, 40] = -0.0, 0.0
    check_logprobs(z.to(DEV), torch.zeros(T, dtype=torch.int64, device=DEV), 32, 1.0)


@pytest.mark.parametrize("T", [6, 700])
@pytest.mark.parametrize("V", [40, 9001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_logprobs_masks(V, dtype, T):
    """Masked entries, whole rows of -infinity and of the type's lowest value,
    NaN and +infinity in a row; targets that are no tokens."""
    z = logits(50, T, V, dtype)
    z[0, 3:] = -float("inf")
    z[1] = -float("inf")
    z[2] = torch.finfo(dtype).min
    z[3, 1::2] = torch.finfo(dtype).min
    z[4, V // 3] = float("nan")
    z[5, V // 3] = float("inf")
    y = torch.zeros(T, dtype=torch.int64)
    y[3], y[T // 2], y[-1] = -100, V - 1, 1
    check_logprobs(z.to(DEV), y.to(DEV), 20, 1.0)
    bad = torch.tensor([V, V + 5, 1 << 40] + [0] * (T - 3))
    got = O.token_logprobs(z.to(DEV), bad.to(DEV))
    assert torch.isnan(got.logprob[:3]).all()


def test_logprobs_strides_and_slices():
    big = torch.full((9, 1111), float("nan"))
    big[1:8, 3:1004] = logits(51, 7, 1001, torch.float32)
    for dtype in DTYPES:
        z = big.to(dtype).to(DEV)[1:8, 3:1004]
        targets = (torch.arange(9, device=DEV) * 31)[1:8]
        got = check_logprobs(z, targets, 4, 1.0)
        want = O.token_logprobs(z.contiguous(), targets.clone(), 4)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def check_logprobs_grad(z, y, gl, gh, scale, **kw):
    st = O.token_logprobs(z, y, 0, scale)
    x = f64(z)      # before it may be written over
    d = O.token_logprobs_backward(z, y, st, gl, gh, scale, **kw)
    l64 = f64(gl) if gl is not None else np.zeros(len(x))
    h64 = f64(gh) if gh is not None else np.zeros(len(x))
    y64 = y.cpu().numpy() if y is not None else np.full(len(x), -1)
    with np.errstate(all="ignore"):
        want = H.token_logprobs_backward(x, y64, l64, h64, scale)
        within(f64(d), want, gradient_bound(x, scale, l64, h64, z.dtype, want))
    return d


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V", [(1, 1), (1, 20011), (3, 7), (5, 1000), (40, 4097), (600, 259)])
def test_logprobs_backward(T, V, dtype):
    z = logits(60 + V, T, V, dtype).to(DEV)
    y = torch.arange(T, device=DEV) * 7919 % V
    gl, gh = randn(61, T).to(DEV), randn(62, T).to(DEV)
    check_logprobs_grad(z, y, gl, gh, 1.25)
    check_logprobs_grad(z, y, gl, None, 1.0)
    check_logprobs_grad(z, None, None, gh, 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_logprobs_backward_masks_and_padding(dtype):
    T, V = 9, 3001
    z = logits(63, T, V, dtype)
    z[0, 3:] = -float("inf")
    z[1] = -float("inf")
    z[2] = torch.finfo(dtype).min
    z[3, 1::2] = torch.finfo(dtype).min
    z[4, 9] = float("nan")
    z[5, 9] = float("nan")
    gl, gh = torch.ones(T), torch.ones(T)
    gl[5] = gh[5] = 0.0                    # padding: its logits may hold anything
    y = torch.full((T,), 2)
    y[6], y[7] = -100, V
    d = check_logprobs_grad(z.to(DEV), y.to(DEV), gl.to(DEV), gh.to(DEV), 1.0)
    assert (d[1] == 0).all() and (d[5] == 0).all() and torch.isnan(d[4]).all()
    assert (d[0, 3:] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_logprobs_backward_in_place_and_strided(dtype):
    T, V = 6, 1003
    z = logits(64, T, V, dtype).to(DEV)
    y, gl = torch.arange(T, device=DEV), randn(65, T).to(DEV)
    want = check_logprobs_grad(z, y, gl, None, 1.0)
    out = torch.full((T, V + 5), 7.0, dtype=dtype, device=DEV)
    got = check_logprobs_grad(z, y, gl, None, 1.0, dlogits=out[:, 2:V + 2])
    assert torch.equal(got, want) and (out[:, :2] == 7).all() and (out[:, V + 2:] == 7).all()
    own = z.clone()
    got = check_logprobs_grad(own, y, gl, None, 1.0, dlogits=own)
    assert got is own and torch.equal(own, want)


# --------------------------------------------------------------------------
# KL divergence
# --------------------------------------------------------------------------

def kl_bound(xs, xt, scale):
    """kl = ln2 sum p u + ln(1 + sum p (2^-u - 1)).  A term p u errs by the
    rounding of u (two roundings of |x - w| scale, one of |u|) and by p's
    relative error; a term of the second sum by the exponential's 2u and u's
    rounding times q, and by its sum with p; V terms of each are summed in some
    order (V u of the absolute terms).  What the statistics are off by (eps)
    shifts u for all, which the two sums feel in opposite ways: second order."""
    V = xs.shape[1]
    lq, lp = (np.maximum(H.log_softmax(v, scale), -200.0) for v in (xs, xt))
    p, q, u = np.exp(lp), np.exp(lq), lp - lq
    gap = np.abs(np.where(np.isfinite(xs) & np.isfinite(xt), xs - xt, 0.0)) * scale
    eps = softmax_eps(V)
    du = 4 * U * (gap + np.abs(u) + 1)
    rel = eps + 4 * U * np.abs(lp) + 8 * U
    err = p * du + q * (du + 4 * U) + rel * (np.abs(p * u) + np.abs(q - p))
    # entries that the teacher masks take q from its own exponential
    err = err + np.where(p < 2.0 ** -100, q * (eps + 4 * U * np.abs(lq)), 0.0)
    return (err + V * U * (np.abs(p * u) + np.abs(q - p))).sum(1) + 2 * eps ** 2 + 4 * U * U


def check_kl(s, t, scale=1.0, w=None, **kw):
    xs, xt = f64(s), f64(t)
    kl, d = O.distill_kl(s, t, scale, w, **kw)
    w64 = f64(w) if w is not None else np.ones(len(xs))
    with np.errstate(all="ignore"):
        want = H.distill_kl(xs, xt, scale)
        empty = np.isneginf(xt).all(1)
        want = np.where(empty, 0.0, want)
        within(kl.cpu(), want, np.nan_to_num(kl_bound(xs, xt, scale), nan=0.0))
        if d is not None:
            dw = H.distill_kl_backward(xs, xt, w64, scale)
            q, p = (np.exp(np.maximum(H.log_softmax(v, scale), -200.0)) for v in (xs, xt))
            lq, lp = (np.maximum(H.log_softmax(v, scale), -200.0) for v in (xs, xt))
            rel = softmax_eps(xs.shape[1]) + 8 * U
            acc = np.abs(w64)[:, None] * scale * (q * (rel + 4 * U * np.abs(lq))
                                                  + p * (rel + 4 * U * np.abs(lp)))
            bound = acc + HALF[s.dtype] * (np.abs(dw) + acc) + FLOOR[s.dtype]
            within(f64(d), dw, np.nan_to_num(bound, nan=0.0))
    return kl, d


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V", [(1, 1), (1, 2), (1, 20011), (3, 7), (5, 1000), (40, 4097),
                                 (300, 1030), (600, 259)])
def test_distill_kl(T, V, dtype):
    print(f"kl T={T} V={V} {dtype}", flush=True)
    s = logits(70 + V, T, V, torch.float32)
    for noise, scale in ((0.3, 1.0), (3.0, 0.5), (0.003, 1.25)):
        t = (s + noise * randn(71, T, V)).to(dtype).to(DEV)
        check_kl(s.to(dtype).to(DEV), t, scale, randn(72, T).to(DEV))


def test_distill_kl_small_and_none():
    """Equal logits: nothing, and no negative values near it; without a
    gradient the loss is the same."""
    s = logits(73, 4, 5000, torch.float32).to(DEV)
    kl, d = O.distill_kl(s, s.clone())
    assert (kl == 0).all() and (d == 0).all()
    t = s + 1e-4 * randn(74, 4, 5000).to(DEV)
    a, _ = check_kl(s, t)
    b, none = O.distill_kl(s, t, grad=False)
    assert none is None and torch.equal(a, b) and (a >= 0).all()


@pytest.mark.parametrize("T", [9, 500])
@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_kl_masks_and_padding(dtype, T):
    V = 3001
    inf = float("inf")
    s, t = logits(75, T, V, dtype), logits(76, T, V, dtype)
    s[0, 5:90] = t[0, 5:90] = -inf              # both masked
    t[1, 7:] = -inf                             # the teacher masks more
    s[2, 11] = -inf                             # the student masks what has mass
    t[3] = -inf
    s[4] = -inf
    s[5] = t[5] = torch.finfo(dtype).min
    t[6, 1::2] = torch.finfo(dtype).min
    s[7, 3] = float("nan")
    s[8, 3] = float("nan")
    w = torch.ones(T)
    w[8] = 0.0
    kl, d = check_kl(s.to(DEV), t.to(DEV), 1.0, w.to(DEV))
    assert kl[3] == 0 and kl[2] == inf and kl[4] == inf and torch.isnan(kl[7:9]).all()
    assert (d[3] == 0).all() and (d[4] == 0).all() and (d[8] == 0).all()
    assert torch.isfinite(d[2]).all() and torch.isnan(d[7]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_kl_in_place_and_strided(dtype):
    T, V = 6, 1003
    s, t = logits(77, T, V, dtype).to(DEV), logits(78, T, V, dtype).to(DEV)
    kl, want = check_kl(s, t)
    pad = torch.full((T, V + 5), 7.0, dtype=dtype, device=DEV)
    a, b, out = pad.clone(), pad.clone(), pad.clone()
    a[:, 1:V + 1], b[:, 4:V + 4] = s, t
    k2, got = check_kl(a[:, 1:V + 1], b[:, 4:V + 4], dstudent=out[:, 2:V + 2])
    assert torch.equal(k2, kl) and torch.equal(got, want)
    assert (out[:, :2] == 7).all() and (out[:, V + 2:] == 7).all()
    own = s.clone()
    k3, got = check_kl(own, t, dstudent=own)
    assert got is own and torch.equal(k3, kl) and torch.equal(own, want)


def test_zero_tokens():
    z = torch.empty((0, 50), device=DEV)
    y = torch.empty(0, dtype=torch.int64, device=DEV)
    st = O.token_logprobs(z, y, 3)
    assert st.logprob.shape == (0,) and st.top_index.shape == (0, 3)
    assert O.token_logprobs_backward(z, y, st, st.logprob, st.entropy).shape == (0, 50)
    kl, d = O.distill_kl(z, z)
    assert kl.shape == (0,) and d.shape == (0, 50)


def test_rows_beyond_32_bit_offsets():
    """The last rows of logits whose byte offsets pass 2^32."""
    T, V = 33, 1 << 24
    ld = V + 7 * (1 << 23)
    big = torch.empty(T * ld, dtype=torch.bfloat16, device=DEV)
    z = big.as_strided((T, V), (ld, 1))
    assert (T - 1) * ld * 2 > 1 << 32
    z.zero_()
    z[-1, V - 1] = 20.0
    y = torch.full((T,), V - 1, device=DEV)
    st = O.token_logprobs(z, y, 1)
    lnV = np.log(V)
    # all terms are equal: sums are exact up to their rounding to 24 bits
    np.testing.assert_allclose(st.lse[:-1].cpu(), lnV, rtol=4 * U)
    want = -np.log1p((V - 1) * np.exp(-20.0))
    assert abs(st.logprob[-1].item() - want) <= softmax_eps(V) * abs(want) and st.top_index[-1, 0] == V - 1
    d = O.token_logprobs_backward(z, y, st, torch.ones(T, device=DEV), dlogits=z)
    p = (1 - np.exp(want)) / (V - 1)
    assert abs(d[-1, 0].item() + p) <= (2.0 ** -7) * p
    assert abs(d[-1, V - 1].item() - (1 - np.exp(want))) <= 2.0 ** -7


# --------------------------------------------------------------------------
# streams, graphs, and a run of all of them
# --------------------------------------------------------------------------

def decode(head8, h, y, k, ws):
    z = head8.forward(h, ws=ws, dtype=torch.float32)
    return O.token_logprobs(z, y, k)


def test_other_stream():
    layer = O.Fp8Linear.from_dense(randn(80, 3000, 512).to(DEV))
    h, y = randn(81, 4, 512).to(DEV), torch.tensor([1, 2, 3, 2999], device=DEV)
    want = decode(layer, h, y, 5, None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    z = layer.forward(h, dtype=torch.float32, stream=s)
    got = O.token_logprobs(z, y, 5, stream=s)
    d = O.token_logprobs_backward(z, y, got, torch.ones(4, device=DEV), stream=s)
    s.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert torch.isfinite(d).all()


def test_one_workspace_for_fewer_tokens():
    """A workspace for 500 tokens serves calls of fewer, which need more of it."""
    layer = O.Fp8Linear.from_dense(randn(3, 4096, 4096).to("cuda"))
    ws = layer.workspace(500)
    for T in (500, 130, 45, 17, 1):
        x = randn(T, T, 4096).to("cuda")
        assert torch.equal(layer.forward(x, ws=ws), layer.forward(x))


def test_two_calls_at_once():
    """Calls that overlap in time on two streams give what they give alone; the
    divergence's rows are work of several blocks that wait for each other."""
    layer = O.Fp8Linear.from_dense(randn(4, 3001, 1000).to("cuda"))
    x = [randn(5 + i, 45, 1000).to("cuda") for i in range(2)]
    z = [randn(7 + i, 40, 130000).to("cuda") for i in range(3)]
    y = torch.zeros(40, dtype=torch.int64, device="cuda")

    def calls(i):
        kl, grad = O.distill_kl(z[i], z[2])
        p = O.token_logprobs(z[i], y, 7)
        return [kl, grad, p.logprob, p.entropy, p.top_index, layer.forward(x[i])]

    alone = [calls(0), calls(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        got = [None, None]
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = calls(i)
        torch.cuda.synchronize()
        for g, w in zip(got[0] + got[1], alone[0] + alone[1]):
            assert torch.equal(g, w)


def test_transposed_weight_is_not_captured():
    """The transposed weight is made outside a graph, and once made it is used
    by calls on other streams."""
    layer = O.Fp8Linear.from_dense(randn(1, 300, 515).to("cuda"))
    dy = randn(2, 45, 300).to("cuda")
    dx = torch.zeros((45, 515), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError, match="transposed"):
            layer.input_grad(dy, dx)
        dx.zero_()
    side = torch.cuda.Stream()
    first = layer.input_grad(dy, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(layer.input_grad(dy), first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.input_grad(dy, dx)
    for _ in range(3):
        dx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dx, first)


def test_captured_graphs():
    """A decode step and a training step captured, replayed on new inputs with
    eager work between the replays."""
    layer = O.Fp8Linear.from_dense(randn(82, 5000, 640).to(DEV))
    layer.transposed()
    h, y = torch.empty((3, 640), device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV)
    t = randn(83, 3, 5000).to(DEV)

    def train():
        z = layer.forward(h, dtype=torch.float32)
        kl, dz = O.distill_kl(z, t)
        return kl, layer.input_grad(dz)

    def step():
        return [*decode(layer, h, y, 4, None), *train()]

    h.copy_(randn(84, 3, 640))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        h.copy_(randn(85 + i, 3, 640))
        y.copy_(torch.tensor([i, 7 * i, 4999 - i]))
        want = [a.clone() for a in step()]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T,dtype", [(3, torch.float32), (80, torch.float32), (80, torch.bfloat16)])
def test_reconstruction_step(oracle, T, dtype):
    """A scale-only step of a factorized linear below the head, against the
    oracles' fp64 chain.  The chain rounds to bfloat16 (hidden states, their
    gradient: 2^-8) and to 8 bits (activations 2^-4, gradients 2^-3); the
    oracle makes the same 8-bit roundings from its own values, so a rounding
    that falls the other way moves an entry by a whole step of them; entries of
    random sign add up in squares, so the norms stay within a step."""
    m, n, r, V = 512, 768, 224, 1500
    lin = synth.make_linear(90, m, n, r, T)
    # scales of a trained layer: outputs of the inputs' magnitude
    lin.s_mid = synth.f32_to_f16_bits(lin.s_mid.view(np.float16).astype(np.float32) * n ** -0.5)
    lin.s_out = synth.f32_to_f16_bits(lin.s_out.view(np.float16).astype(np.float32) * r ** -0.5)
    L = DeviceLayer.from_host(lin)
    w = randn(91, V, m) * m ** -0.5
    head8 = O.Fp8Linear.from_dense(w.to(DEV))
    teacher = (randn(92, T, V) * 2).to(dtype)
    weight = torch.full((T,), 1.0 / T)
    weight[0] = 0.0
    kl, dx, grads = O.reconstruction_step(L, head8, to_device(lin.x), teacher.to(DEV),
                                          weight.to(DEV))
    hid = oracle.forward(m, n, r, lin.Bu, lin.Bv, lin.s_out, lin.s_mid, lin.s_in, lin.x)
    hid = f64(torch.from_numpy(hid).to(torch.bfloat16))
    codes, scales = H.quantize(f64(w), "e4m3")
    z, _ = H.linear(hid, codes, scales, V, m, "e4m3", "e4m3")
    want = H.distill_kl(z, f64(teacher))
    assert np.linalg.norm(f64(kl) - want) <= 2.0 ** -6 * np.linalg.norm(want)
    dz = H.distill_kl_backward(z, f64(teacher), f64(weight))
    ct, st = H.quantize(f64(w).T, "e4m3")
    dh, _ = H.linear(dz, ct, st, m, V, "e4m3", "e5m2")
    ref = oracle.backward(m, n, r, lin.Bu, lin.Bv, lin.s_out, lin.s_mid, lin.s_in, lin.x,
                          synth.f32_to_bf16_bits(dh.astype(np.float32)))
    for got, e in zip((dx.view(torch.bfloat16), *grads), ref):
        assert np.linalg.norm(f64(got) - e) <= 2.0 ** -3 * np.linalg.norm(e)
    assert (dx[0] == 0).all()          # weight 0: no gradient
