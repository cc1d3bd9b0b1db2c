"""fp64 oracle of the output head and its losses (numpy, CPU), written from the
definitions in include/af1_head.h and sharing no code with the GPU path.

8-bit values are enumerated from the formats' definitions (OCP e4m3 and e5m2)
and codes found by search among them; softmaxes, divergences and gradients are
the textbook sums."""
import numpy as np

BLK = 128
MAX = {"e4m3": 448.0, "e5m2": 57344.0}


def code_values(fmt):
    """The value of every code 0..255 (NaN where it is one)."""
    man, bias = (3, 7) if fmt == "e4m3" else (2, 15)
    out = np.empty(256)
    for c in range(256):
        sign = -1.0 if c & 0x80 else 1.0
        e, f = (c & 0x7f) >> man, c & ((1 << man) - 1)
        if e == 0:
            v = f * 2.0 ** (1 - bias - man)
        else:
            v = (1 + f / 2 ** man) * 2.0 ** (e - bias)
        if fmt == "e4m3" and (c & 0x7f) == 0x7f:
            v = np.nan
        if fmt == "e5m2" and e == 31:
            v = np.inf if f == 0 else np.nan
        out[c] = sign * v
    return out


def encode(v, fmt):
    """Codes of values within the format's range, rounded to nearest, ties to
    the even code; NaN to 0x7f, infinities to 0x7f (e4m3) or 0x7c (e5m2)."""
    grid = code_values(fmt)[:0x7f if fmt == "e4m3" else 0x7c]     # 0, ascending
    a = np.abs(np.asarray(v, np.float64))
    hi = np.clip(np.searchsorted(grid, a), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.isfinite(a), code, 0x7f if fmt == "e4m3" else 0x7c)
    code = np.where(np.isnan(a), 0x7f, code).astype(np.uint8)
    return code | np.where(np.signbit(v), 0x80, 0).astype(np.uint8)


def exponent(amax, fmt):
    """Smallest e with amax <= MAX 2^e, at least -127; 0 for 0."""
    e = np.full(np.shape(amax), 127)
    for k in range(126, -128, -1):
        e = np.where(amax <= MAX[fmt] * 2.0 ** k, k, e)
    return np.where(amax == 0, 0, e)


def finite_max(v, axis):
    return np.max(np.where(np.isfinite(v), np.abs(v), 0.0), axis=axis)


def tiles(a):
    """[R, C, 128, 128], zero outside the matrix."""
    r, c = a.shape
    R, C = -(-r // BLK), -(-c // BLK)
    p = np.zeros((R * BLK, C * BLK))
    p[:r, :c] = a
    return p.reshape(R, BLK, C, BLK).transpose(0, 2, 1, 3)


def quantize(a, fmt):
    """(codes [R, C, 128, 128], scale bytes [R, C]) of a matrix."""
    t = tiles(np.asarray(a, np.float64))
    e = exponent(finite_max(t, (2, 3)), fmt)
    return encode(t * 2.0 ** -e[:, :, None, None].astype(np.float64), fmt), (e + 127).astype(np.uint8)


def dequantize(codes, scales, rows, cols, fmt):
    v = code_values(fmt)[codes] * 2.0 ** (scales.astype(np.float64) - 127)[:, :, None, None]
    R, C = scales.shape
    return v.transpose(0, 2, 1, 3).reshape(R * BLK, C * BLK)[:rows, :cols]


def round_rows(x, fmt):
    """Values of x with each row's pieces of 128 columns rounded to 8 bits."""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    for j in range(0, x.shape[1], BLK):
        p = x[:, j:j + BLK]
        s = 2.0 ** exponent(finite_max(p, 1), fmt).astype(np.float64)[:, None]
        out[:, j:j + BLK] = code_values(fmt)[encode(p / s, fmt)] * s
    return out


def linear(x, codes, scales, m, n, wfmt, xfmt):
    """(y, sum |x_j w_ij|) of the 8-bit linear."""
    W, q = dequantize(codes, scales, m, n, wfmt), round_rows(x, xfmt)
    return q @ W.T, np.abs(q) @ np.abs(W).T


def log_softmax(x, scale=1.0):
    """Row-wise; -inf everywhere for a row of -inf, NaN for NaN or +inf."""
    z = np.asarray(x, np.float64) * scale
    with np.errstate(all="ignore"):
        m = z.max(1, keepdims=True)
        d = np.where(np.isneginf(m), 0.0, z - m)
        lse = np.log(np.exp(d).sum(1, keepdims=True))
        return np.where(np.isneginf(m), -np.inf, d - lse)


def lse(x, scale=1.0):
    z = np.asarray(x, np.float64) * scale
    with np.errstate(all="ignore"):
        m = z.max(1, keepdims=True)
        out = m + np.log(np.exp(np.where(np.isneginf(m), -np.inf, z - m)).sum(1, keepdims=True))
        return np.where(np.isneginf(m), -np.inf, out)[:, 0]


def xlogx(p, lp):
    return np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, lp))


def token_logprobs(x, targets, scale=1.0):
    """(logprob, entropy) in fp64."""
    lp = log_softmax(x, scale)
    H = -xlogx(np.exp(lp), lp).sum(1)
    y = np.asarray(targets)
    V = lp.shape[1]
    got = lp[np.arange(len(y)), np.clip(y, 0, V - 1)]
    return np.where(y < 0, 0.0, np.where(y >= V, np.nan, got)), H


def top(x, k):
    """Indices of the k largest (equal ones by index, NaN first), -1 beyond V."""
    x = np.asarray(x, np.float64)
    out = np.full((x.shape[0], k), -1, np.int64)
    for r, row in enumerate(x):
        key = np.where(np.isnan(row), np.inf, row)
        order = sorted(range(len(row)), key=lambda i: (not np.isnan(row[i]), -key[i], i))[:k]
        out[r, :len(order)] = order
    return out


def token_logprobs_backward(x, targets, g_logprob, g_entropy, scale=1.0):
    """Gradient of sum g_logprob logprob + g_entropy entropy."""
    lp = log_softmax(x, scale)
    p = np.exp(lp)
    H = -xlogx(p, lp).sum(1, keepdims=True)
    y = np.asarray(targets)
    gl = np.where(y < 0, 0.0, g_logprob)
    onehot = np.arange(p.shape[1]) == y[:, None]
    plogp = xlogx(p, lp)
    d = scale * (gl[:, None] * (onehot - p) - np.asarray(g_entropy)[:, None] * (plogp + p * H))
    d[(y >= p.shape[1]) & (np.asarray(g_logprob) != 0)] = np.nan
    d[np.isneginf(np.asarray(x)).all(1)] = 0.0
    d[(gl == 0) & (np.asarray(g_entropy) == 0)] = 0.0
    return d


def distill_kl(student, teacher, scale=1.0):
    """Row-wise sum p (log p - log q), p the teacher's."""
    lq, lp = log_softmax(student, scale), log_softmax(teacher, scale)
    p = np.exp(lp)
    with np.errstate(all="ignore"):
        return np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, lp - lq)).sum(1)


def distill_kl_backward(student, teacher, weight, scale=1.0):
    q, p = np.exp(log_softmax(student, scale)), np.exp(log_softmax(teacher, scale))
    d = np.asarray(weight)[:, None] * scale * (q - p)
    none = np.isneginf(np.asarray(student)).all(1) | np.isneginf(np.asarray(teacher)).all(1)
    d[none | (np.asarray(weight) == 0)] = 0.0
    return d
