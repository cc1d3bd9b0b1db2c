"""Cases and plain forms of the output head's operators: the linear with 8-bit
block-scaled weights (decode, prefill and input gradient), its quantisation,
the log probabilities of given tokens with entropy and top alternatives, and
the KL divergence to a teacher, the last two with their gradients (the KL's for
tokens' weights that are known before).

Block-scaled 8-bit matrix: blocks of 128 x 128, each with a power-of-two scale
2^e, e the smallest integer with amax <= MAX * 2^e (MAX is 448 for e4m3 and
57344 for e5m2; e = 0 for a block of zeros, kept within -127..127), and codes
of x * 2^-e rounded to nearest even.  Storage: tiles of 128 x 128 codes (row
major within a tile, tiles row major, zeros outside the matrix), and one byte
e + 127 for each tile.  Activations get one scale for each row and 128 columns.

listed() gives the fixed cases, draw(rng) one more of the same ranges.
"""
import math

import torch

own = False
DEV = "cuda"
FMT = {"e4m3": (448.0, torch.float8_e4m3fn), "e5m2": (57344.0, torch.float8_e5m2)}
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
# 2^e at e + 127, exact (a power computed on the GPU need not be)
POWERS = [math.ldexp(1.0, e) for e in range(-127, 128)]


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def listed():
    return [
        # one k or v projection of an 8B decoder layer kept in 8 bits, one
        # token: the smallest call, launch and memory latency
        dict(name="linear_kv_b1", kind="linear", T=1, m=1024, n=4096, wfmt="e4m3", xfmt="e4m3",
             y="bf16"),
        # the output head of an 8B-shaped model, one token being decoded
        dict(name="head_b1", kind="linear", T=1, m=128256, n=4096, wfmt="e4m3", xfmt="e4m3",
             y="bf16"),
        # the same head for a batch of twelve sequences, logits in fp32
        dict(name="head_b12", kind="linear", T=12, m=128256, n=4096, wfmt="e4m3", xfmt="e4m3",
             y="f32"),
        # a chunk of a chunked prefill through a 70B attention projection
        dict(name="linear_8192_T500", kind="linear", T=500, m=8192, n=8192, wfmt="e4m3",
             xfmt="e4m3", y="bf16"),
        # a whole training sequence through the head: the largest case
        dict(name="head_T2048", kind="linear", T=2048, m=128256, n=4096, wfmt="e4m3", xfmt="e4m3",
             y="bf16"),
        # and the gradient of its input: a contraction over an odd vocabulary
        dict(name="head_grad_T1000", kind="grad", T=1000, m=50257, n=4096, wfmt="e4m3",
             xfmt="e5m2", y="bf16"),
        # a 70B attention linear quantised and read back
        dict(name="quantise_8192", kind="quantise", m=8192, n=8192, wfmt="e4m3", src="bf16"),
        # one decoded token's log probability and the twenty best alternatives
        dict(name="logprobs_b1_top20", kind="logprobs", T=1, V=128256, dtype="f32", k=20,
             scale=1.0),
        # the scoring of a prompt: an odd vocabulary, five alternatives
        dict(name="logprobs_T1500_top5", kind="logprobs", T=1500, V=50257, dtype="bf16", k=5,
             scale=1.0),
        # a policy's training step: log probabilities and entropies at a
        # sampling temperature, and their gradient
        dict(name="logprobs_train_T2048", kind="logprobs_train", T=2048, V=32000, dtype="bf16",
             scale=1.25),
        # scale-only reconstruction of a short odd sequence, logits in fp32
        dict(name="kl_train_T45", kind="kl_train", T=45, V=50257, dtype="f32", scale=1.0),
        # and of a whole training sequence of an 8B-shaped model
        dict(name="kl_train_T2048", kind="kl_train", T=2048, V=128256, dtype="bf16", scale=0.5),
    ]


def _int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "grad", "quantise", "logprobs", "logprobs",
                       "logprobs_train", "kl_train", "kl_train"])
    if kind in ("linear", "grad", "quantise"):
        m, n = _int(rng, 256, 131072), _int(rng, 256, 16384)
        if rng.random() < 0.5:
            m, n = 32 * max(8, m // 32), 128 * max(2, n // 128)
        if kind == "quantise":
            return dict(kind=kind, m=min(m, 32768), n=min(n, 8192),
                        wfmt=rng.choice(["e4m3", "e4m3", "e5m2"]), src=rng.choice(list(DTYPE)))
        T = _int(rng, 1, 2048)
        T = max(1, min(T, 2048 * 128256 * 4096 // (m * n)))
        return dict(kind=kind, T=T, m=m, n=n, wfmt=rng.choice(["e4m3", "e4m3", "e5m2"]),
                    xfmt="e5m2" if kind == "grad" else "e4m3", y=rng.choice(["bf16", "f32"]))
    V, dtype = _int(rng, 1000, 160000), rng.choice(list(DTYPE))
    T = max(1, min(_int(rng, 1, 2048), 2048 * 128256 * 2 // (V * SIZE[dtype])))
    case = dict(kind=kind, T=T, V=V, dtype=dtype, scale=rng.choice([1.0, 1.0, 0.5, 1.25]))
    if kind == "logprobs":
        case["k"] = rng.choice([0, 1, 5, 20])
    return case


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def weight(g, m, n):
    """A trained linear's weight: rows of unequal norm, some input channels small."""
    w = torch.randn((m, n), generator=g, device=DEV) * n ** -0.5
    w *= torch.exp(0.5 * torch.randn((m, 1), generator=g, device=DEV))
    w *= torch.exp(0.5 * torch.randn((1, n), generator=g, device=DEV))
    return w


def activations(g, T, n):
    """N(0, 1), one percent of the channels 20 times larger, in bf16."""
    x = torch.randn((T, n), generator=g, device=DEV)
    x[:, torch.randperm(n, generator=g, device=DEV)[:max(1, n // 100)]] *= 20.0
    return x.to(torch.bfloat16)


def logits(g, T, V, dtype):
    """A model's logits: a bulk of width 2 below a few large ones, whose size
    (and so the entropy) differs from token to token."""
    z = torch.randn((T, V), generator=g, device=DEV) * 2.0 - 2.0
    top = torch.randint(0, V, (T, 32), generator=g, device=DEV)
    height = 4.0 + 12.0 * torch.rand((T, 1), generator=g, device=DEV)
    # the largest where a place is drawn twice
    z.scatter_reduce_(1, top, height - torch.rand((T, 32), generator=g, device=DEV) * 8.0, "amax")
    return z.to(DTYPE[dtype]), top


def blocks_up(n):
    return -(-n // 128)


def tiled(a):
    """A matrix in tiles of 128 x 128, [rows/128, cols/128, 128, 128], zeros outside."""
    R, C = blocks_up(a.shape[0]), blocks_up(a.shape[1])
    a = torch.nn.functional.pad(a, (0, 128 * C - a.shape[1], 0, 128 * R - a.shape[0]))
    return a.view(R, 128, C, 128).transpose(1, 2).contiguous()


def exponent(amax, fmt):
    """Smallest e with amax <= MAX * 2^e: MAX is 0.875 of a power of two."""
    f, x = torch.frexp(amax)
    e = x - (9 if fmt == "e4m3" else 16) + (f > 0.875)
    return torch.where(amax > 0, e, 0).clamp(-127, 127).to(torch.int32)


def power(e):
    """2^e in fp32, for e in -127..127."""
    return torch.tensor(POWERS, dtype=torch.float32, device=DEV)[(e + 127).long()]


def stored(w, fmt):
    """Codes and scales of a matrix in the storage above."""
    t = tiled(w)
    e = exponent(t.abs().amax((2, 3)), fmt)
    codes = (t * power(-e)[:, :, None, None]).to(FMT[fmt][1]).view(torch.uint8)
    return codes, (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    k = case["kind"]
    s = dict(case)
    if k in ("linear", "grad"):
        T, m, n = case["T"], case["m"], case["n"]
        w = weight(g, m, n)
        # frozen weights: quantised once, and transposed once for the gradient
        s["codes"], s["scales"] = stored(w if k == "linear" else w.T, case["wfmt"])
        if k == "linear":
            s["x"] = activations(g, T, n)
        else:
            # the gradient of a cross entropy: a softmax less the given token
            p = torch.softmax(logits(g, T, m, "f32")[0], 1)
            p[torch.arange(T, device=DEV), torch.randint(0, m, (T,), generator=g, device=DEV)] -= 1
            s["x"] = (p / T).to(torch.bfloat16)
        if own:
            # the handle (pointers to the codes and scales above) and buffers
            # that a program keeps for a layer
            from paper_2609_06161_amd.output import Fp8Linear, Fp8Matrix
            rows, cols = (m, n) if k == "linear" else (n, m)
            s["layer"] = Fp8Linear(Fp8Matrix(rows, cols, case["wfmt"], s["codes"], s["scales"]))
            s["out"] = torch.empty((T, rows), dtype=DTYPE[case["y"]], device=DEV)
            s["ws"] = s["layer"].workspace(T)
    elif k == "quantise":
        s["w"] = weight(g, case["m"], case["n"]).to(DTYPE[case["src"]])
    else:
        T, V = case["T"], case["V"]
        s["logits"], top = logits(g, T, V, case["dtype"])
        # the mean over the tokens; scaled up where fp16 would lose the gradient
        mean = (16384.0 if case["dtype"] == "f16" else 1.0) / T
        if k == "kl_train":
            # a teacher close to the student, as a calibrated model's is
            noise = torch.randn((T, V), generator=g, device=DEV) * 0.5
            s["teacher"] = (s["logits"].float() + noise).to(DTYPE[case["dtype"]])
            s["weight"] = torch.full((T,), mean, device=DEV)
        else:
            # the given token is mostly one of the likely ones
            rare = torch.randint(0, V, (T,), generator=g, device=DEV)
            likely = torch.rand((T,), generator=g, device=DEV) < 0.8
            s["targets"] = torch.where(likely, top[:, 0], rare)
        if k == "logprobs_train":
            s["g_logprob"] = torch.randn((T,), generator=g, device=DEV) * mean
            s["g_entropy"] = torch.full((T,), 0.01 * mean, device=DEV)
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(s):
    if own:
        return run_own(s)
    return {"linear": plain_linear, "grad": plain_linear, "quantise": plain_quantise,
            "logprobs": plain_logprobs, "logprobs_train": plain_logprobs_train,
            "kl_train": plain_kl_train}[s["kind"]](s)


def run_own(s):
    from paper_2609_06161_amd import output as O
    k = s["kind"]
    if k in ("linear", "grad"):
        return s["layer"].forward(s["x"], s["out"], s["ws"], fmt=s["xfmt"])
    if k == "quantise":
        return O.Fp8Matrix.quantize(s["w"], s["wfmt"]).dequantize(torch.bfloat16)
    if k == "kl_train":
        kl, ds = O.distill_kl(s["logits"], s["teacher"], s["scale"], s["weight"])
        return dict(kl=kl, dlogits=ds)
    if k == "logprobs":
        st = O.token_logprobs(s["logits"], s["targets"], s["k"], s["scale"])
        out = dict(logprob=st.logprob, entropy=st.entropy)
        return dict(out, top_logprob=st.top_logprob, top_index=st.top_index) if s["k"] else out
    st = O.token_logprobs(s["logits"], s["targets"], 0, s["scale"])
    dz = O.token_logprobs_backward(s["logits"], s["targets"], st, s["g_logprob"], s["g_entropy"],
                                   s["scale"])
    return dict(logprob=st.logprob, entropy=st.entropy, dlogits=dz)


# the plain forms, in fp32

def values(s, rows, cols):
    """The matrix that codes and scales stand for, in fp32."""
    v = s["codes"].view(FMT[s["wfmt"]][1]).float()
    v = v * power(s["scales"].to(torch.int32) - 127)[:, :, None, None]
    R, C = v.shape[:2]
    return v.transpose(1, 2).reshape(128 * R, 128 * C)[:rows, :cols]


def rounded_rows(x, fmt):
    """x with each row's 128-column pieces rounded to 8 bits at their scale."""
    T, n = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -n % 128)).view(T, -1, 128)
    e = exponent(b.abs().amax(2, keepdim=True), fmt)
    q = (b * power(-e)).to(FMT[fmt][1]).float() * power(e)
    return q.view(T, -1)[:, :n]


def plain_linear(s):
    rows, cols = (s["m"], s["n"]) if s["kind"] == "linear" else (s["n"], s["m"])
    y = rounded_rows(s["x"], s["xfmt"]) @ values(s, rows, cols).T
    return y.to(DTYPE[s["y"]])


def plain_quantise(s):
    t = tiled(s["w"].float())
    e = exponent(t.abs().amax((2, 3)), s["wfmt"])[:, :, None, None]
    v = (t * power(-e)).to(FMT[s["wfmt"]][1]).float() * power(e)
    R, C = v.shape[:2]
    v = v.transpose(1, 2).reshape(128 * R, 128 * C)[:s["m"], :s["n"]]
    return v.to(torch.bfloat16)


def log_softmax(x, scale, dtype=torch.float32):
    z = x.to(dtype) * scale
    z = z - z.amax(1, keepdim=True)
    return z - z.exp().sum(1, keepdim=True).log()


def plain_logprobs(s):
    lp = log_softmax(s["logits"], s["scale"])
    out = dict(logprob=lp.gather(1, s["targets"][:, None])[:, 0],
               entropy=-(lp.exp() * lp).sum(1))
    if s["k"]:
        # stable: equal logits keep the order of their indices
        index = torch.sort(s["logits"], dim=1, descending=True, stable=True)[1][:, :s["k"]]
        out["top_logprob"], out["top_index"] = lp.gather(1, index), index
    return out


def plain_logprobs_train(s):
    lp = log_softmax(s["logits"], s["scale"])
    p = lp.exp()
    H = -(p * lp).sum(1, keepdim=True)
    onehot = torch.arange(s["V"], device=DEV) == s["targets"][:, None]
    dz = s["g_logprob"][:, None] * (onehot.float() - p) - s["g_entropy"][:, None] * p * (lp + H)
    return dict(logprob=lp.gather(1, s["targets"][:, None])[:, 0], entropy=H[:, 0],
                dlogits=(dz * s["scale"]).to(DTYPE[s["dtype"]]))


def plain_kl_train(s):
    # in 64 bits: a small divergence is a small difference of large logarithms
    ls = log_softmax(s["logits"], s["scale"], torch.float64)
    lt = log_softmax(s["teacher"], s["scale"], torch.float64)
    kl = (lt.exp() * (lt - ls)).sum(1)
    ds = (s["weight"] * s["scale"])[:, None] * (ls.exp() - lt.exp())
    return dict(kl=kl.float(), dlogits=ds.to(DTYPE[s["dtype"]]))


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    k = case["kind"]
    if k in ("linear", "grad"):
        T, m, n = case["T"], case["m"], case["n"]
        rows, cols = (m, n) if k == "linear" else (n, m)
        return dict(bytes=m * n + blocks_up(m) * blocks_up(n) + 2 * T * cols
                    + T * rows * SIZE[case["y"]], flops=2 * T * m * n)
    if k == "quantise":
        # the matrix read, its codes and scales written, its values written
        m, n = case["m"], case["n"]
        return dict(bytes=m * n * (SIZE[case["src"]] + 1 + 2) + blocks_up(m) * blocks_up(n),
                    flops=3 * m * n)
    T, V, size = case["T"], case["V"], SIZE[case["dtype"]]
    if k == "logprobs":
        # logits and tokens read; log probability, entropy, alternatives written
        return dict(bytes=T * V * size + T * (8 + 8 + 12 * case["k"]), flops=6 * T * V)
    if k == "logprobs_train":
        return dict(bytes=2 * T * V * size + T * (8 + 8 + 8), flops=13 * T * V)
    return dict(bytes=3 * T * V * size + T * 8, flops=16 * T * V)


# --------------------------------------------------------------------------
# results in 64 bits
# --------------------------------------------------------------------------

def grid64(v, amax, fmt):
    """v (float64) rounded to the 8-bit grid that amax sets, from the format's
    definition: the scale by search among the powers of two, the step by the
    value's own binade (at least the smallest normal one), ties to even."""
    top, mantissa, lowest = (448.0, 3, -6) if fmt == "e4m3" else (57344.0, 2, -14)
    powers = torch.tensor(POWERS, dtype=torch.float64, device=v.device)
    scale = powers[torch.searchsorted(top * powers, amax).clamp(max=254)]
    scale = torch.where(amax > 0, scale, 1.0)
    u = v / scale
    binade = (torch.frexp(u)[1] - 1).clamp(min=lowest) - mantissa
    step = powers[(binade + 127).long()]
    return torch.round(u / step) * step * scale


def matrix64(w, fmt):
    """A matrix as it is stored, in float64, a band of 128 rows times its blocks at a time."""
    m, n = w.shape
    out = torch.empty((m, n), dtype=torch.float64, device=DEV)
    for i in range(0, m, 4096):
        band = w[i:i + 4096].double()
        r = band.shape[0]
        t = torch.nn.functional.pad(band, (0, -n % 128, 0, -r % 128))
        t = t.view(t.shape[0] // 128, 128, -1, 128)
        q = grid64(t, t.abs().amax((1, 3), keepdim=True), fmt)
        out[i:i + 4096] = q.reshape(-1, q.shape[2] * 128)[:r, :n]
    return out


def rows64(x, fmt):
    T, n = x.shape
    b = torch.nn.functional.pad(x.double(), (0, -n % 128)).view(T, -1, 128)
    return grid64(b, b.abs().amax(2, keepdim=True), fmt).view(T, -1)[:, :n]


def log_probabilities64(logits, scale):
    z = logits.double() * scale
    return z - torch.logsumexp(z, 1, keepdim=True)


def exact(case, seed):
    k = case["kind"]
    s = prepare(case, seed)
    if k in ("linear", "grad", "quantise"):
        g = torch.Generator(device=DEV).manual_seed(seed)
        w = weight(g, case["m"], case["n"])
        if k == "quantise":
            return matrix64(w.to(DTYPE[case["src"]]), case["wfmt"])
        W = matrix64(w if k == "linear" else w.T, case["wfmt"])
        return rows64(s["x"], case["xfmt"]) @ W.T
    T, scale = case["T"], case["scale"]
    got = []
    # 64 rows at a time: float64 copies of the whole would not fit thrice
    for i in range(0, T, 64):
        rows = slice(i, min(T, i + 64))
        lp = log_probabilities64(s["logits"][rows], scale)
        p = lp.exp()
        if k == "kl_train":
            lt = log_probabilities64(s["teacher"][rows], scale)
            pt = lt.exp()
            got.append(dict(kl=(pt * (lt - lp)).sum(1),
                            dlogits=s["weight"][rows, None].double() * scale * (p - pt)))
            continue
        y = s["targets"][rows, None]
        H = -(p * lp).sum(1)
        one = dict(logprob=lp.gather(1, y)[:, 0], entropy=H)
        if k == "logprobs_train":
            dz = -p * s["g_logprob"][rows, None].double()
            dz.scatter_add_(1, y, s["g_logprob"][rows, None].double())
            dz -= s["g_entropy"][rows, None].double() * p * (lp + H[:, None])
            one["dlogits"] = dz * scale
        elif case["k"]:
            # equal values in the order of their indices
            value, index = torch.sort(lp, dim=1, descending=True, stable=True)
            one["top_logprob"], one["top_index"] = value[:, :case["k"]], index[:, :case["k"]]
        got.append(one)
    return {name: torch.cat([o[name] for o in got]) for name in got[0]}
