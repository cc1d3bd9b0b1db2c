"""Rows that are several workgroups' work: what each part gives has to arrive.

One part of a row carries most of a sum, so that losing it, or taking another's
in its place, changes the result by a tenth and more.  Tolerances count the
roundings on a path of additions: D of them, a thread's terms (eight a chunk),
the wave's and the block's trees and the parts in order, beside 60 for a term's
own; a sum of terms of one sign is within D u of itself, u = 2^-24."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_06161_amd import af1, build_lib, head, output as O

from test_gpu_head import DEV, U

pytestmark = pytest.mark.gpu


def log_softmax64(x, scale=1.0):
    return torch.log_softmax(x.double() * scale, 1)


def kl64(s, t):
    ls, lt = log_softmax64(s), log_softmax64(t)
    return (lt.exp() * (lt - ls)).sum(1), ls.exp() - lt.exp()


def close(got, want, rtol):
    err = (got.double() - want).abs() / want.abs()
    assert err.max() <= rtol, f"{err.max():.3g} of the value"


@pytest.mark.parametrize("T,dtype", [(1, torch.float32), (2, torch.bfloat16)])
def test_kl_of_rows_beyond_what_runs_at_once(T, dtype):
    """The largest vocabulary: a row of 2048 (1024) parts."""
    V = head.AF1_HEAD_MAX_VOCAB
    print(f"kl T={T} V={V} {dtype}", flush=True)
    g = torch.Generator(device=DEV).manual_seed(T)
    s = torch.randn((T, V), generator=g, device=DEV).to(dtype)
    t = (s + 0.5 * torch.randn((T, V), generator=g, device=DEV)).to(dtype)
    t[:, -5000:] += 9.0         # most of the mass in the last parts
    want, dwant = kl64(s, t)
    O.distill_kl(s[:, :100000], t[:, :100000])
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    kl, d = O.distill_kl(s, t)
    end.record()
    torch.cuda.synchronize()
    close(kl, want, 1e-5)
    # a probability is within 2^-18 of itself here, the output within half a step
    half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[dtype]
    p = log_softmax64(t).exp()
    bound = (dwant.abs() + 2.0 ** -17 * (dwant.abs() + 2 * p)) * half + 2.0 ** -17 * (dwant.abs() + 2 * p)
    assert ((d.double() - dwant).abs() <= bound + 2.0 ** -126).all()
    # some ten times what reading the rows twice takes; each part's statistics
    # computed by every workgroup would take seconds
    assert begin.elapsed_time(end) < 20.0
    own = s.clone()
    k2, d2 = O.distill_kl(own, t, dstudent=own)
    assert torch.equal(k2, kl) and torch.equal(d2, d)


@pytest.fixture(scope="module")
def plans():
    """(parts of a KL row, parts of a row of log probabilities)."""
    L = ctypes.CDLL(build_lib.HEAD_TEST_LIB)
    out = (ctypes.c_int32 * 2)()

    def kl(dtype, T, V):
        code = af1.AF1_SRC_F32 if dtype == torch.float32 else af1.AF1_SRC_BF16
        assert L.af1_test_kl_plan(code, ctypes.c_int64(T), ctypes.c_int64(V), out) == 0
        return out[0]

    def logprobs(T, V):
        assert L.af1_test_logprobs_plan(ctypes.c_int64(T), ctypes.c_int64(V), out) == 0
        return out[0]
    return kl, logprobs


def piece(V, parts, p):
    """The logits of part p: parts are whole turns of 256 threads by eight."""
    chunks = -(-V // 8)
    size = -(-(-(-chunks // parts)) // 256) * 2048
    assert -(-V // size) == parts
    return slice(p * size, min((p + 1) * size, V)), size // 2048


@pytest.mark.parametrize("T,V,dtype,parts", [(2, 140001, torch.float32, 69),
                                             (2, 300001, torch.bfloat16, 74),
                                             (4, 600007, torch.float32, 74),
                                             (3, 20011, torch.float32, 10)])
def test_every_part_of_a_kl_row(plans, T, V, dtype, parts):
    """The loss is a sum over the parts, the statistics join theirs.  With most
    of both masses in one part, D (2 + |u|) u sum p |u| and its like stay under
    1e-4 of the loss (D = 60 + 64 + 16 + 70, |u| < 1, the loss 0.06 and more)."""
    assert plans[0](dtype, T, V) == parts
    g = torch.Generator(device=DEV).manual_seed(parts)
    base, noise = (torch.randn((T, V), generator=g, device=DEV) for _ in range(2))
    for p in sorted({0, 1, 31, 62, 63, 64, 65, parts - 2, parts - 1} & set(range(parts))):
        print(f"kl T={T} V={V} {dtype} part {p} of {parts}", flush=True)
        at, _ = piece(V, parts, p)
        share = (at.stop - at.start) / V
        s, t = base.clone(), base + 0.1 * noise
        # odds 6 and 2 of the part against the rest
        t[:, at] += np.log(6 * (1 - share) / share)
        s[:, at] += np.log(2 * (1 - share) / share)
        s, t = s.to(dtype), t.to(dtype)
        want, dwant = kl64(s, t)
        kl, d = O.distill_kl(s, t)
        assert (want > 0.06).all()
        close(kl, want, 1e-4)
        half = {torch.float32: U, torch.bfloat16: 2.0 ** -8}[dtype]
        q = 2.0 ** -14 * (log_softmax64(s).exp() + log_softmax64(t).exp())
        assert ((d.double() - dwant).abs() <= half * (dwant.abs() + q) + q).all()
        assert torch.equal(O.distill_kl(s, t, grad=False)[0], kl)


@pytest.mark.parametrize("T,V,dtype,parts", [(1, 128256, torch.float32, 63),
                                             (3, 131072, torch.bfloat16, 64),
                                             (20, 128256, torch.float32, 32),
                                             (400, 50257, torch.float16, 3),
                                             (2, 5003, torch.float32, 3)])
def test_every_part_of_a_row_of_log_probabilities(plans, T, V, dtype, parts):
    """lse and log probabilities within D u (2 + |value|), entropies within
    D u (4 + 2 ln V): ln Z and sum p |t| are at most ln V."""
    assert plans[1](T, V) == parts
    g = torch.Generator(device=DEV).manual_seed(V)
    base = torch.randn((T, V), generator=g, device=DEV)
    for p in sorted({0, 1, parts // 2, parts - 2, parts - 1} & set(range(parts))):
        print(f"logprobs T={T} V={V} {dtype} part {p} of {parts}", flush=True)
        at, chunks = piece(V, parts, p)
        D = 60 + 8 * chunks + 16 + parts
        z = base.clone()
        z[:, at] += np.log(6 * (V - at.stop + at.start) / (at.stop - at.start))
        z = z.to(dtype)
        y = torch.randint(0, V, (T,), generator=g, device=DEV)
        y[0] = at.stop - 1
        lp = log_softmax64(z)
        H = -(lp.exp() * lp).sum(1)
        lse = torch.logsumexp(z.double(), 1)
        got = O.token_logprobs(z, y, 9)
        want = lp.gather(1, y[:, None])[:, 0]
        assert ((got.logprob - want).abs() <= D * U * (2 + want.abs())).all()
        assert ((got.lse - lse).abs() <= D * U * (2 + lse.abs())).all()
        limit = D * U * (4 + 2 * np.log(V))
        assert limit < 2e-3 and ((got.entropy - H).abs() <= limit).all()
        top = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :9]
        assert torch.equal(got.top_index, top)


def test_kl_of_long_rows_captured_and_on_two_streams():
    """Statistics in front of the rows: replayed on new logits with eager calls
    between, and two such calls at once."""
    T, V = 2, 4_300_003
    s, t = (torch.empty((T, V), device=DEV) for _ in range(2))
    g = torch.Generator(device=DEV).manual_seed(3)

    def fresh():
        s.normal_(generator=g)
        t.copy_(s).add_(torch.randn((T, V), generator=g, device=DEV), alpha=0.3)

    fresh()
    O.distill_kl(s, t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = O.distill_kl(s, t)
    for _ in range(3):
        fresh()
        want = O.distill_kl(s, t)
        close(want[0], kl64(s, t)[0], 1e-4)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for side in streams:
        with torch.cuda.stream(side):
            got.append(O.distill_kl(s, t))
    torch.cuda.synchronize()
    for kl, d in got:
        assert torch.equal(kl, want[0]) and torch.equal(d, want[1])
