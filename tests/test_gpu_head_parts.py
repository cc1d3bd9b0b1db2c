"""Rows that are several workgroups' work: what each part gives has to arrive.

In most tests one part carries most of a sum, so that losing it, or taking
another part's in its place, changes the result by far more than 1e-5 of it;
the sums themselves have at most 1000 additions on any path and terms of one
sign where it matters, so rounding leaves 2000 u = 1.2e-4 of a term at the very
most and in squares about 1e-6."""
import pytest
import torch

from paper_2609_06161_amd import head, output as O

from test_gpu_head import DEV

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
