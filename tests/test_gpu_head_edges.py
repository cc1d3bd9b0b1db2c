"""The losses' gradients and values at their documented edges."""
import pytest
import torch

from paper_2609_06161_amd import output as O, synth
from paper_2609_06161_amd.layer import DeviceLayer, to_device

from test_gpu_head import DEV, DTYPES, check_logprobs_grad, logits, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V", [(6, 3001), (2100, 259)])
def test_logprobs_gradient_of_targets_beyond_the_vocabulary(T, V, dtype):
    """NaN in the whole row, where entries have probability 0 as well; nothing
    where the target's factor is zero."""
    z = logits(1, T, V, dtype)
    z[:3, 3:] = -float("inf")          # masked
    z[3, 5] = 30000.0                  # one logit beside which all are 0
    y = torch.full((T,), 2)
    y[[0, 1, 3, 4]] = torch.tensor([V, V + 7, V, 1 << 40])
    gl, gh = torch.ones(T), torch.ones(T)
    gl[1] = 0.0
    z, y, gl, gh = (a.to(DEV) for a in (z, y, gl, gh))
    d = check_logprobs_grad(z, y, gl, gh, 1.0)
    assert torch.isnan(d[[0, 3, 4]]).all() and torch.isfinite(d[[1, 2, 5]]).all()
    d = check_logprobs_grad(z, y, gl, None, 1.0)
    assert torch.isnan(d[[0, 3, 4]]).all() and (d[1] == 0).all()
    assert torch.isfinite(check_logprobs_grad(z, y, None, gh, 1.0)).all()


@pytest.mark.parametrize("T", [4, 2100])
def test_logprobs_gradient_of_nan_factors(T):
    z = logits(2, T, 1003, torch.float32)
    z[:, 3:] = -float("inf")
    z[3] = -float("inf")
    gl, gh = torch.ones(T), torch.ones(T)
    gl[0] = gh[1] = gl[3] = float("nan")
    y = torch.zeros(T, dtype=torch.int64)
    d = check_logprobs_grad(z.to(DEV), y.to(DEV), gl.to(DEV), gh.to(DEV), 1.0)
    assert torch.isnan(d[:2]).all() and torch.isfinite(d[2:]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_reconstruction_step_of_padded_tokens(dtype, bad):
    """A padding token's teacher row may hold anything: the loss and all the
    gradients are those of a step where it holds zeros."""
    m, n, r, V, T = 512, 768, 224, 1500, 5
    lin = synth.make_linear(3, m, n, r, T)
    layer = DeviceLayer.from_host(lin)
    head8 = O.Fp8Linear.from_dense((randn(4, V, m) * m ** -0.5).to(DEV))
    teacher = logits(5, T, V, dtype).to(DEV)
    weight = torch.tensor([0.25, 0.0, 0.25, 0.0, 0.25], device=DEV)

    def step(row):
        teacher[3] = row
        kl, dx, grads = O.reconstruction_step(layer, head8, to_device(lin.x), teacher, weight)
        return (weight * kl).sum(), kl, dx, *grads

    want, got = step(0.0), step(bad)
    assert torch.isfinite(want[0]) and torch.isfinite(want[1]).all() and (want[1] > 0).all()
    assert got[1][3] == 0 and torch.equal(got[1][[0, 1, 2, 4]], want[1][[0, 1, 2, 4]])
    for a, b in zip((got[0], *got[2:]), (want[0], *want[2:])):
        assert torch.equal(a, b)
