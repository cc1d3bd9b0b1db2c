"""Temporaries of calls that run on a given stream, which may be an integer
handle: memory that a call drops is not handed to work on another stream while
its kernels still wait to use it."""
import pytest
import torch

from paper_2609_06161_amd import output as O, synth
from paper_2609_06161_amd.layer import DeviceLayer, to_device

from test_gpu_head import DEV, randn

pytestmark = pytest.mark.gpu


def late(call, side):
    """call(handle) behind 10 ms of other work on `side`, while the current
    stream allocates and overwrites whatever memory it can get."""
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = call(side.cuda_stream)
    junk = [torch.full((n,), 255, dtype=torch.uint8, device=DEV)
            for n in (1 << k for k in range(9, 26)) for _ in range(3)]
    torch.cuda.synchronize()
    del junk
    return got


@pytest.mark.parametrize("T", [9, 45, 300])
def test_linear_on_an_integer_stream(T):
    n = 5000
    layer = O.Fp8Linear.from_dense(randn(1, 2000, n).to(DEV))
    x, dy = randn(2, T, n).to(DEV), randn(3, T, 2000).to(DEV)
    want = layer.forward(x), layer.input_grad(dy)
    side = torch.cuda.Stream()
    got = late(lambda s: (layer.forward(x, stream=s), layer.input_grad(dy, stream=s)), side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_losses_on_an_integer_stream():
    z, t = randn(4, 9, 40000).to(DEV), randn(5, 9, 40000).to(DEV)
    y = torch.arange(9, device=DEV)

    def calls(s):
        p = O.token_logprobs(z, y, 5, stream=s)
        kl, d = O.distill_kl(z, t, stream=s)
        return [*p, O.token_logprobs_backward(z, y, p, p.lse, stream=s), kl, d]

    want = calls(None)
    for a, b in zip(late(calls, torch.cuda.Stream()), want):
        assert torch.equal(a, b)


def test_reconstruction_on_an_integer_stream():
    m, n, r, V, T = 512, 768, 224, 1500, 45
    lin = synth.make_linear(6, m, n, r, T)
    layer = DeviceLayer.from_host(lin)
    head8 = O.Fp8Linear.from_dense((randn(7, V, m) * m ** -0.5).to(DEV))
    x, teacher = to_device(lin.x), randn(8, T, V).to(DEV)

    def step(s):
        kl, dx, grads = O.reconstruction_step(layer, head8, x, teacher, stream=s)
        return [kl, dx, *grads]

    want = step(None)
    for a, b in zip(late(step, torch.cuda.Stream()), want):
        assert torch.equal(a, b)


def test_signs_are_transposed_for_every_stream():
    """The first backward of a layer is captured, a later one runs on a stream
    while another is busy: each has complete transposed signs."""
    lin = synth.make_linear(9, 512, 768, 224, 45)
    x = to_device(lin.x)
    dy = randn(10, 45, 512).to(torch.bfloat16).to(DEV).view(torch.int16)
    known = DeviceLayer.from_host(lin)
    saved = known.forward_train(x)[1]
    dx, grads = known.backward(x, dy, saved)
    want = [dx, *grads]
    layer = DeviceLayer.from_host(lin)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dx, grads = layer.backward(x, dy, saved)
    held = [dx, *grads]
    side = torch.cuda.Stream()
    dx, grads = late(lambda s: layer.backward(x, dy, saved, stream=s), side)
    for a, b in zip([dx, *grads], want):
        assert torch.equal(a, b)
    dx, grads = layer.backward(x, dy, saved)
    for a, b in zip([dx, *grads], want):
        assert torch.equal(a, b)
    for _ in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)
