"""Which stream the tensor calls allocate on (CPU, torch's stream objects
replaced): memory of a call that runs on a given stream has to come from that
stream's pool, or it is handed to other work while the call still uses it."""
import contextlib
import types

import pytest
import torch

from paper_2609_06161_amd import layer, output, synth


class Device:
    index = 0


@pytest.fixture
def entered(monkeypatch):
    """The streams that are entered, in order."""
    seen = []

    @contextlib.contextmanager
    def stream(s):
        seen.append(s)
        yield
        seen.append("left")

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, device=None: ("external", h, device))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: ("default", device))
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda device=None: types.SimpleNamespace(cuda_stream=77))
    return seen


@pytest.mark.parametrize("handle,want", [(1234, ("external", 1234, Device)),
                                         (0, ("default", Device))])
def test_an_integer_is_a_streams_handle(entered, handle, want):
    with layer.on_stream(handle, Device):
        assert entered == [want]
    assert entered == [want, "left"]


def test_other_streams(entered):
    for current in (None, 77):
        with layer.on_stream(current, Device):
            assert entered == []
    with layer.on_stream("a stream"):
        assert entered == ["a stream"]


@pytest.mark.parametrize("capturing", [False, True])
def test_transposed_signs_are_complete_before_they_are_kept(monkeypatch, capturing):
    done = []

    class Stream:
        def synchronize(self):
            done.append("complete")

    monkeypatch.setattr(layer.af1, "af1_pack_transpose", lambda *a: done.append("moved"))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream())
    lin = synth.make_linear(1, 64, 96, 32, 1)
    L = layer.DeviceLayer.from_host(lin, device="cpu")
    first, second = L.transposed(), L.transposed()
    assert [t.shape for t in first] == [(32, 2), (96, 1)]
    if capturing:       # made in each graph that needs them, kept by none
        assert done == ["moved"] * 4 and first[0] is not second[0]
    else:
        assert done == ["moved"] * 2 + ["complete"] and first is second


def test_reconstruction_enters_its_tensors_device(monkeypatch):
    """The layer's calls launch on the current device and stream."""
    inside = []

    @contextlib.contextmanager
    def on(device, stream):
        inside.append((device, stream))
        yield
        inside.pop()

    def within(value):
        def call(*a, **kw):
            assert inside == [(torch.device("cpu"), 1234)]
            return value
        return call

    class Step:
        m = n = 32
        forward_train = within((torch.zeros(3, 32), None))
        backward = within((None, "grads"))
        forward = input_grad = within(torch.zeros(3, 50))

    monkeypatch.setattr(output, "_on", on)
    monkeypatch.setattr(output, "distill_kl", within(("kl", None)))
    got = output.reconstruction_step(Step(), Step(), torch.zeros(3, 32), torch.zeros(3, 50),
                                     stream=1234)
    assert got == ("kl", None, "grads") and not inside
