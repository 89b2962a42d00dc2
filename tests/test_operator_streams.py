"""Which tensors the operators' Python calls mark as used on which stream, with a stand-in for torch's device calls."""
import contextlib
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

from paper_2108_09413_b200 import operators  # noqa: E402


class Tensor:
    def __init__(self, elements=4):
        self.elements, self.streams = elements, []

    def numel(self):
        return self.elements

    def record_stream(self, stream):
        self.streams.append(stream)


def stand_in(monkeypatch, streams, current=0):
    """A machine whose device i has the current stream streams[i]; device `current` is the current one."""
    state = dict(device=current, streams=dict(enumerate(streams)))

    @contextlib.contextmanager
    def device(index):
        before, state["device"] = state["device"], index
        yield
        state["device"] = before

    @contextlib.contextmanager
    def use(stream):
        before, state["streams"][stream.device_index] = state["streams"][stream.device_index], stream
        yield
        state["streams"][stream.device_index] = before
    cuda = SimpleNamespace(current_device=lambda: state["device"], current_stream=lambda i: state["streams"][i], device=device, stream=use)
    monkeypatch.setattr(operators, "_torch", SimpleNamespace(cuda=cuda, _C=SimpleNamespace(_cuda_getCurrentRawStream=lambda i: state["streams"][i].cuda_stream)))


def stream(raw, device=0):
    return SimpleNamespace(cuda_stream=raw, device_index=device)


def run(given, device=0):
    tensors, raws = [Tensor(), None, Tensor(0), Tensor()], []
    operators._enqueue("isc_log_probs", SimpleNamespace(index=device), given, lambda raw: raws.append(raw) or 0, tensors)
    assert len(raws) == 1 and tensors[2].streams == [] and tensors[0].streams == tensors[3].streams
    return raws[0], tensors[0].streams


def test_on_the_default_stream(monkeypatch):
    stand_in(monkeypatch, [stream(0)])
    assert run(None) == (0, [])


def test_on_a_current_side_stream(monkeypatch):
    side = stream(0x70)
    stand_in(monkeypatch, [side])
    assert run(None) == (0x70, [side])


def test_on_a_stream_that_was_given(monkeypatch):
    side, default = stream(0x70), stream(0)
    stand_in(monkeypatch, [default])
    assert run(side) == (0x70, [side])
    stand_in(monkeypatch, [side])
    assert run(default) == (0, [default])


@pytest.mark.parametrize("raw", [0, 0x71])
def test_on_another_device_s_current_stream(monkeypatch, raw):
    theirs = stream(raw, 1)
    stand_in(monkeypatch, [stream(0x70), theirs])
    assert run(None, 1) == (raw, [theirs] if raw else [])
