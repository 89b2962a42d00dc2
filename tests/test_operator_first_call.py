"""The first call of two threads at once."""
import threading

import pytest

import paper_2108_09413_b200 as isc

torch = pytest.importorskip("torch")


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def test_a_second_thread_finds_the_types(monkeypatch):
    """While the first thread is on its way through the start, the second's call gets as far as it would later: here to the
    weight's length, which it checks after the type."""
    from paper_2108_09413_b200 import operators
    inside, go_on = threading.Event(), threading.Event()

    class Slow(dict):
        def update(self, *what):
            if threading.current_thread() is first:
                inside.set()
                assert go_on.wait(60)
            super().update(*what)
    monkeypatch.setattr(operators, "_torch", None)
    monkeypatch.setattr(operators, "_types", Slow())
    first = threading.Thread(target=operators._start)
    first.start()
    try:
        assert inside.wait(60)
        x = torch.ones(4, 64).bfloat16().as_subclass(OnGpu)
        with pytest.raises(isc.IscError, match="weight"):
            isc.rms_norm_quant(x, torch.ones(63).bfloat16().as_subclass(OnGpu))
    finally:
        go_on.set()
        first.join()
    assert operators._torch is torch and operators._types[torch.bfloat16] == 0
