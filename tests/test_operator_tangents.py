"""Tensors with a tangent are refused: the operators would drop it without a word.  (Host tensors that say they are on a GPU: the refusal
comes before anything reaches one.)"""
import pytest

import paper_2108_09413_b200 as isc

torch = pytest.importorskip("torch")
fwd = torch.autograd.forward_ad


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def on_gpu(*shape, dtype=torch.float32):
    return torch.ones(shape, dtype=dtype).as_subclass(OnGpu)


CALLS = {
    "norm": (isc.rms_norm_quant, dict(x=on_gpu(4, 64), weight=on_gpu(64), residual=on_gpu(4, 64), sum_out=on_gpu(4, 64))),
    "linear": (isc.quant_linear, dict(x=on_gpu(4, 64, dtype=torch.int8), x_scale=on_gpu(4), w=on_gpu(8, 64, dtype=torch.int8), w_scale=on_gpu(8), bias=on_gpu(8), out=on_gpu(4, 8))),
    "log_probs": (isc.log_probs, dict(logits=on_gpu(4, 64))),
}


@pytest.mark.parametrize("name,argument", [(n, a) for n, (_, given) in CALLS.items() for a, t in given.items() if t.is_floating_point()])
@pytest.mark.parametrize("mode", [torch.enable_grad, torch.no_grad])
def test_refused(name, argument, mode):
    call, given = CALLS[name]
    with fwd.dual_level(), mode():
        t = given[argument].as_subclass(torch.Tensor)
        dual = fwd.make_dual(t, torch.ones_like(t)).as_subclass(OnGpu)
        with pytest.raises(isc.IscError, match="no gradients") as e:
            call(**dict(given, **{argument: dual}))
        assert e.value.code == -1


@pytest.mark.parametrize("at", [0, 1, 2])
def test_adapters_are_refused(at):
    call, given = CALLS["linear"]
    with fwd.dual_level():
        parts = [torch.ones(2, 8, 64).bfloat16(), torch.ones(2, 8, 8).bfloat16(), torch.ones(2)]
        parts[at] = fwd.make_dual(parts[at], torch.ones_like(parts[at]))
        parts = tuple(t.as_subclass(OnGpu) for t in parts)
        with pytest.raises(isc.IscError, match="no gradients"):
            call(**given, adapters=parts, adapter_ids=torch.zeros(4, dtype=torch.int32).as_subclass(OnGpu))


def test_a_level_without_tangents_refuses_nothing():
    from paper_2108_09413_b200 import operators
    operators._start()
    with fwd.dual_level():
        for _, given in CALLS.values():
            assert operators._same_device("test", tuple(given.values())) == torch.device("cpu")
