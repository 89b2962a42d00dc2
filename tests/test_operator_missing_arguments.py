"""Arguments that are missing or out of range are refused as such, before anything is allocated.  (Host tensors that say they are
on a GPU: nothing reaches one.)"""
import pytest

import paper_2108_09413_b200 as isc

torch = pytest.importorskip("torch")


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def on_gpu(*shape, dtype=torch.float32):
    return torch.ones(shape, dtype=dtype).as_subclass(OnGpu)


X, W, S4, S8 = on_gpu(4, 64, dtype=torch.int8), on_gpu(8, 64, dtype=torch.int8), on_gpu(4), on_gpu(8)
A, B, F, IDS = on_gpu(2, 8, 64, dtype=torch.float16), on_gpu(2, 8, 8, dtype=torch.float16), on_gpu(2), on_gpu(4, dtype=torch.int32)


@pytest.mark.parametrize("call", [
    lambda: isc.rms_norm_quant(None, on_gpu(64)), lambda: isc.rms_norm_quant(on_gpu(4, 64), None), lambda: isc.rms_norm_quant(on_gpu(4, 64), [1.0] * 64),
    lambda: isc.quant_linear(None, S4, W, S8), lambda: isc.quant_linear(X, None, W, S8), lambda: isc.quant_linear(X, S4, None, S8), lambda: isc.quant_linear(X, S4, W, None),
    lambda: isc.quant_linear(X, 1.0, W, S8), lambda: isc.quant_linear(X, S4, W, S8, adapters=(None, B, F), adapter_ids=IDS),
    lambda: isc.quant_linear(X, S4, W, S8, adapters=(A, None, F), adapter_ids=IDS), lambda: isc.quant_linear(X, S4, W, S8, adapters=(A, B, None), adapter_ids=IDS),
    lambda: isc.quant_linear(X, S4, W, S8, adapters=(A, B), adapter_ids=IDS), lambda: isc.quant_linear(X, S4, W, S8, adapters=(A, B, F, F), adapter_ids=IDS),
    lambda: isc.log_probs(None), lambda: isc.log_probs(on_gpu(4, 64), top=33), lambda: isc.log_probs(on_gpu(4, 64), top=-1), lambda: isc.log_probs(on_gpu(4, 64), top=2**32 + 5)])
def test_refused(call, monkeypatch):
    from paper_2108_09413_b200 import operators
    monkeypatch.setattr(operators, "_enqueue", lambda *a, **k: pytest.fail("went through"))
    with pytest.raises(isc.IscError) as e:
        call()
    assert e.value.code == -1
