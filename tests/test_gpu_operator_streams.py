"""Calls under a current stream that is not the inputs': what they were given may go out of use right after them."""
import pytest

import paper_2108_09413_b200 as isc

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_inputs_may_be_dropped_after_calls_on_a_current_side_stream():
    g = torch.Generator(device="cuda").manual_seed(7)
    x, w = torch.randn(512, 1024, device="cuda", generator=g), torch.rand(1024, device="cuda", generator=g)
    matrix = torch.randint(-127, 128, (2048, 1024), device="cuda", generator=g).to(torch.int8)
    factors = torch.rand(2048, device="cuda", generator=g) / 1e4
    q, scale, _ = isc.rms_norm_quant(x, w)
    y = isc.quant_linear(q, scale, matrix, factors)
    p = isc.log_probs(y, top=2)
    side = torch.cuda.Stream()

    def behind(call, inputs):
        for cycles in (1, 100_000_000):                  # the first time loads every kernel and leaves memory for the results
            copies = [t.clone() for t in inputs]
            sizes = [(t.shape, t.dtype) for t in copies]
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                torch.cuda._sleep(cycles)                # some fifty milliseconds ahead of the call
                result = call(*copies)
            del copies
            others = [torch.zeros(shape, dtype=dtype, device="cuda") for shape, dtype in sizes for _ in range(10)]
            torch.cuda.synchronize()
            del others
        return result

    got_q, got_scale, _ = behind(isc.rms_norm_quant, (x, w))
    assert torch.equal(got_q, q) and torch.equal(got_scale, scale)
    assert torch.equal(behind(isc.quant_linear, (q, scale, matrix, factors)), y)
    for got, want in zip(behind(lambda t: isc.log_probs(t, top=2), (y,)), p):
        assert (got is None and want is None) or torch.equal(got, want)
