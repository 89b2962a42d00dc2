"""The operators' arguments on a GPU: what is refused, rows far apart, large and small factors."""
import ctypes as C

import numpy as np
import pytest

import paper_2108_09413_b200 as isc

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def refused(call):
    with pytest.raises(isc.IscError) as e:
        call()
    return e.value.code


def test_norm_refuses():
    x, w = torch.zeros(4, 64, device="cuda").bfloat16(), torch.ones(64, device="cuda").bfloat16()
    for call in (lambda: isc.rms_norm_quant(x.to(torch.int8), w), lambda: isc.rms_norm_quant(x.double(), w.double()), lambda: isc.rms_norm_quant(x, w.half()),
                 lambda: isc.rms_norm_quant(x, w[:63]), lambda: isc.rms_norm_quant(x[0], w), lambda: isc.rms_norm_quant(x.t(), w[:4]), lambda: isc.rms_norm_quant(x, w, residual=x[:3]),
                 lambda: isc.rms_norm_quant(x, w, residual=x.half()), lambda: isc.rms_norm_quant(x, w, sum_out=x.float()), lambda: isc.rms_norm_quant(x, w.cpu()),
                 lambda: isc.rms_norm_quant(x, w, eps=-1.0), lambda: isc.rms_norm_quant(x[:1].expand(4, 64), w), lambda: isc.rms_norm_quant(x, w.requires_grad_())):
        assert refused(call) == -1
    with torch.no_grad():
        assert isc.rms_norm_quant(x, w)[1].eq(0).all()


def test_linear_refuses():
    x, w = torch.zeros(4, 64, device="cuda", dtype=torch.int8), torch.zeros(10, 64, device="cuda", dtype=torch.int8)
    xs, ws, ids = torch.ones(4, device="cuda"), torch.ones(10, device="cuda"), torch.zeros(4, device="cuda", dtype=torch.int32)
    ad = (torch.zeros(2, 8, 64, device="cuda").half(), torch.zeros(2, 10, 8, device="cuda").half(), torch.ones(2, device="cuda"))
    for call in (lambda: isc.quant_linear(x.float(), xs, w, ws), lambda: isc.quant_linear(x, xs[:3], w, ws), lambda: isc.quant_linear(x, xs, w[:, :48], ws), lambda: isc.quant_linear(x, xs, w, ws.half()),
                 lambda: isc.quant_linear(x, xs, w, ws, bias=torch.zeros(9, device="cuda")), lambda: isc.quant_linear(x, xs, w, ws, out_dtype=torch.int8),
                 lambda: isc.quant_linear(x, xs, w, ws, out=torch.zeros(4, 11, device="cuda")), lambda: isc.quant_linear(x, xs, w, ws, adapters=ad),
                 lambda: isc.quant_linear(x, xs, w, ws, adapters=ad, adapter_ids=ids.long()), lambda: isc.quant_linear(x, xs, w, ws, adapters=(ad[0].float(), ad[1].float(), ad[2]), adapter_ids=ids),
                 lambda: isc.quant_linear(x, xs, w, ws, adapters=(ad[0], ad[1][:1], ad[2]), adapter_ids=ids), lambda: isc.quant_linear(x, xs, w, ws, adapters=(ad[0][:, ::2], ad[1][:, :, :4], ad[2]), adapter_ids=ids)):
        assert refused(call) == -1
    wide = torch.zeros(4, 72, device="cuda", dtype=torch.int8)
    assert refused(lambda: isc.quant_linear(wide[:, :64], xs, w, ws)) == -3            # a pitch of 72
    assert refused(lambda: isc.quant_linear(wide.view(-1)[8:8 + 256].view(4, 64), xs, w, ws)) == -3
    assert refused(lambda: isc.quant_linear(x, xs, w, ws, adapters=(ad[0][:, :6].contiguous(), ad[1][:, :, :6].contiguous(), ad[2]), adapter_ids=ids)) == -3


def test_log_probs_refuses():
    x = torch.zeros(4, 64, device="cuda")
    t = torch.zeros(4, device="cuda", dtype=torch.int64)
    for call in (lambda: isc.log_probs(x.double()), lambda: isc.log_probs(x.t()), lambda: isc.log_probs(x, t.int()), lambda: isc.log_probs(x, t[:3]), lambda: isc.log_probs(x, t.cpu()),
                 lambda: isc.log_probs(x, t, top=33), lambda: isc.log_probs(x, t, scale=0.0), lambda: isc.log_probs(x, t, votes=torch.zeros(63, device="cuda", dtype=torch.int32)),
                 lambda: isc.log_probs(x, t, votes=torch.zeros(64, device="cuda")), lambda: isc.log_probs(x.requires_grad_(), t)):
        assert refused(call) == -1


def test_rows_further_apart_than_32_bits():
    far = 1_200_000_016                                                    # elements; three rows of 16-bit numbers span 4.8 GB
    base = torch.empty(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    rows = base.as_strided((3, 4096), (far, 1))
    near = torch.randn(3, 4096, device="cuda").bfloat16()
    rows.copy_(near)
    w = torch.ones(4096, device="cuda").bfloat16()
    for a, b in zip(isc.rms_norm_quant(rows, w, residual=near), isc.rms_norm_quant(near, w, residual=near)):
        assert torch.equal(a, b)
    targets = torch.tensor([5, 4000, -1], device="cuda")
    for width in (4096, 3000, 60):
        for a, b in zip(isc.log_probs(rows[:, :width], targets.clamp(max=width - 1), top=7), isc.log_probs(near[:, :width].contiguous(), targets.clamp(max=width - 1), top=7)):
            assert torch.equal(a, b)
    x = torch.randint(-127, 128, (3, 512), device="cuda").to(torch.int8)
    w8 = torch.randint(-127, 128, (4096, 512), device="cuda").to(torch.int8)
    one, scale = torch.ones(3, device="cuda"), torch.full((4096,), 1e-4, device="cuda")
    y = isc.quant_linear(x, one, w8, scale, out=rows)
    assert torch.equal(y, isc.quant_linear(x, one, w8, scale))
    bytes_ = base.view(torch.int8)
    xf = bytes_.as_strided((3, 512), (2 * far // 16 * 16, 1))
    xf.copy_(x)
    assert torch.equal(isc.quant_linear(xf, one, w8, scale), isc.quant_linear(x, one, w8, scale))
    wf = bytes_.as_strided((3, 512), (2 * far // 16 * 16, 1), 4096)
    wf.copy_(w8[:3])
    assert torch.equal(isc.quant_linear(x, one, wf, scale[:3]), isc.quant_linear(x, one, w8[:3], scale[:3]))
    assert torch.equal(isc.quant_linear(x[:1], one[:1], wf, scale[:3]), isc.quant_linear(x[:1], one[:1], w8[:3], scale[:3]))


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 50.0, 1e9, 1e30, 1e38])
def test_log_probs_of_extreme_factors(scale):
    for vocab in (12, 50, 700, 20000):
        g = torch.Generator(device="cuda").manual_seed(vocab)
        x = torch.randn(5, vocab, device="cuda", generator=g)
        x[1, 3] = x[1].max()                                               # two share everything at a large factor
        targets = torch.tensor([0, 3, 1, int(x[3].argmax()), 2], device="cuda")
        given, entropy, ids, top = isc.log_probs(x, targets, top=3, scale=scale)
        z = (x.double() - x.double().amax(1, keepdim=True)) * scale
        log_p = z - torch.logsumexp(z, 1, keepdim=True)
        exact = log_p.gather(1, targets[:, None])[:, 0]
        assert torch.equal(ids.long(), torch.sort(x, dim=1, descending=True, stable=True).indices[:, :3])
        # relative to the size: three roundings of z and the sum's; beyond single precision's range minus infinity
        lost = exact.abs() > 3.4e38
        assert torch.isinf(given[lost]).all()
        np.testing.assert_allclose(given[~lost].double().cpu(), exact[~lost].cpu(), rtol=8 * 2.0**-24, atol=400 * 2.0**-24)
        h = -(log_p.exp() * torch.where(log_p.exp() > 0, log_p, 0.0)).sum(1)
        np.testing.assert_allclose(entropy.double().cpu(), h.cpu(), atol=400 * 2.0**-24 * 12)


def test_status_after_ordinary_work():
    assert isc.lib().isc_operator_status(C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
