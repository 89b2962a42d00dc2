"""isc_rms_norm_quant against its definition in 64 bits: codes bit for bit, the scale and the sum to their roundings."""
import ctypes as C

import numpy as np
import pytest

import paper_2108_09413_b200 as isc

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def definition(x, r, w, eps):
    h = x.double().cpu()
    if r is not None:
        h = h + r.double().cpu()
    p = h * w.double().cpu()
    most = p.abs().amax(1)
    scale = most / torch.sqrt(h.square().mean(1) + eps) / 127.0
    codes = torch.where(most[:, None] > 0, torch.round(p * 127.0 / most[:, None]), 0.0)
    bad = ~(torch.isfinite(p).all(1) & torch.isfinite(h).all(1))
    codes[bad] = 0
    scale[bad] = float("nan")
    scale[~bad & (most == 0)] = 0.0
    return codes.to(torch.int8), scale, h


def check(got, x, r, w, eps=EPS):
    q, scale, total = got
    codes, exact, h = definition(x, r, w, eps)
    assert torch.equal(q.cpu(), codes)
    # the sum of squares takes at most 32 + 9 + 16 roundings to a thread, a warp and a block; the root halves their sum, and six
    # more follow.  Rows in double precision are nearer
    np.testing.assert_allclose(scale.double().cpu().numpy(), exact.numpy(), rtol=64 * 2.0**-24, atol=2.0**-149)
    if total is not None:
        # rounded to single precision and then to its type: half a step, and what the first rounding adds to it
        half = torch.finfo(total.dtype).eps / 2
        fine = torch.isfinite(h)
        off = (total.double().cpu() - h).abs()[fine]
        assert (off <= half * (1 + 2.0**-7) * h.abs()[fine] + torch.finfo(total.dtype).smallest_normal * half).all()
        assert torch.equal(torch.isfinite(total.cpu()), fine)


def rows_of(values, pad):
    wide = torch.zeros(values.shape[0], values.shape[1] + pad, dtype=values.dtype, device="cuda")
    wide[:, :values.shape[1]] = values
    return wide[:, :values.shape[1]]


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 7), (5, 8), (1, 4096), (37, 1024), (9, 1025), (130, 1032), (4, 5000), (300, 64), (2, 16384), (2, 16385), (3, 20001)])
@pytest.mark.parametrize("pad", [0, 8, 13])
def test_codes_scale_and_sum(kind, rows, width, pad):
    g = torch.Generator(device="cuda").manual_seed(rows * width + pad)
    dtype = TYPES[kind]
    x, r = (rows_of((torch.randn(rows, width, device="cuda", generator=g) * 3).to(dtype), pad) for _ in range(2))
    w = 1 + 0.2 * torch.randn(width, device="cuda", generator=g)
    check(isc.rms_norm_quant(x, w.to(dtype), EPS, residual=r), x, r, w.to(dtype))
    check(isc.rms_norm_quant(x, w, EPS), x, None, w)                    # weights in single precision, no residual
    assert isc.rms_norm_quant(x, w, EPS)[2] is None


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("width", [64, 900, 3000, 17000])
def test_codes_between_two(kind, width):
    """Quotients that lie exactly between two codes, and next to that: half integers times the step, with and without an
    element's last bit changed."""
    dtype = TYPES[kind]
    g = torch.Generator(device="cuda").manual_seed(width)
    k = torch.randint(-127, 127, (40, width), device="cuda", generator=g).double() + 0.5
    k[:, width // 2] = 127.0
    x = (k * 0.25).to(dtype)
    near = torch.nextafter(x.float(), torch.where(torch.rand(x.shape, device="cuda", generator=g) < 0.5, 1e9, -1e9).float())
    for v in (x, near.to(dtype), (x.double() * 3.3).to(dtype)):
        w = torch.ones(width, device="cuda", dtype=dtype)
        check(isc.rms_norm_quant(v, w), v, None, w)
        check(isc.rms_norm_quant(v, w, residual=torch.zeros_like(v)), v, torch.zeros_like(v), w)


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("width", [100, 2048, 2051, 18000])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 0.5])
def test_rows_at_the_ends_of_the_range(kind, width, eps):
    """Zeros, subnormal and largest numbers, infinities and NaN, each in a row of its own between ordinary ones."""
    dtype = TYPES[kind]
    g = torch.Generator(device="cuda").manual_seed(width)
    x = torch.randn(12, width, device="cuda", generator=g)
    top = torch.finfo(dtype).max
    x[1] = 0.0
    x[2] = 0.0
    x[2, width // 3] = torch.finfo(dtype).smallest_normal
    x[3] *= top / 8
    x[4] = -top
    x[5, width - 1] = float("inf")
    x[6, 0] = float("-inf")
    x[7, width // 2] = float("nan")
    x[8] *= torch.finfo(dtype).smallest_normal * 4
    x[9, 5] = top / 2
    x = x.to(dtype)
    w = (1 + 0.2 * torch.randn(width, device="cuda", generator=g)).to(dtype)
    check(isc.rms_norm_quant(x, w, eps), x, None, w, eps)
    w[3] = 0.0
    check(isc.rms_norm_quant(x, w, eps), x, None, w, eps)
    w[7] = float("inf")
    q, scale, _ = isc.rms_norm_quant(x, w, eps)
    assert torch.isnan(scale).all() and not q.any()


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,width", [(5000, 1032), (2600, 2048), (1301, 4096), (700, 8192), (400, 16384)])
@pytest.mark.parametrize("pad", [0, 8])
def test_many_rows(kind, rows, width, pad):
    """More rows than teams: rows are brought ahead, among them rows of every sort, with the sum in place and without a residual."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    dtype = TYPES[kind]
    top = torch.finfo(dtype).max
    x, r = (3 * torch.randn(rows, width, device="cuda", generator=g) for _ in range(2))
    for t in (x, r):
        t[1::40] = 0.0
        t[3::40, 7] = float("inf")
        t[4::40, width - 1] = float("nan")
        t[6::40] *= torch.finfo(dtype).smallest_normal * 4
    x[5::40] = -top / 2
    x[8::40] = (torch.randint(-127, 127, (width,), device="cuda", generator=g) + 0.5) * 0.25     # quotients between two codes
    x[8::40, width // 2] = 31.75
    r[8::40] = 0.0
    x, r = rows_of(x.to(dtype), pad), rows_of(r.to(dtype), pad)
    w = (1 + 0.2 * torch.randn(width, device="cuda", generator=g))
    check(isc.rms_norm_quant(x, w.to(dtype), EPS), x, None, w.to(dtype))
    check(isc.rms_norm_quant(x, torch.ones_like(w), EPS, residual=r), x, r, torch.ones_like(w))
    kept = r.clone()
    got = isc.rms_norm_quant(x, w, EPS, residual=r, sum_out=r)
    check(got, x, kept, w)
    again = isc.rms_norm_quant(x, w, EPS, residual=kept)
    for a, b in zip(got, again):
        assert torch.equal(a.nan_to_num(1.0), b.nan_to_num(1.0))


def test_sum_that_leaves_its_type():
    x = torch.full((2, 40), 60000.0, device="cuda", dtype=torch.float16)
    w = torch.ones(40, device="cuda", dtype=torch.float16)
    q, scale, total = isc.rms_norm_quant(x, w, residual=x)
    assert torch.isinf(total).all() and (q == 127).all()               # the norm is of the sum before it is rounded
    np.testing.assert_allclose(scale.cpu().numpy() * 127, 1.0, rtol=64 * 2.0**-24)


@pytest.mark.parametrize("width", [300, 4096, 20000])
def test_sum_in_place(width):
    for into in ("x", "residual"):
        t = {n: torch.randn(20, width, device="cuda").bfloat16() for n in ("x", "residual")}
        w = torch.randn(width, device="cuda").bfloat16()
        x, r = t["x"].clone(), t["residual"].clone()
        got = isc.rms_norm_quant(t["x"], w, residual=t["residual"], sum_out=t[into])
        assert got[2] is t[into]
        check(got, x, r, w)
        assert torch.equal(t["x" if into == "residual" else "residual"], x if into == "residual" else r)


def test_bytes_outside_the_rows_stay():
    rows, width, pitch = 11, 333, 352
    x = torch.randn(rows, width, device="cuda")
    q = torch.full((rows + 2, pitch), 77, dtype=torch.int8, device="cuda")
    total = torch.full((rows + 2, pitch), 5.0, device="cuda")
    scale = torch.full((rows + 2,), 5.0, device="cuda")
    w = torch.ones(width, device="cuda")
    rc = isc.lib().isc_rms_norm_quant(x.data_ptr(), width, None, 0, w.data_ptr(), 2, 2, rows, width, EPS, total[1:].data_ptr(), pitch,
                                      q[1:].data_ptr(), pitch, scale[1:].data_ptr(), C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    check((q[1:-1, :width], scale[1:-1], total[1:-1, :width]), x, None, w)
    assert (q[0] == 77).all() and (q[-1] == 77).all() and (q[:, width:] == 77).all()
    assert (total[0] == 5).all() and (total[-1] == 5).all() and (total[:, width:] == 5).all()
    assert scale[0] == 5 and scale[-1] == 5


def test_captured_and_on_another_stream():
    x, r = (torch.randn(64, 2048, device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(2048, device="cuda").bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = isc.rms_norm_quant(x, w, residual=r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check(got, x, r, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = isc.rms_norm_quant(x, w, residual=r)
    for seed in range(3):
        x.copy_(torch.randn(64, 2048, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        check(got, x, r, w)
