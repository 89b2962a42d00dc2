"""isc_quant_linear against its definition in 64 bits."""
import ctypes as C

import pytest

import paper_2108_09413_b200 as isc

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def problem(rows, k, n, seed=0, adapters=0, rank=16, adapter_type="bf16", bias=False, order="mixed", pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * rows + 11 * k + 13 * n)
    dev = dict(device="cuda", generator=g)
    pitch = (k + 15 & ~15) + 16 * pad
    x = torch.randint(-128, 128, (rows, pitch), **dev).to(torch.int8)[:, :k]
    w = torch.randint(-128, 128, (n, pitch), **dev).to(torch.int8)[:, :k]
    s = dict(x=x, w=w, x_scale=0.01 + torch.rand(rows, **dev), w_scale=(0.1 + torch.rand(n, **dev)) / (5000.0 * k**0.5),
             bias=torch.randn(n, **dev) if bias else None, adapters=None, adapter_ids=None)
    if adapters:
        t = TYPES[adapter_type]
        a = (torch.randn(adapters, rank, k, **dev) / (70.0 * k**0.5)).to(t)
        b = (torch.randn(adapters, n, rank, **dev) / rank**0.5).to(t)
        s["adapters"] = (a, b, 0.5 + torch.rand(adapters, **dev))
        if order == "mixed":
            ids = torch.randint(-1, adapters, (rows,), **dev)
        else:
            ids = torch.arange(rows, device="cuda") * (adapters + 1) // rows - 1
        s["adapter_ids"] = ids.to(torch.int32)
    return s


def definition(s):
    x = s["x"].double()
    base = (x @ s["w"].double().T) * s["w_scale"].double()
    inner = torch.zeros_like(base)
    size = torch.zeros_like(base)                       # what the second product's terms come to
    if s["adapters"] is not None:
        a, b, c = (t.double() for t in s["adapters"])
        for i in range(a.shape[0]):
            mine = (s["adapter_ids"] == i).nonzero()[:, 0]
            if len(mine):
                part = x[mine] @ a[i].T
                inner[mine] = c[i] * (part @ b[i].T)
                size[mine] = c[i] * ((x[mine].abs() @ a[i].abs().T) @ b[i].abs().T)
        inner[s["adapter_ids"] >= a.shape[0]] = float("nan")
    scale = s["x_scale"].double()[:, None]
    bias = s["bias"].double() if s["bias"] is not None else 0.0
    return (base + inner) * scale + bias, (base.abs() + inner.abs()) * scale, size * scale


def check(got, s, dtype):
    exact, terms, size = definition(s)
    assert got.dtype == dtype and got.shape == exact.shape
    half = torch.finfo(dtype).eps / 2
    # The integer sum is exact; turned into single precision, scaled twice, added to and offset: six roundings of the terms.  The
    # inner sums: products of codes and adapter are exact, their sums are off by at most 2^-18 of the absolute terms (32 additions in
    # a row to a chain, the rest tree-like, and the matrix unit's own truncations); the outer ones take 64 additions at most.
    off = (got.double() - exact).abs()
    allowed = half * exact.abs() + 8 * 2.0**-24 * terms + 2.0**-18 * size + torch.finfo(dtype).smallest_normal * half
    fine = ~torch.isnan(exact)
    assert torch.equal(torch.isnan(got), ~fine)
    assert (off[fine] <= allowed[fine]).all(), (off - allowed)[fine].max()


def call(s, **more):
    return isc.quant_linear(s["x"], s["x_scale"], s["w"], s["w_scale"], bias=s["bias"], adapters=s["adapters"], adapter_ids=s["adapter_ids"], **more)


@pytest.mark.parametrize("out", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,k,n", [(1, 1, 1), (1, 16, 8), (2, 20, 33), (5, 128, 128), (16, 129, 130), (17, 640, 200), (33, 512, 1000), (64, 4096, 512), (100, 1000, 36), (129, 2048, 260),
                                      (257, 300, 300), (300, 1024, 2050), (1, 4096, 4096), (1000, 640, 520), (2500, 256, 1027)])
def test_without_adapters(out, rows, k, n):
    for bias in (False, True):
        s = problem(rows, k, n, bias=bias, pad=int(bias))
        check(call(s, out_dtype=TYPES[out]), s, TYPES[out])


@pytest.mark.parametrize("out", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,k,n,adapters,rank", [(1, 16, 8, 1, 4), (1, 4096, 4096, 8, 16), (7, 333, 100, 3, 8), (16, 1024, 640, 20, 16), (64, 2048, 768, 40, 16), (70, 640, 257, 2, 64),
                                                    (130, 520, 1025, 5, 36), (300, 1024, 512, 7, 128), (1100, 256, 384, 4, 20), (2049, 640, 160, 60, 32), (1024, 1030, 130, 1, 100)])
@pytest.mark.parametrize("order", ["mixed", "runs"])
def test_with_adapters(out, kind, rows, k, n, adapters, rank, order):
    s = problem(rows, k, n, adapters=adapters, rank=rank, adapter_type=kind, order=order, bias=rank == 64)
    check(call(s, out_dtype=TYPES[out]), s, TYPES[out])


def test_largest_sums_are_exact():
    """The int32 sums at their largest: k = 65,536 products of -128 and -128, 2^30, and a power of two as scale."""
    x = torch.full((3, 65536), -128, dtype=torch.int8, device="cuda")
    w = torch.full((40, 65536), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    one = torch.ones(40, device="cuda")
    y = isc.quant_linear(x, one[:3], w, one, out_dtype=torch.float32)
    assert (y[:, 0] == 2.0**30).all() and (y[:, 1] == -128.0 * 127 * 65536).all() and (y[:, 2:] == 2.0**30).all()


def test_integers_that_single_precision_holds_are_exact_at_every_split():
    for rows, k, n in ((1, 8192, 128), (9, 4096, 130), (40, 2048, 640), (200, 1536, 1000), (3000, 512, 300)):
        g = torch.Generator(device="cuda").manual_seed(rows)
        x = torch.randint(-20, 21, (rows, k), device="cuda", generator=g).to(torch.int8)
        w = torch.randint(-20, 21, (n, k), device="cuda", generator=g).to(torch.int8)
        y = isc.quant_linear(x, torch.ones(rows, device="cuda"), w, torch.ones(n, device="cuda"), out_dtype=torch.float32)
        assert torch.equal(y.double(), x.double() @ w.double().T)


@pytest.mark.parametrize("rows,order", [(40, "mixed"), (600, "runs"), (1500, "mixed")])
def test_other_rows_adapters_do_not_reach_a_row(rows, order):
    s = problem(rows, 640, 200, adapters=4, rank=24, order=order)
    clean = call(s)
    a, b, c = s["adapters"]
    for t, value in ((a, float("nan")), (b, float("inf")), (a, float("-inf"))):
        poisoned = [a.clone(), b.clone(), c]
        poisoned[0 if t is a else 1][2, 1] = value
        y = isc.quant_linear(s["x"], s["x_scale"], s["w"], s["w_scale"], adapters=tuple(poisoned), adapter_ids=s["adapter_ids"])
        others = s["adapter_ids"] != 2
        assert torch.equal(y[others], clean[others])
        assert not torch.isfinite(y[~others]).all(1).any()


def test_ids_out_of_range_are_seen():
    for rows in (10, 1200):
        s = problem(rows, 256, 140, adapters=3, rank=8)
        s["adapter_ids"][::5] = 3
        s["adapter_ids"][1] = 2**31 - 1
        s["adapter_ids"][2] = -(2**31)
        check(call(s, out_dtype=torch.float32), s, torch.float32)


def test_inner_sums_beyond_half_precision_s_range():
    s = problem(50, 1024, 130, adapters=2, rank=16, adapter_type="fp16")
    a, b, c = s["adapters"]
    a *= 20000.0
    s["adapters"] = (a, b, c * 1e-4)
    check(call(s, out_dtype=torch.float32), s, torch.float32)
    a[0] *= 0
    a[1] = torch.where(torch.rand_like(a[1].float()) < 0.5, 6e-8, -6e-8).half()
    check(call(s, out_dtype=torch.float32), s, torch.float32)


@pytest.mark.parametrize("rows,n,split_out", [(3, 100, True), (60, 1000, True), (700, 333, False)])
def test_into_a_wider_tensor(rows, n, split_out):
    s = problem(rows, 512, n, adapters=3)
    for dtype in TYPES.values():
        for pitch, at in ((n + 16, 0), (n + 13, 5)):
            wide = torch.full((rows + 2, pitch), 7.0, dtype=dtype, device="cuda")
            out = wide[1:-1, at:at + n]
            assert call(s, out=out) is out
            check(out, s, dtype)
            assert (wide[0] == 7).all() and (wide[-1] == 7).all() and (wide[:, :at] == 7).all() and (wide[:, at + n:] == 7).all()


def test_captured_on_two_streams_at_once():
    """Two graphs with work spaces of their own, replayed side by side, and an eager call on a third stream."""
    problems = [problem(33, 1024, 700, seed=i, adapters=5) for i in range(3)]
    graphs = []
    for s in problems[:2]:
        call(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = call(s, out_dtype=torch.float32)
        graphs.append((g, y))
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(20):
        for (g, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        third = call(problems[2], out_dtype=torch.float32, stream=streams[2])
    torch.cuda.synchronize()
    for y, s in zip([graphs[0][1], graphs[1][1], third], problems):
        check(y, s, torch.float32)
    assert isc.lib().isc_operator_status(C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0


def test_zero_rows_and_no_adapters_at_all():
    s = problem(4, 64, 50)
    assert isc.quant_linear(s["x"][:0], s["x_scale"][:0], s["w"], s["w_scale"]).shape == (0, 50)
    none = (torch.zeros(0, 8, 64, device="cuda").half(), torch.zeros(0, 50, 8, device="cuda").half(), torch.zeros(0, device="cuda"))
    ids = torch.full((4,), -1, dtype=torch.int32, device="cuda")
    assert torch.equal(call(s), isc.quant_linear(s["x"], s["x_scale"], s["w"], s["w_scale"], adapters=none, adapter_ids=ids))


def test_ids_without_adapters_are_too_large():
    """A row whose id is the number of adapters or more is NaN, with no adapters too."""
    for rows in (1, 4, 300):
        s = problem(rows, 64, 50)
        none = (torch.zeros(0, 8, 64, device="cuda").half(), torch.zeros(0, 50, 8, device="cuda").half(), torch.zeros(0, device="cuda"))
        ids = torch.arange(rows, dtype=torch.int32, device="cuda") % 2 - 1
        y, plain = isc.quant_linear(s["x"], s["x_scale"], s["w"], s["w_scale"], adapters=none, adapter_ids=ids), call(s)
        assert torch.equal(y[ids < 0], plain[ids < 0]) and torch.isnan(y[ids >= 0]).all()


@pytest.mark.parametrize("rows,k,n,adapters,rank", [(16, 8192, 1024, 8, 16), (13, 8192, 1000, 40, 4), (48, 16384, 2000, 9, 20), (100, 32768, 300, 5, 64), (3, 65536, 70, 2, 128)])
@pytest.mark.parametrize("order", ["mixed", "runs"])
def test_long_sums_of_few_outputs(rows, k, n, adapters, rank, order):
    """Where the most blocks share a tile, narrow and wide ones."""
    s = problem(rows, k, n, adapters=adapters, rank=rank, order=order, bias=True)
    check(call(s, out_dtype=torch.float32), s, torch.float32)
    s["adapters"] = s["adapter_ids"] = None
    check(call(s, out_dtype=torch.bfloat16), s, torch.bfloat16)
