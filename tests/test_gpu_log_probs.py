"""isc_log_probs against its definition in 64 bits: alternatives and votes exactly, numbers to their roundings."""
import math

import numpy as np
import pytest

import paper_2108_09413_b200 as isc

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "int8": torch.int8}


def definition(logits, targets, top, scale):
    l = logits.double().cpu() * 1.0
    rows, vocab = l.shape
    bad = torch.isnan(l).any(1) | (l == math.inf).any(1)
    empty = ~bad & (l == -math.inf).all(1)
    clean = torch.where((bad | empty)[:, None], 0.0, l)
    log_p = torch.log_softmax(clean * scale, 1)
    entropy = -torch.where(log_p == -math.inf, 0.0, log_p.exp() * log_p).sum(1)
    log_p[empty] = -math.inf
    log_p[bad] = math.nan
    entropy[empty], entropy[bad] = 0.0, math.nan
    given = None
    if targets is not None:
        t = targets.cpu()
        given = log_p.gather(1, t.clamp(0, vocab - 1)[:, None])[:, 0]
        given = torch.where(t < 0, 0.0, torch.where(t >= vocab, math.nan, given))
    order = torch.sort(torch.where(bad[:, None], -math.inf, l), dim=1, descending=True, stable=True)
    n = min(max(top, 1), vocab)
    ids = torch.where(order.values[:, :n] == -math.inf, -1, order.indices[:, :n])
    votes = torch.bincount(ids[:, 0] + 1, minlength=vocab + 1)[1:]
    alternatives = torch.where(ids < 0, -math.inf, log_p.gather(1, ids.clamp(min=0)))
    alternatives[bad] = math.nan
    more = top - n
    if more > 0:
        ids = torch.cat([ids, torch.full((rows, more), -1)], 1)
        rest = torch.where(bad, math.nan, -math.inf)[:, None].expand(rows, more)
        alternatives = torch.cat([alternatives, rest], 1)
    return given, entropy, ids[:, :top], alternatives[:, :top], votes


def close(got, exact, tolerance):
    # (1.3 times the lowest bfloat16 is -4.4e38: no single-precision number but minus infinity is near it)
    got, exact = got.double().cpu(), torch.where(exact < -3.4028235677973366e38, -math.inf, exact)
    fine = torch.isfinite(exact)
    assert torch.equal(torch.isnan(got), torch.isnan(exact))
    assert torch.equal(got[~fine & ~torch.isnan(exact)], exact[~fine & ~torch.isnan(exact)])
    assert ((got - exact).abs()[fine] <= tolerance[fine]).all(), ((got - exact).abs()[fine] - tolerance[fine]).max()


def check(logits, targets, top, scale=1.0):
    votes = torch.full((logits.shape[1],), 3, dtype=torch.int32, device="cuda")
    given, entropy, ids, alternatives = isc.log_probs(logits, targets, top=top, scale=scale, votes=votes)
    e_given, e_entropy, e_ids, e_alternatives, e_votes = definition(logits, targets, top, scale)
    assert torch.equal(votes.cpu().long() - 3, e_votes)
    # A logit's difference to the largest is rounded three times (subtraction, factor, the factor itself), its exponential is within
    # two units, a sum takes a rounding for each term of a thread and for each step of joining: 256 + 40 at most here.  The
    # terms' errors grow with |z|, weighted by probability: at most 20 where they count.  The logarithm turns the sum's relative
    # error into an absolute one; the entropy's second term has it relative to its size.
    unit = 2.0**-24
    part = (256 + 40 + 4 + 3 * 20) * unit
    lp = lambda e: part + 4 * unit * e.abs()  # noqa: E731
    if targets is not None:
        close(given, e_given, lp(e_given))
    close(entropy, e_entropy, part * (2 + 2 * e_entropy.abs()))
    if top:
        assert torch.equal(ids.cpu().long(), e_ids)
        close(alternatives, e_alternatives, lp(e_alternatives))
    else:
        assert ids is None and alternatives is None


def some_targets(rows, vocab, g):
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    return torch.where(torch.rand(rows, device="cuda", generator=g) < 0.1, -1, t)


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32", "int8"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (70, 10), (33, 64), (40, 65), (7, 1000), (9, 1024), (5, 1025), (300, 2000), (3, 5003), (2, 33000), (1, 131072), (160, 12001)])
@pytest.mark.parametrize("top,pad", [(0, 0), (1, 0), (5, 7), (32, 16)])
def test_against_the_definition(kind, rows, vocab, top, pad):
    g = torch.Generator(device="cuda").manual_seed(rows * vocab + top)
    logits = torch.randn(rows, vocab + pad, device="cuda", generator=g) * (30.0 if kind == "int8" else 3.0)
    logits = (logits.round().clamp(-128, 127) if kind == "int8" else logits).to(TYPES[kind])[:, :vocab]
    check(logits, some_targets(rows, vocab, g), top, 0.1 if kind == "int8" else 0.8)


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("vocab", [10, 63, 700, 1030, 9001, 66000])
@pytest.mark.parametrize("top", [1, 4, 32])
def test_masks_and_values_that_are_no_numbers(kind, vocab, top):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    rows = 14
    low = torch.finfo(TYPES[kind]).min
    x = torch.randn(rows, vocab, device="cuda", generator=g)
    x[0] = -math.inf                                           # nothing left
    x[1] = -math.inf
    x[1, vocab // 2] = -5.0                                    # one left
    x[2, torch.rand(vocab, device="cuda", generator=g) < 0.97] = -math.inf
    x[3] = low                                                 # all at the type's lowest value: even
    x[4, 1:] = low
    x[5, vocab - 1] = math.nan
    x[6, 0] = math.inf
    x[7] = -math.inf
    x[7, vocab - 1] = math.nan
    x[8] = math.inf
    x[9, : vocab // 2] = -math.inf
    x[10, ::2] = low
    x[11] = torch.finfo(TYPES[kind]).max
    targets = torch.arange(rows, device="cuda") % vocab
    targets[12], targets[13] = vocab, 2**40
    check(x.to(TYPES[kind]), targets, top)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("vocab", [50, 900, 4096, 40001])
def test_ties_go_to_the_lowest_index(kind, vocab):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    few = torch.randint(0, 3, (6, vocab), device="cuda", generator=g)
    few[0] = 1
    few[1] = torch.arange(vocab, device="cuda") // 7 % 3
    x = few.to(TYPES[kind])
    if kind != "int8":
        x[2] = torch.where(few[2] == 1, 0.0, -0.0)             # the two zeros are one value
    for top in (1, 3, 32):
        check(x, None, top)


@pytest.mark.parametrize("vocab", [8192, 65536, 131072])
def test_large_logits_in_one_thread_s_share(vocab):
    """Rows whose large logits share one thread's chunks, so that the candidates outnumber the room for them; rising and falling rows."""
    i = torch.arange(vocab, device="cuda", dtype=torch.float32)
    rows = [torch.where(i // 8 % step < 1, 100.0 - i * 2.0**-12, i * 2.0**-20) for step in (128, 256, 512, 1024)]
    rows += [torch.where(i // 8 % step < 32, 50.0 + (i * 37 % 1021) * 2.0**-7, -i) for step in (128, 512, 1024)]
    rows += [i * 2.0**-10, -i * 2.0**-10]
    x = torch.stack(rows)
    for r in (x, x[2:3], x.expand(9, vocab).repeat(40, 1)):
        check(r, None, 32)


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32", "int8"])
@pytest.mark.parametrize("vocab,pad", [(17001, 0), (20480, 16), (70003, 5)])
def test_many_long_rows(kind, vocab, pad):
    """More rows than blocks: each block's copies run on from row to row, over rows of every sort."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    rows = 900
    x = torch.randn(rows, vocab + pad, device="cuda", generator=g) * (30.0 if kind == "int8" else 3.0)
    x[::7] = x[::7].round()                                    # many ties
    x[3::50] = 1.0                                             # nothing but ties: more candidates than there is room for
    x[4::50] = torch.where(torch.arange(vocab + pad, device="cuda") // (16 if kind == "int8" else 8) % 512 < 1, 20.0, 0.0)
    if kind != "int8":
        x[5::50] = -math.inf
        x[6::50, vocab // 2:] = -math.inf
        x[8::50, vocab - 1] = math.nan
        x[9::50, 0] = math.inf
        x[10::50] = torch.finfo(TYPES[kind]).min
        x[11::50, torch.rand(vocab + pad, device="cuda", generator=g) < 0.999] = torch.finfo(TYPES[kind]).min
    x = (x.round().clamp(-128, 127) if kind == "int8" else x).to(TYPES[kind])[:, :vocab]
    for top in (0, 3, 32):
        check(x, some_targets(rows, vocab, g), top, 0.1 if kind == "int8" else 1.3)


def test_zero_rows_and_parts_not_asked_for():
    x = torch.randn(4, 100, device="cuda")
    assert [t if t is None else tuple(t.shape) for t in isc.log_probs(x[:0], torch.zeros(0, dtype=torch.int64, device="cuda"), top=2)] == [(0,), (0,), (0, 2), (0, 2)]
    assert isc.log_probs(x, None, entropy=False) == (None, None, None, None)


def test_same_call_same_bits_on_a_stream_and_in_a_graph():
    g = torch.Generator(device="cuda").manual_seed(3)
    for rows, vocab in ((2, 70000), (500, 3000), (900, 30)):
        x = torch.randn(rows, vocab, device="cuda", generator=g).bfloat16()
        t = some_targets(rows, vocab, g)
        first = isc.log_probs(x, t, top=5)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        second = isc.log_probs(x, t, top=5, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        votes = torch.zeros(vocab, dtype=torch.int32, device="cuda")
        with torch.cuda.graph(graph):
            third = isc.log_probs(x, t, top=5, votes=votes)
        graph.replay()
        graph.replay()
        for a, b, c in zip(first, second, third):
            assert torch.equal(a, b) and torch.equal(a, c)
        assert votes.sum() == 2 * rows


def test_votes_are_the_library_s_own():
    """The int8 logits of a layer list's noisy copies: the votes are isc_sample_counts', and the decision follows."""
    import workloads as wl
    model = isc.Model(wl.spread_model("tiny_cnn"))
    counts, logits = model.sample_counts(wl.spread_image(), wl.NOISE_SEED, 0, 1, 0, 3000, 0.25, want_logits=True)
    votes = torch.zeros(10, dtype=torch.int32, device="cuda")
    labels = torch.full((3000,), 4, device="cuda")
    lp, entropy, ids, _ = isc.log_probs(torch.from_numpy(logits).cuda(), labels, top=2, scale=0.25, votes=votes)
    np.testing.assert_array_equal(votes.cpu().numpy(), counts)
    assert isc.predict_decide(votes.cpu().numpy(), 0.001) == isc.predict_decide(counts, 0.001)
    check(torch.from_numpy(logits).cuda(), labels, 2, 0.25)
