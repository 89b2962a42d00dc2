"""The operators as they are used together: the residual stream's norm, the vocabulary's projection with the adapters of the rows'
requests, the log probabilities, and the decision on the votes of noisy copies."""
import numpy as np
import pytest

import paper_2108_09413_b200 as isc

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

EPS = 1e-6


class Head:
    """The answer end of a quantised language model with random weights."""

    def __init__(self, width, vocab, adapters, rank, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dev = dict(device="cuda", generator=g)
        self.norm = (1 + 0.1 * torch.randn(width, **dev)).bfloat16()
        pitch = (width + 15) // 16 * 16                                            # as quant_linear takes it
        self.w = torch.randint(-127, 128, (vocab, pitch), **dev).to(torch.int8)[:, :width]
        self.w_scale = (0.5 + torch.rand(vocab, **dev)) / (73.0 * width**0.5)
        self.adapters = ((torch.randn(adapters, rank, width, **dev) / width**0.5).bfloat16(), (0.3 * torch.randn(adapters, vocab, rank, **dev) / rank**0.5).bfloat16(),
                         torch.ones(adapters, device="cuda")) if adapters else None

    def __call__(self, x, residual, ids, targets, top, votes):
        q, scale, _ = isc.rms_norm_quant(x, self.norm, EPS, residual=residual, sum_out=residual)
        logits = isc.quant_linear(q, scale, self.w, self.w_scale, adapters=self.adapters, adapter_ids=ids, out_dtype=torch.float32)
        return logits, isc.log_probs(logits, targets, top=top, votes=votes)

    def exact(self, x, residual, ids):
        h = x.double() + residual.double()
        p = h * self.norm.double()
        most = p.abs().amax(1, keepdim=True)
        q = torch.round(p * 127.0 / most)
        scale = most / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) / 127.0
        y = (q @ self.w.double().T) * self.w_scale.double()
        if self.adapters is not None:
            a, b, c = (t.double() for t in self.adapters)
            for i in range(len(c)):
                mine = (ids == i).nonzero()[:, 0]
                y[mine] += c[i] * ((q[mine] @ a[i].T) @ b[i].T)
        return y * scale


@pytest.mark.parametrize("rows,width,vocab,adapters,rank", [(1, 2048, 1000, 3, 16), (40, 1000, 5003, 8, 8), (300, 512, 2050, 2, 32), (700, 1024, 40, 0, 16), (3, 4096, 32000, 2, 64)])
def test_log_probs_of_the_whole_path(rows, width, vocab, adapters, rank):
    head = Head(width, vocab, adapters, rank, rows)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r = ((2 * torch.randn(rows, width, device="cuda", generator=g)).bfloat16() for _ in range(2))
    ids = torch.randint(-1, adapters, (rows,), device="cuda", generator=g).int() if adapters else None
    targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    exact = head.exact(x, r, ids)
    before = r.clone()
    votes = torch.zeros(vocab, dtype=torch.int32, device="cuda")
    logits, (given, entropy, top_ids, top) = head(x, r, ids, targets, 4, votes)
    assert torch.equal(r, (x.float() + before.float()).bfloat16())                 # the stream goes on
    # Codes are exact, so a logit is off by its single-precision roundings and those of the row's scale (2^-18 of it in all), and by
    # the adapters' sums, whose terms come to at most 40 times the logits' size here (2^-18 of that)
    off = 41 * 2.0**-18 * exact.abs().amax(1, keepdim=True)
    assert ((logits.double() - exact).abs() <= off).all()
    log_p = torch.log_softmax(exact, 1)
    slack = 2 * off[:, 0] + 4e-5                                                   # a log probability moves by two logits' errors
    assert ((given.double() - log_p.gather(1, targets[:, None])[:, 0]).abs() <= slack).all()
    assert ((entropy.double() + (log_p.exp() * log_p).sum(1)).abs() <= slack * (2 + np.log(vocab))).all()
    # alternatives are those of the logits that were computed
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :4]
    assert torch.equal(top_ids.long(), order)
    assert torch.equal(votes.long(), torch.bincount(order[:, 0], minlength=vocab))


def test_noisy_copies_of_a_prompt_are_certified():
    """Votes of noisy hidden states, counted on the GPU in two batches, decided by Algorithms 1 and 2."""
    width, vocab, n = 512, 30, 4000
    head = Head(width, vocab, 0, 16, 5)
    g = torch.Generator(device="cuda").manual_seed(2)
    prompt = torch.randn(width, device="cuda", generator=g)
    favourite = int(head(prompt[None].bfloat16(), torch.zeros(1, width, device="cuda").bfloat16(), None, torch.zeros(1, dtype=torch.int64, device="cuda"), 1, None)[1][2])
    counts = []
    for copies in (100, n):
        votes = torch.zeros(vocab, dtype=torch.int32, device="cuda")
        for _ in range(2):
            noisy = (prompt + 0.05 * torch.randn(copies // 2, width, device="cuda", generator=g)).bfloat16()
            head(noisy, torch.zeros_like(noisy), None, torch.full((copies // 2,), -1, device="cuda"), 0, votes)
        counts.append(votes.cpu().numpy())
        assert counts[-1].sum() == copies
    cls, radius, p_lower = isc.certify_decide(counts[0], counts[1], n, 0.05, 0.001)
    assert cls == favourite and radius > 0 and p_lower > 0.5
    assert isc.predict_decide(counts[1], 0.001) == favourite


def test_the_path_in_a_graph():
    head = Head(1024, 3000, 4, 16, 9)
    g = torch.Generator(device="cuda").manual_seed(3)
    x, r = (torch.randn(20, 1024, device="cuda", generator=g).bfloat16() for _ in range(2))
    ids = torch.randint(-1, 4, (20,), device="cuda", generator=g).int()
    targets = torch.randint(0, 3000, (20,), device="cuda", generator=g)
    votes = torch.zeros(3000, dtype=torch.int32, device="cuda")
    head(x, r.clone(), ids, targets, 3, None)
    graph = torch.cuda.CUDAGraph()
    stream = r.clone()
    with torch.cuda.graph(graph):
        stream.copy_(r)
        captured = head(x, stream, ids, targets, 3, votes)[1]
    for step in range(4):
        x.copy_(torch.randn(20, 1024, device="cuda", generator=g))
        ids.copy_(torch.randint(-1, 4, (20,), device="cuda", generator=g))
        graph.replay()
        torch.cuda.synchronize()
        again = head(x, r.clone(), ids, targets, 3, None)[1]
        for a, b in zip(captured, again):
            assert torch.equal(a, b)
    assert votes.sum() == 80


def test_inputs_of_another_stream_may_be_dropped():
    """What the calls on a side stream, which is behind, were given goes out of use right after them; its memory is not handed out again
    before they have run."""
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

    got_q, got_scale, _ = behind(lambda *t: isc.rms_norm_quant(*t, stream=side), (x, w))
    assert torch.equal(got_q, q) and torch.equal(got_scale, scale)
    assert torch.equal(behind(lambda *t: isc.quant_linear(*t, stream=side), (q, scale, matrix, factors)), y)
    for got, want in zip(behind(lambda t: isc.log_probs(t, top=2, stream=side), (y,)), p):
        assert (got is None and want is None) or torch.equal(got, want)
