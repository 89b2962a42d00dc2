"""Cases of the operators at the answer end of a quantised language model: the norm that ends the residual stream and hands
on int8 rows, the int8 projection with the low-rank adapters of many requests, and the log probabilities of its logits.

`run` computes a case in its plain form, with elementary torch operations, or, where `own` is true, by the library's
operators; `exact` is each operator's definition in 64 bits.  Rows are tokens (or noisy copies); all data is on the GPU.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


# ------------------------------------------------------------------------------------------- cases

def _norm(rows, width, dtype="bf16", residual=True, pad=0):
    """pad: elements between the end of a row and the next one's start"""
    return dict(op="norm", rows=rows, width=width, dtype=dtype, residual=residual, pad=pad)


def _linear(rows, k, n, rank=16, adapters=8, order="runs", dtype="bf16", bias=False):
    """rank 0: no adapters.  order: "runs" (rows of a request lie together) or "mixed" (every row another request); a tenth
    of the requests has no adapter.  dtype: of the adapters and the output."""
    return dict(op="linear", rows=rows, k=k, n=n, rank=rank, adapters=adapters if rank else 0, order=order, dtype=dtype, bias=bias)


def _log_probs(rows, vocab, dtype="bf16", top=5, masked=0.0, scale=1.0, votes=False, pad=0):
    """masked: the share of logits at minus infinity; with any, every 50th row has nothing else"""
    return dict(op="log_probs", rows=rows, vocab=vocab, dtype=dtype, top=top, masked=masked, scale=scale, votes=votes, pad=pad)


def listed():
    return [
        # one new token of one request: the norm before a projection, where a launch's latency is the time
        dict(name="norm_token", **_norm(1, 4096)),
        # a batch of tokens whose rows are slices of a wider tensor, a width no block divides
        dict(name="norm_batch_slices", **_norm(250, 5000, "fp16", pad=24)),
        # rows in single precision without a residual: a network's first norm
        dict(name="norm_single", **_norm(2048, 2048, "fp32", residual=False)),
        # long prompts in one batch
        dict(name="norm_prompt", **_norm(16384, 8192)),
        # one new token of one request through a square projection: the weights' bytes are the time
        dict(name="linear_token", **_linear(1, 4096, 4096)),
        # one new token for each of 64 requests with 32 adapters among them
        dict(name="linear_decode", **_linear(64, 4096, 12288, adapters=32, order="mixed")),
        # a few prompts of odd lengths, odd sizes everywhere, biases
        dict(name="linear_prompts_odd", **_linear(1003, 2000, 5004, rank=24, adapters=5, dtype="fp16", bias=True)),
        # long prompts of a few requests: the tensor cores' rate is the time
        dict(name="linear_prompt", **_linear(8192, 8192, 8192, rank=32, adapters=4)),
        # one new token: a vocabulary's logits and twenty alternatives
        dict(name="log_probs_token", **_log_probs(1, 131072, top=20)),
        # the votes of N = 100,000 noisy copies over ten classes, from the network's int8 logits
        dict(name="log_probs_classes", **_log_probs(100_000, 10, "int8", top=2, scale=0.1, votes=True)),
        # constrained answers: most tokens masked, some rows altogether; single precision, an odd vocabulary
        dict(name="log_probs_masked", **_log_probs(333, 50_001, "fp32", top=8, masked=0.7, scale=1.25)),
        # every token of a long prompt scored
        dict(name="log_probs_prompt", **_log_probs(4096, 131072, top=5)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "linear", "log_probs"])
    if op == "norm":
        width = _log_int(rng, 64, 20_000)
        rows = max(1, min(_log_int(rng, 1, 60_000), (1 << 27) // width))
        return _norm(rows, width, rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.random() < 0.7, rng.choice([0, 0, 8, 13]))
    if op == "linear":
        k, n = 16 * _log_int(rng, 16, 768), _log_int(rng, 100, 20_000)
        rows = max(1, min(_log_int(rng, 1, 12_000), (1 << 38) // (k * n)))
        rank = rng.choice([0, 4, 8, 16, 16, 32, 40, 64, 128])
        return _linear(rows, k, n, rank, _log_int(rng, 1, 40), rng.choice(["runs", "mixed"]), rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                       rng.random() < 0.4)
    vocab = _log_int(rng, 2, 260_000)
    rows = max(1, min(_log_int(rng, 1, 200_000), (1 << 28) // vocab))
    masked = rng.choice([0.0, 0.0, 0.3, 0.95])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"] if masked else ["bf16", "bf16", "fp16", "fp32", "int8"])
    scale = 0.1 if dtype == "int8" else rng.choice([1.0, 1.0, 0.7, 1.4])
    return _log_probs(rows, vocab, dtype, rng.choice([0, 1, 2, 5, 20, 32]), masked, scale, rng.random() < 0.3, rng.choice([0, 0, 7, 16]))


# ------------------------------------------------------------------------------------------- inputs

def _rows_of(values, pad):
    """`values` as the rows of a tensor that is `pad` elements wider"""
    if not pad:
        return values
    wide = torch.zeros(values.shape[0], values.shape[1] + pad, dtype=values.dtype, device=values.device)
    wide[:, :values.shape[1]] = values
    return wide[:, :values.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = dict(device="cuda", generator=g)
    state = dict(case=case)
    if case["op"] == "norm":
        rows, width, dtype = case["rows"], case["width"], DTYPES[case["dtype"]]
        # a residual stream: a few channels are far larger than the rest
        channel = 0.5 + 20.0 * (torch.rand(width, **dev) > 0.995)
        state["x"] = _rows_of((torch.randn(rows, width, **dev) * channel).to(dtype), case["pad"])
        state["residual"] = _rows_of((torch.randn(rows, width, **dev) * channel).to(dtype), case["pad"]) if case["residual"] else None
        state["weight"] = (1.0 + 0.2 * torch.randn(width, **dev)).to(dtype)
    elif case["op"] == "linear":
        rows, k, n, rank, adapters = (case[f] for f in ("rows", "k", "n", "rank", "adapters"))
        dtype = DTYPES[case["dtype"]]
        adapter_type = torch.bfloat16 if dtype == torch.float32 else dtype

        def codes(r, c):
            return (torch.randn(r, c, **dev) * 32.0).round().clamp_(-127, 127).to(torch.int8)
        state["x"], state["w"] = codes(rows, k), codes(n, k)
        state["x_scale"] = 0.01 + 0.02 * torch.rand(rows, **dev)
        state["w_scale"] = (0.5 + torch.rand(n, **dev)) / (32.0 * math.sqrt(k))
        state["bias"] = torch.randn(n, **dev) * 0.1 if case["bias"] else None
        state["adapters"] = state["ids"] = None
        if rank:
            a = (torch.randn(adapters, rank, k, **dev) / math.sqrt(k)).to(adapter_type)
            b = (torch.randn(adapters, n, rank, **dev) / math.sqrt(rank)).to(adapter_type)
            state["adapters"] = (a, b, 0.5 + torch.rand(adapters, **dev))
            if case["order"] == "mixed":
                ids = torch.randint(0, adapters, (rows,), **dev)
                ids = torch.where(torch.rand(rows, **dev) < 0.1, -1, ids)
            else:
                request = (torch.rand(rows, **dev) < 8.0 / rows).cumsum(0)          # about eight requests
                of_request = torch.randint(0, adapters, (rows + 1,), **dev)
                of_request = torch.where(torch.rand(rows + 1, **dev) < 0.1, -1, of_request)
                ids = of_request[request]
            state["ids"] = ids.to(torch.int32)
    else:
        rows, vocab = case["rows"], case["vocab"]
        if case["dtype"] == "int8":
            logits = (torch.randn(rows, vocab, **dev) * 30.0).round().clamp_(-128, 127).to(torch.int8)
        else:
            logits = torch.randn(rows, vocab, **dev)
            logits *= 1.0 + 3.0 * torch.rand(rows, 1, **dev)                        # sure and unsure rows
            logits = logits.to(DTYPES[case["dtype"]])
        if case["masked"]:
            logits.masked_fill_(torch.rand(rows, vocab, **dev) < case["masked"], -math.inf)
            logits[::50] = -math.inf
        state["logits"] = _rows_of(logits, case["pad"])
        targets = torch.randint(0, vocab, (rows,), **dev)
        state["targets"] = torch.where(torch.rand(rows, **dev) < 0.05, -1, targets)  # some positions are padding
    return state


# ------------------------------------------------------------------------------------------- one pass

def _plain_norm(s):
    # in 64 bits: which of two codes a quotient next to their border rounds to is lost in 32
    h = s["x"].double()
    if s["residual"] is not None:
        h = h + s["residual"].double()
    p = h * s["weight"].double()
    most = p.abs().amax(1, keepdim=True)
    q = torch.where(most > 0, (p * 127.0 / most).round(), 0.0)
    scale = most * (h.square().mean(1, keepdim=True) + EPS).rsqrt() / 127.0
    return dict(values=(q * scale).float(), scale=scale[:, 0].float(), sum=h.to(s["x"].dtype) if s["residual"] is not None else None)


def _plain_linear(s):
    case = s["case"]
    x = s["x"].float()
    y = (x @ s["w"].float().T) * s["w_scale"]
    if case["rank"]:
        a, b, c = s["adapters"]
        adapters, rank, k = a.shape
        of_row = (s["ids"].long()[:, None] == torch.arange(adapters, device="cuda")) * c           # row by adapter
        shrunk = (x @ a.float().reshape(adapters * rank, k).T).reshape(-1, adapters, rank) * of_row[:, :, None]
        y += shrunk.reshape(-1, adapters * rank) @ b.float().permute(0, 2, 1).reshape(adapters * rank, -1)
    y *= s["x_scale"][:, None]
    if s["bias"] is not None:
        y += s["bias"]
    return y.to(DTYPES[case["dtype"]])


def _plain_log_probs(s):
    case = s["case"]
    x = s["logits"].float() + 0.0                                                    # one zero
    vocab = x.shape[1]
    most = x.amax(1, keepdim=True)
    empty = most[:, 0] == -math.inf
    z = (x - most.masked_fill(empty[:, None], 0.0)) * case["scale"]
    e = z.exp()
    total = e.sum(1)
    log_total = total.masked_fill(empty, 1.0).log()
    entropy = log_total - (e * z.masked_fill(e == 0, 0.0)).sum(1) / total.masked_fill(empty, 1.0)
    targets = s["targets"]
    given = z.gather(1, targets.clamp(min=0)[:, None])[:, 0] - log_total
    out = dict(log_probs=given.masked_fill(targets < 0, 0.0), entropy=entropy)
    top = min(max(case["top"], 1 if case["votes"] else 0), vocab)
    if top:
        # order by logit, then by lowest index: one integer whose high half orders as the logit does
        bits = x.view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (vocab - 1 - torch.arange(vocab, device="cuda"))
        ids = vocab - 1 - (key.topk(top, dim=1).values & 0xFFFFFFFF)
        of_top = z.gather(1, ids)
        none = of_top == -math.inf
        ids = ids.masked_fill(none, -1)
        if case["top"]:
            missing = case["top"] - top
            out["top_ids"] = torch.nn.functional.pad(ids.int(), (0, missing), value=-1)
            out["top_log_probs"] = torch.nn.functional.pad(of_top - log_total[:, None], (0, missing), value=-math.inf)
        if case["votes"]:
            out["votes"] = (ids[:, :1] == torch.arange(vocab, device="cuda")).sum(0).int() if vocab <= 64 else \
                torch.zeros(vocab + 1, dtype=torch.int32, device="cuda").index_add_(0, ids[:, 0] + 1, torch.ones_like(ids[:, 0], dtype=torch.int32))[1:]
    return out


def run(state):
    case = state["case"]
    if not own:
        return {"norm": _plain_norm, "linear": _plain_linear, "log_probs": _plain_log_probs}[case["op"]](state)
    import paper_2108_09413_b200 as isc
    if case["op"] == "norm":
        q, scale, total = isc.rms_norm_quant(state["x"], state["weight"], EPS, residual=state["residual"])
        return dict(values=q * scale[:, None], scale=scale, sum=total)
    if case["op"] == "linear":
        return isc.quant_linear(state["x"], state["x_scale"], state["w"], state["w_scale"], bias=state["bias"],
                                adapters=state["adapters"], adapter_ids=state["ids"], out_dtype=DTYPES[case["dtype"]])
    votes = torch.zeros(case["vocab"], dtype=torch.int32, device="cuda") if case["votes"] else None
    given, entropy, ids, alternatives = isc.log_probs(state["logits"], state["targets"], top=case["top"], scale=case["scale"], votes=votes)
    out = dict(log_probs=given, entropy=entropy)
    if case["top"]:
        out.update(top_ids=ids, top_log_probs=alternatives)
    if case["votes"]:
        out["votes"] = votes
    return out


def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4, "int8": 1}[case["dtype"]]
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        # codes count a byte; the values that they stand for are what is compared
        return {"bytes": n * (size + 1 + (2 * size if case["residual"] else 0)) + case["width"] * size + 4 * case["rows"], "flops": 6.0 * n}
    if case["op"] == "linear":
        rows, k, n, rank = case["rows"], case["k"], case["n"], case["rank"]
        used = min(case["adapters"], rows if case["order"] == "mixed" else 8)
        return {"bytes": rows * k + n * k + 4 * (rows + n) + 2 * used * rank * (k + n) + size * rows * n,
                "flops": 2.0 * rows * k * n + 2.0 * rows * rank * (k + n)}
    return {"bytes": case["rows"] * (case["vocab"] * size + 16 + 8 * case["top"]) + (4 * case["vocab"] if case["votes"] else 0),
            "flops": 5.0 * case["rows"] * case["vocab"]}


# ------------------------------------------------------------------------------------------- the definitions in 64 bits

def _exact_norm(s):
    rows, x, r, w = s["x"].shape[0], s["x"], s["residual"], s["weight"].to(torch.float64)
    out = dict(values=[], scale=[], sum=[] if r is not None else None)
    for at in range(0, rows, 2048):
        h = x[at:at + 2048].to(torch.float64)
        if r is not None:
            h = h + r[at:at + 2048].to(torch.float64)
            out["sum"].append(h)
        n = h * w / torch.sqrt((h * h).sum(1, keepdim=True) / h.shape[1] + EPS)
        largest = (h * w).abs().max(1, keepdim=True).values
        step = n.abs().max(1, keepdim=True).values / 127.0
        out["values"].append(torch.where(largest > 0, torch.round(h * w * 127.0 / largest), torch.zeros_like(h)) * step)
        out["scale"].append(step[:, 0])
    return {k: torch.cat(v) if v is not None else None for k, v in out.items()}


def _exact_linear(s):
    x = s["x"].to(torch.float64)
    y = torch.matmul(x, s["w"].to(torch.float64).t()).mul_(s["w_scale"].to(torch.float64))
    if s["adapters"] is not None:
        a, b, c = s["adapters"]
        for i in range(a.shape[0]):
            mine = (s["ids"] == i).nonzero()[:, 0]
            if len(mine):
                y[mine] += float(c[i]) * torch.matmul(torch.matmul(x[mine], a[i].to(torch.float64).t()), b[i].to(torch.float64).t())
    y.mul_(s["x_scale"].to(torch.float64)[:, None])
    return y + s["bias"].to(torch.float64) if s["bias"] is not None else y


def _exact_log_probs(s):
    case, logits, targets = s["case"], s["logits"], s["targets"]
    rows, vocab, top = logits.shape[0], logits.shape[1], case["top"]
    out = dict(log_probs=[], entropy=[])
    if top:
        out.update(top_ids=[], top_log_probs=[])
    votes = torch.zeros(vocab, dtype=torch.int64, device="cuda")
    step = max(1, (1 << 26) // vocab)
    for at in range(0, rows, step):
        l64, t = logits[at:at + step].to(torch.float64), targets[at:at + step]
        log_p = torch.log_softmax(l64 * case["scale"], dim=1)
        empty = (l64 == -math.inf).all(1)
        log_p[empty] = -math.inf
        given = log_p[torch.arange(len(t), device="cuda"), t.clamp(min=0)]
        out["log_probs"].append(torch.where(t < 0, torch.zeros_like(given), given))
        out["entropy"].append(-torch.where(log_p == -math.inf, torch.zeros_like(log_p), log_p.exp() * log_p).sum(1))
        if top or case["votes"]:
            order = torch.sort(l64, dim=1, descending=True, stable=True).indices[:, :max(top, 1)]
            of_top = log_p.gather(1, order)
            order = torch.where(of_top == -math.inf, torch.full_like(order, -1), order)
            votes += torch.bincount(order[:, 0] + 1, minlength=vocab + 1)[1:]
            if top:
                more = torch.full((len(t), max(0, top - vocab)), -1, device="cuda")
                out["top_ids"].append(torch.cat([order, more], 1).int())
                out["top_log_probs"].append(torch.cat([of_top, torch.full(more.shape, -math.inf, dtype=torch.float64, device="cuda")], 1))
    out = {k: torch.cat(v) for k, v in out.items()}
    if case["votes"]:
        out["votes"] = votes.int()
    return out


def exact(case, seed):
    return {"norm": _exact_norm, "linear": _exact_linear, "log_probs": _exact_log_probs}[case["op"]](prepare(case, seed))
