"""The library's operators on device tensors (the last part of include/isc.h) for torch tensors.

Every call checks its arguments, allocates its outputs and enqueues one of the library's operators on `stream` (a torch
stream; the current one of the tensors' device by default).  Outputs belong to that stream.  The operators compute no
gradients: inputs that require one are refused while gradients are enabled.
"""
from __future__ import annotations

import contextlib
import ctypes as C

from .binding import IscError, _check, lib

_ARG = -1


def _refuse(what, why):
    raise IscError(_ARG, f"{what}: {why}")


def _type_code(t):
    import torch
    return {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2, torch.int8: 3}.get(t.dtype)


def _tensors(what, first, *others):
    """Every tensor is on the first one's GPU and needs no gradient."""
    import torch
    if not isinstance(first, torch.Tensor) or not first.is_cuda:
        _refuse(what, "tensors have to be on a GPU")
    grad = torch.is_grad_enabled()
    for t in (first, *others):
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or t.device != first.device:
            _refuse(what, "tensors have to be on one GPU")
        if grad and t.requires_grad:
            _refuse(what, "no gradients are computed")


def _matrix(what, name, t, dtype=None, shape=None):
    """Pitch of a matrix whose rows' elements are adjacent."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        _refuse(what, f"{name} has to be a matrix whose rows' elements are adjacent")
    if dtype is not None and t.dtype != dtype:
        _refuse(what, f"{name} has to be {dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        _refuse(what, f"{name} has to be {tuple(shape)}, not {tuple(t.shape)}")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _vector(what, name, t, dtype, n):
    if t is not None and (t.dim() != 1 or t.shape[0] != n or t.dtype != dtype or not t.is_contiguous()):
        _refuse(what, f"{name} has to be {n} adjacent elements of {dtype}")


def _ptr(t):
    return t.data_ptr() if t is not None else None


@contextlib.contextmanager
def _on(device, stream):
    import torch
    with torch.cuda.device(device), (torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext()):
        yield


def _enqueue(device, stream, call):
    """`call(raw stream)` with the tensors' device and `stream` current."""
    import torch
    if stream is None and device.index == torch.cuda.current_device():
        return call(torch.cuda.current_stream().cuda_stream)
    with _on(device, stream):
        return call(torch.cuda.current_stream(device).cuda_stream)


def rms_norm_quant(x, weight, eps=1e-6, residual=None, sum_out=None, stream=None):
    """(q, scale, sum): root-mean-square norm of x + residual as int8 rows with a scale each; q * scale[:, None] is the
    normed value.  isc_rms_norm_quant.

    x, residual: [rows, width] of bfloat16, float16 or float32, any row pitch; weight: [width] of the same type or float32.
    sum: x + residual in x's type, in `sum_out` where given (x or residual for in place); None without a residual and
    `sum_out`.  q's rows are 16 bytes aligned, as quant_linear takes them.
    """
    import torch
    what = "rms_norm_quant"
    _tensors(what, x, weight, residual, sum_out)
    code = _type_code(x)
    if code is None or code == 3:
        _refuse(what, "x has to be bfloat16, float16 or float32")
    ldx = _matrix(what, "x", x)
    rows, width = x.shape
    ldr = _matrix(what, "residual", residual, x.dtype, x.shape) if residual is not None else 0
    if weight.dtype != torch.float32:
        _vector(what, "weight", weight, x.dtype, width)
    else:
        _vector(what, "weight", weight, torch.float32, width)

    def call(raw):
        total = sum_out
        if total is None and residual is not None:
            total = torch.empty((rows, width), dtype=x.dtype, device=x.device)
        lds = _matrix(what, "sum_out", total, x.dtype, x.shape) if total is not None else 0
        pitch = (width + 15) & ~15
        q = torch.empty((rows, pitch), dtype=torch.int8, device=x.device)
        scale = torch.empty(rows, dtype=torch.float32, device=x.device)
        _check(lib().isc_rms_norm_quant(_ptr(x), ldx, _ptr(residual), ldr, _ptr(weight), _type_code(weight), code, rows, width, eps,
                                        _ptr(total), lds, _ptr(q), pitch, _ptr(scale), raw), "isc_rms_norm_quant")
        return (q if pitch == width else q[:, :width]), scale, total
    return _enqueue(x.device, stream, call)


class _Adapters(C.Structure):
    _fields_ = [("a", C.c_void_p), ("b", C.c_void_p), ("scale", C.c_void_p), ("ids", C.c_void_p), ("type", C.c_int32),
                ("n_adapters", C.c_int32), ("rank", C.c_int32)]


def quant_linear(x, x_scale, w, w_scale, bias=None, adapters=None, adapter_ids=None, out_dtype=None, out=None, stream=None):
    """[rows, n]: x_scale * (w_scale * (x w^T) + scale B (A x)) + bias, A, B and scale those of each row's adapter.
    isc_quant_linear.

    x: [rows, k] int8 with x_scale [rows], as rms_norm_quant gives them; w: [n, k] int8 with w_scale [n]; bias: [n] float32.
    adapters: (A [adapters, rank, k], B [adapters, n, rank], scale [adapters] float32), A and B bfloat16 or float16;
    adapter_ids: [rows] int32, negative for rows without one.  out_dtype: bfloat16 (the default), float16 or float32;
    `out`: where the result goes, any row pitch.
    """
    import torch
    what = "quant_linear"
    a, b, factor = adapters if adapters is not None else (None, None, None)
    _tensors(what, x, x_scale, w, w_scale, bias, a, b, factor, adapter_ids, out)
    ldx, ldw = _matrix(what, "x", x, torch.int8), _matrix(what, "w", w, torch.int8)
    rows, k = x.shape
    n = w.shape[0]
    if w.shape[1] != k:
        _refuse(what, f"w has {w.shape[1]} columns, x {k}")
    _vector(what, "x_scale", x_scale, torch.float32, rows)
    _vector(what, "w_scale", w_scale, torch.float32, n)
    _vector(what, "bias", bias, torch.float32, n)
    dtype = out.dtype if out is not None else out_dtype if out_dtype is not None else torch.bfloat16
    if out is not None and out_dtype not in (None, out.dtype):
        _refuse(what, "out is not of out_dtype")
    code = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}.get(dtype)
    if code is None:
        _refuse(what, "the result is bfloat16, float16 or float32")
    parts, space = None, 0
    if adapters is not None:
        if a.dim() != 3 or b.dim() != 3 or a.dtype not in (torch.bfloat16, torch.float16) or b.dtype != a.dtype:
            _refuse(what, "adapters are bfloat16 or float16 [adapters, rank, k] and [adapters, n, rank]")
        count, rank = a.shape[0], a.shape[1]
        if a.shape[2] != k or tuple(b.shape) != (count, n, rank) or not a.is_contiguous() or not b.is_contiguous():
            _refuse(what, f"adapters have to be {(count, rank, k)} and {(count, n, rank)} without gaps")
        _vector(what, "the adapters' scale", factor, torch.float32, count)
        if adapter_ids is None:
            _refuse(what, "adapters need adapter_ids")
        _vector(what, "adapter_ids", adapter_ids, torch.int32, rows)
        if count:
            parts = _Adapters(_ptr(a), _ptr(b), _ptr(factor), _ptr(adapter_ids), _type_code(a), count, rank)
            space = ((rank + 15) // 16) * 64 * rows

    def call(raw):
        y = torch.empty((rows, n), dtype=dtype, device=x.device) if out is None else out
        ldy = _matrix(what, "out", y, dtype, (rows, n))
        work = torch.empty(space, dtype=torch.uint8, device=x.device) if space else None
        _check(lib().isc_quant_linear(_ptr(x), ldx, _ptr(x_scale), rows, _ptr(w), ldw, _ptr(w_scale), k, n, _ptr(bias),
                                      C.addressof(parts) if parts is not None else None, _ptr(y), ldy, code, _ptr(work), space, raw),
               "isc_quant_linear")
        return y
    return _enqueue(x.device, stream, call)


def log_probs(logits, targets=None, top=0, scale=1.0, votes=None, entropy=True, stream=None):
    """(log_probs, entropy, top_ids, top_log_probs) of rows of logits; None for what is not asked for.  isc_log_probs.

    logits: [rows, vocab] of bfloat16, float16, float32 or int8, any row pitch, minus infinity for masked tokens; the
    probabilities are softmax(scale * logits).  targets: [rows] int64, negative for positions without one (their log
    probability is 0).  top: the number of alternatives, at most 32.  votes: [vocab] int32, to which 1 is added at every
    row's first alternative, as certify_decide and predict_decide take them (on the host).
    """
    import torch
    what = "log_probs"
    _tensors(what, logits, targets, votes)
    code = _type_code(logits)
    if code is None:
        _refuse(what, "logits have to be bfloat16, float16, float32 or int8")
    ld = _matrix(what, "logits", logits)
    rows, vocab = logits.shape
    _vector(what, "targets", targets, torch.int64, rows)
    _vector(what, "votes", votes, torch.int32, vocab)

    def call(raw):
        given = torch.empty(rows, dtype=torch.float32, device=logits.device) if targets is not None else None
        h = torch.empty(rows, dtype=torch.float32, device=logits.device) if entropy else None
        ids = torch.empty((rows, top), dtype=torch.int32, device=logits.device) if top > 0 else None
        alternatives = torch.empty((rows, top), dtype=torch.float32, device=logits.device) if top > 0 else None
        _check(lib().isc_log_probs(_ptr(logits), ld, code, rows, vocab, scale, _ptr(targets), top, _ptr(given), _ptr(h), _ptr(ids),
                                   _ptr(alternatives), _ptr(votes), raw), "isc_log_probs")
        return given, h, ids, alternatives
    return _enqueue(logits.device, stream, call)
