"""The library's operators on device tensors (the last part of include/isc.h) for torch tensors.

Every call checks its arguments, allocates its outputs and enqueues one of the library's operators on `stream` (a torch
stream; the current one of the tensors' device by default).  Outputs belong to that stream.  Inputs may be dropped after a
call on a side stream, whichever stream they belong to; on a device's default stream, as with torch's own operators, those
of a side stream need `record_stream` first.  The operators compute no gradients: inputs that require one are refused
while gradients are enabled, and inputs with a tangent (forward-mode differentiation) always.
"""
from __future__ import annotations

import ctypes as C

from .binding import IscError, lib

_ARG = -1
_torch = _forward = None      # imported with the first call: the rest of the package works without them
_types = {}


def _start():
    global _torch, _forward
    import torch
    from torch.autograd import forward_ad as _forward
    _types.update({torch.bfloat16: 0, torch.float16: 1, torch.float32: 2, torch.int8: 3})
    _torch = torch            # last: another thread that finds it set looks into _types
    return torch


def _refuse(what, why):
    raise IscError(_ARG, f"{what}: {why}")


def _same_device(what, tensors):
    """The one GPU that all of the tensors (or None) are on; none of them may need a gradient or have a tangent."""
    torch = _torch
    first = tensors[0]
    if not isinstance(first, torch.Tensor) or not first.is_cuda:
        _refuse(what, "tensors have to be on a GPU")
    device, grad, dual = first.device, torch.is_grad_enabled(), _forward._current_level >= 0
    for t in tensors:
        if t is not None:
            if not isinstance(t, torch.Tensor) or t.device != device:
                _refuse(what, "tensors have to be on one GPU")
            if grad and t.requires_grad or dual and _forward.unpack_dual(t).tangent is not None:
                _refuse(what, "no gradients are computed")
    return device


def _pitch(what, name, t, dtype=None, shape=None):
    """Pitch of a matrix whose rows' elements are adjacent."""
    own = t.shape
    if len(own) != 2 or (own[1] > 1 and t.stride(1) != 1):
        _refuse(what, f"{name} has to be a matrix whose rows' elements are adjacent")
    if dtype is not None and t.dtype != dtype:
        _refuse(what, f"{name} has to be {dtype}")
    if shape is not None and own != shape:
        _refuse(what, f"{name} has to be {tuple(shape)}, not {tuple(own)}")
    ld = t.stride(0)
    return ld if own[0] > 1 or ld > own[1] else own[1]


def _vector(what, name, t, dtype, n):
    if t is not None and (t.dtype != dtype or t.shape != (n,) or not t.is_contiguous()):
        _refuse(what, f"{name} has to be {n} adjacent elements of {dtype}")


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _empty(shape, dtype, device):
    # (torch.empty takes 0.9 us more)
    return _torch.empty_strided(shape, (shape[1], 1) if len(shape) == 2 else (1,), dtype=dtype, device=device)


def _enqueue(what, device, stream, call, tensors=()):
    """`call(raw stream)`, a status, with the tensors' device and `stream` (None: the current one) current.  The memory of `tensors`
    (or None), which may be another stream's, is not given to others before a `stream` that was given, or is not the default one, has
    used it."""
    torch = _torch
    index = device.index
    if stream is not None and stream.device_index != index:
        _refuse(what, "the stream belongs to another device than the tensors")
    if stream is None and index == torch.cuda.current_device():
        raw = torch._C._cuda_getCurrentRawStream(index)
        rc = call(raw)
    else:
        with torch.cuda.device(index), torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(index)):
            raw = torch._C._cuda_getCurrentRawStream(index)
            rc = call(raw)
    if raw or stream is not None:
        if stream is None:
            stream = torch.cuda.current_stream(index)
        for t in tensors:
            if t is not None and t.numel():
                t.record_stream(stream)
    if rc != 0:
        raise IscError(rc, what)


def rms_norm_quant(x, weight, eps=1e-6, residual=None, sum_out=None, stream=None):
    """(q, scale, sum): root-mean-square norm of x + residual as int8 rows with a scale each; q * scale[:, None] is the
    normed value.  isc_rms_norm_quant.

    x, residual: [rows, width] of bfloat16, float16 or float32, any row pitch; weight: [width] of the same type or float32.
    sum: x + residual in x's type, in `sum_out` where given (x or residual for in place); None without a residual and
    `sum_out`.  q's rows are 16 bytes aligned, as quant_linear takes them.
    """
    torch = _torch or _start()
    what = "rms_norm_quant"
    given = (x, weight, residual, sum_out)
    if weight is None:
        _refuse(what, "the weight is missing")
    device = _same_device(what, given)
    dtype, shape = x.dtype, x.shape
    code = _types.get(dtype, 3)
    if code == 3:
        _refuse(what, "x has to be bfloat16, float16 or float32")
    ldx = _pitch(what, "x", x)
    rows, width = shape
    ldr = _pitch(what, "residual", residual, dtype, shape) if residual is not None else 0
    wide = weight.dtype == torch.float32
    _vector(what, "weight", weight, torch.float32 if wide else dtype, width)
    if sum_out is not None:
        _pitch(what, "sum_out", sum_out, dtype, shape)
    pitch = (width + 15) & ~15
    q = scale = total = None

    def call(raw):
        nonlocal q, scale, total
        total = _empty(shape, dtype, device) if sum_out is None and residual is not None else sum_out
        q = _empty((rows, pitch), torch.int8, device)
        scale = _empty((rows,), torch.float32, device)
        return lib().isc_rms_norm_quant(x.data_ptr(), ldx, _ptr(residual), ldr, weight.data_ptr(), 2 if wide else code, code, rows, width, eps,
                                        _ptr(total), total.stride(0) if total is not None and rows > 1 else width, q.data_ptr(), pitch, scale.data_ptr(), raw)
    _enqueue("isc_rms_norm_quant", device, stream, call, given)
    return (q if pitch == width else q[:, :width]), scale, total


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
    torch = _torch or _start()
    what = "quant_linear"
    a = b = factor = None
    if adapters is not None:
        adapters = tuple(adapters)
        if len(adapters) != 3 or any(t is None for t in adapters):
            _refuse(what, "adapters are three tensors")
        a, b, factor = adapters
    given = (x, x_scale, w, w_scale, bias, a, b, factor, adapter_ids, out)
    if x_scale is None or w is None or w_scale is None:
        _refuse(what, "the scales and w are needed")
    device = _same_device(what, given)
    ldx, ldw = _pitch(what, "x", x, torch.int8), _pitch(what, "w", w, torch.int8)
    rows, k = x.shape
    n = w.shape[0]
    if w.shape[1] != k:
        _refuse(what, f"w has {w.shape[1]} columns, x {k}")
    _vector(what, "x_scale", x_scale, torch.float32, rows)
    _vector(what, "w_scale", w_scale, torch.float32, n)
    _vector(what, "bias", bias, torch.float32, n)
    dtype = out.dtype if out is not None else out_dtype if out_dtype is not None else torch.bfloat16
    if out is not None and out_dtype not in (None, dtype):
        _refuse(what, "out is not of out_dtype")
    code = _types.get(dtype, 3)
    if code == 3:
        _refuse(what, "the result is bfloat16, float16 or float32")
    if out is not None:
        _pitch(what, "out", out, dtype, (rows, n))
    parts, space = None, 0
    if adapters is not None:
        kind = _types.get(a.dtype, 3)
        if kind > 1 or b.dtype != a.dtype or a.dim() != 3:
            _refuse(what, "adapters are bfloat16 or float16 [adapters, rank, k] and [adapters, n, rank]")
        count, rank, depth = a.shape
        if depth != k or b.shape != (count, n, rank) or not a.is_contiguous() or not b.is_contiguous():
            _refuse(what, f"adapters have to be {(count, rank, k)} and {(count, n, rank)} without gaps")
        _vector(what, "the adapters' scale", factor, torch.float32, count)
        if adapter_ids is None:
            _refuse(what, "adapters need adapter_ids")
        _vector(what, "adapter_ids", adapter_ids, torch.int32, rows)
        if count:
            parts = _Adapters(a.data_ptr(), b.data_ptr(), factor.data_ptr(), adapter_ids.data_ptr(), kind, count, rank)
            space = ((rank + 15) // 16) * 64 * rows
    y = out

    def call(raw):
        nonlocal y
        if y is None:
            y = _empty((rows, n), dtype, device)
        work = _empty((space,), torch.uint8, device) if space else None
        factors = x_scale
        if adapters is not None and parts is None:      # no adapter at all: every id that is not negative is too large
            factors = torch.where(adapter_ids < 0, x_scale, float("nan"))
        return lib().isc_quant_linear(x.data_ptr(), ldx, factors.data_ptr(), rows, w.data_ptr(), ldw, w_scale.data_ptr(), k, n, _ptr(bias),
                                      C.addressof(parts) if parts is not None else None, y.data_ptr(), y.stride(0) if rows > 1 else n, code,
                                      _ptr(work), space, raw)
    _enqueue("isc_quant_linear", device, stream, call, given)
    return y


def log_probs(logits, targets=None, top=0, scale=1.0, votes=None, entropy=True, stream=None):
    """(log_probs, entropy, top_ids, top_log_probs) of rows of logits; None for what is not asked for.  isc_log_probs.

    logits: [rows, vocab] of bfloat16, float16, float32 or int8, any row pitch, minus infinity for masked tokens; the
    probabilities are softmax(scale * logits).  targets: [rows] int64, negative for positions without one (their log
    probability is 0).  top: the number of alternatives, at most 32.  votes: [vocab] int32, to which 1 is added at every
    row's first alternative, as certify_decide and predict_decide take them (on the host).
    """
    torch = _torch or _start()
    what = "log_probs"
    device = _same_device(what, (logits, targets, votes))
    code = _types.get(logits.dtype)
    if code is None:
        _refuse(what, "logits have to be bfloat16, float16, float32 or int8")
    ld = _pitch(what, "logits", logits)
    rows, vocab = logits.shape
    if not 0 <= top <= 32:
        _refuse(what, "top is 0 to 32")
    _vector(what, "targets", targets, torch.int64, rows)
    _vector(what, "votes", votes, torch.int32, vocab)
    given = h = ids = alternatives = None

    def call(raw):
        nonlocal given, h, ids, alternatives
        numbers = torch.float32
        if targets is not None:
            given = _empty((rows,), numbers, device)
        if entropy:
            h = _empty((rows,), numbers, device)
        if top > 0:
            ids = _empty((rows, top), torch.int32, device)
            alternatives = _empty((rows, top), numbers, device)
        return lib().isc_log_probs(logits.data_ptr(), ld, code, rows, vocab, scale, _ptr(targets), top, _ptr(given), _ptr(h), _ptr(ids),
                                   _ptr(alternatives), _ptr(votes), raw)
    _enqueue("isc_log_probs", device, stream, call, (logits, targets, votes))
    return given, h, ids, alternatives
