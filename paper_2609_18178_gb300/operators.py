"""The operators around a training step's output head (include/apc.h): the
root-mean-square norm in front of it with its gradient, 8-bit quantization with
block scales, the product of such operands, and distillation from a teacher's
top logits.  Argument marshalling only, as in the package's other entry points:

* :func:`rms_norm`, :func:`rms_norm_fp8`, :func:`rms_norm_grad` ->
  ``apc_rms_norm``, ``apc_rms_norm_fp8``, ``apc_rms_norm_grad``
* :func:`quantize_fp8` -> ``apc_quantize_fp8``
* :func:`matmul_fp8` -> ``apc_matmul_fp8``
* :func:`distill_loss`, :func:`distill_grad`, :func:`distill_loss_grad` ->
  ``apc_distill_loss``, ``apc_distill_grad``, ``apc_distill_loss_grad``

An 8-bit matrix is a pair of tensors: the data, ``[rows, cols]`` of
``torch.float8_e4m3fn`` or ``torch.float8_e5m2`` whose rows start at multiples
of 16 bytes, and the scales, fp32 ``[ceil(cols/128), rows]`` (one for every 128
values of a row) or ``[ceil(cols/128), ceil(rows/128)]`` (square blocks).

``stream`` is a ``torch.cuda.Stream`` or a handle, the current stream if not
given; outputs that a call allocates are memory of that stream.
"""
from __future__ import annotations

import ctypes
from struct import Struct

import torch

__all__ = ["quantize_fp8", "matmul_fp8", "rms_norm", "rms_norm_fp8", "rms_norm_grad", "rms_norm_grad_workspace", "distill_loss",
           "distill_grad", "distill_loss_grad"]

BLOCK = 128
_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_FORMAT = {torch.float8_e4m3fn: 0, torch.float8_e5m2: 1}
_INDEX = {torch.int32: 0, torch.int64: 1}


class _Fp8Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("pitch", ctypes.c_int64),
                ("scale_pitch", ctypes.c_int64), ("format", ctypes.c_uint32), ("block_rows", ctypes.c_uint32)]


class _Distill(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("logits", "ids", "teacher", "teacher_lse", "labels")] + \
               [(n, ctypes.c_int64) for n in ("rows", "vocab", "k", "pitch", "ids_pitch", "teacher_pitch")] + \
               [(n, ctypes.c_uint32) for n in ("dtype", "ids_dtype", "teacher_dtype", "labels_dtype")] + \
               [(n, ctypes.c_double) for n in ("temperature", "kd_weight", "label_weight")]


# The structures of a call as bytes, packed in one step (a ctypes structure takes 0.4 us more)
_pack_fp8, _pack_norm, _pack_norm_grad = (Struct(f).pack for f in ("2P2q2I", "4P5q2Id", "5P5q2I"))

_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # the handle without a Stream object around it
# Workspaces straight from torch's allocator: 0.8 us of a call's host time where torch.empty takes 5
_raw_alloc = getattr(torch._C, "_cuda_cudaCachingAllocator_raw_alloc", None)
_raw_free = getattr(torch._C, "_cuda_cudaCachingAllocator_raw_delete", None)
_lib = None

# The checks below read each attribute of a tensor once (0.1 us apiece): a call of
# small size is bound by them.


def _library():
    global _lib
    if _lib is None:
        from . import library
        _lib = library()
    return _lib


def _stream(stream, device: int) -> int:
    if stream is None and _raw_stream is not None:
        return _raw_stream(device)
    from . import _stream as handle
    return handle(stream)


def _elsewhere(x, name: str, device: int):
    if not x.is_cuda:
        raise ValueError("%s is not on a CUDA device" % name)
    raise ValueError("%s is on cuda:%d but the current device is cuda:%d (use torch.cuda.device(...))"
                     % (name, x.get_device(), device))


def _matrix(x, name: str, kinds, device: int):
    """Code of the type, rows, columns and pitch of a two-dimensional tensor on
    the current device whose type is one of `kinds`."""
    if x.get_device() != device:
        _elsewhere(x, name, device)
    kind = kinds.get(x.dtype)
    if kind is None:
        raise ValueError("%s has type %s" % (name, x.dtype))
    if x.dim() != 2:
        raise ValueError("%s has %d dimensions, expected 2" % (name, x.dim()))
    r, c = x.shape
    pitch, step = x.stride()
    if step != 1 and c > 1:
        raise ValueError("%s: neighbours in a row are %d elements apart, expected 1" % (name, step))
    return kind, r, c, pitch if r > 1 else c


def _sized(x, name: str, kinds, device: int, rows: int, cols: int):
    """Code of the type and pitch of a matrix of the given size."""
    kind, r, c, pitch = _matrix(x, name, kinds, device)
    if r != rows or c != cols:
        raise ValueError("%s is %d x %d, expected %d x %d" % (name, r, c, rows, cols))
    return kind, pitch


def _vector(x, name: str, kinds, device: int, n: int) -> int:
    if x is None:
        raise ValueError("%s is None" % name)
    if x.get_device() != device:
        _elsewhere(x, name, device)
    if x.dtype not in kinds:
        raise ValueError("%s has type %s" % (name, x.dtype))
    if x.numel() != n or not x.is_contiguous():
        raise ValueError("%s: expected %d contiguous elements, got %s" % (name, n, tuple(x.shape)))
    return x.data_ptr()


_F32 = {torch.float32: 0}


def _blocks(n: int) -> int:
    return (n + BLOCK - 1) // BLOCK


def _fp8(data, scale, name: str, device: int, block=None):
    """The C structure of an 8-bit matrix, its rows, columns and format; block: its
    rows per scale, found from the scale's shape if not given."""
    kind, r, c, pitch = _matrix(data, name, _FORMAT, device)
    _, lines, width, scale_pitch = _matrix(scale, name + "_scale", _F32, device)
    if block is None:
        block = 1 if width == r else BLOCK
    if lines != (c + BLOCK - 1) // BLOCK or width != (r if block == 1 else -(-r // block)):
        raise ValueError("%s_scale is %d x %d: expected %d x %d, or %d columns for square blocks"
                         % (name, lines, width, _blocks(c), r, _blocks(r)))
    return _pack_fp8(data.data_ptr(), scale.data_ptr(), pitch, scale_pitch, kind, block), r, c, kind


def _empty(shape, dtype, like, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    from . import _empty as empty
    return empty(shape, dtype, like.device, stream)


class _Workspace:
    """So many bytes of memory of a stream while a call is made: what is enqueued
    there later may have them again, but only behind the call's kernels."""

    def __init__(self, size: int, stream, handle: int):
        if _raw_alloc is None:
            from . import _empty as empty
            self.held = empty((size + 7) // 8, torch.int64, torch.device("cuda", _current_device()), stream)
            self.at = self.held.data_ptr()
        else:
            self.held = None
            self.at = _raw_alloc(size, handle)

    def __enter__(self) -> int:
        return self.at

    def __exit__(self, *error):
        if self.held is None:
            _raw_free(self.at)


def _fp8_empty(rows: int, cols: int, block: int, dtype, like, stream):
    return (_empty((rows, (cols + 15) // 16 * 16), dtype, like, stream)[:, :cols],
            _empty((_blocks(cols), -(-rows // block)), torch.float32, like, stream))


def _check(status: int) -> None:
    if status:
        from . import _check as check
        check(status)


def quantize_fp8(x, block_rows: int = 1, dtype=torch.float8_e4m3fn, transposed: bool = False, out=None, stream=None):
    """Enqueue the quantization of ``x`` (``[rows, cols]``, fp32, bf16 or fp16,
    any row pitch) to 8 bits with a power-of-two scale for every 128 values of
    a row (``block_rows=1``) or every 128 x 128 block (``block_rows=128``).

    Returns ``(data, scale)`` or, with ``transposed``, ``(data, scale, data_t,
    scale_t)`` with the transpose quantized from the same reading of ``x``,
    its blocks along its own rows.  ``out`` takes tensors of those shapes."""
    lib = _library()
    device = _current_device()
    kind, r, c, pitch = _matrix(x, "x", _DTYPE, device)
    if dtype not in _FORMAT:
        raise ValueError("dtype %s is not an 8-bit floating type" % dtype)
    if block_rows not in (1, BLOCK):
        raise ValueError("block_rows %r is neither 1 nor %d" % (block_rows, BLOCK))
    if out is None:
        out = _fp8_empty(r, c, block_rows, dtype, x, stream)
        if transposed:
            out += _fp8_empty(c, r, block_rows, dtype, x, stream)
    elif len(out) != (4 if transposed else 2):
        raise ValueError("out has %d tensors, expected %d" % (len(out), 4 if transposed else 2))
    q, qr, qc, fmt = _fp8(out[0], out[1], "q", device, block_rows)
    if qr != r or qc != c or fmt != _FORMAT[dtype]:
        raise ValueError("out: q is %d x %d of %s, expected %d x %d of %s" % (qr, qc, out[0].dtype, r, c, dtype))
    qt = None
    if transposed:
        qt, qr, qc, fmt = _fp8(out[2], out[3], "qt", device, block_rows)
        if qr != c or qc != r or fmt != _FORMAT[dtype]:
            raise ValueError("out: qt is %d x %d of %s, expected %d x %d of %s" % (qr, qc, out[2].dtype, c, r, dtype))
    _check(lib.apc_quantize_fp8(x.data_ptr(), r, c, pitch, kind, q, qt, _stream(stream, device)))
    return tuple(out)


def _weight(x, name: str, device: int, n: int) -> int:
    """Code of the type of a vector of n values (checked as by _vector)."""
    _vector(x, name, _DTYPE, device, n)
    return _DTYPE[x.dtype]


def _norm(x, weight, eps, residual, sum, rstd, device, stream):
    """The C structure of a norm, its rows and columns, its sum (x itself
    without a residual) and rstd."""
    kind, r, c, pitch = _matrix(x, "x", _DTYPE, device)
    wkind = _weight(weight, "weight", device, c)
    if rstd is None:
        rstd = _empty((r,), torch.float32, x, stream)
    else:
        _vector(rstd, "rstd", _F32, device, r)
    if residual is None:
        if sum is not None:
            raise ValueError("sum without a residual")
        return _pack_norm(x.data_ptr(), 0, weight.data_ptr(), 0, r, c, pitch, 0, 0, kind, wkind, eps), r, c, x, rstd
    same = {x.dtype: kind}
    rpitch = _sized(residual, "residual", same, device, r, c)[1]
    if sum is None:
        sum = _empty((r, c), x.dtype, x, stream)
    spitch = _sized(sum, "sum", same, device, r, c)[1]
    return _pack_norm(x.data_ptr(), residual.data_ptr(), weight.data_ptr(), sum.data_ptr(), r, c, pitch, rpitch, spitch, kind,
                      wkind, eps), r, c, sum, rstd


def rms_norm(x, weight, *, eps=1e-6, residual=None, out=None, sum=None, rstd=None, stream=None):
    """Enqueue the root-mean-square norm of the rows of ``x`` (``[rows,
    cols]``, fp32, bf16 or fp16, any row pitch) with ``weight`` (``[cols]``, of
    any of these types), after the addition of ``residual``.

    Returns ``(out, sum, rstd)``: the normalised rows, ``x + residual`` in its
    type (``x`` itself without a residual) and 1/rms of its rows (fp32
    ``[rows]``), the last two for :func:`rms_norm_grad`.  ``sum`` may be ``x`` or
    ``residual`` itself."""
    lib = _library()
    device = _current_device()
    d, r, c, sum, rstd = _norm(x, weight, eps, residual, sum, rstd, device, stream)
    if out is None:
        out = _empty((r, c), x.dtype, x, stream)
    pitch = _sized(out, "out", {x.dtype: 0}, device, r, c)[1]
    _check(lib.apc_rms_norm(d, out.data_ptr(), pitch, rstd.data_ptr(), _stream(stream, device)))
    return out, sum, rstd


def rms_norm_fp8(x, weight, *, eps=1e-6, residual=None, dtype=torch.float8_e4m3fn, transposed: bool = False, out=None, sum=None,
                 rstd=None, stream=None):
    """Enqueue :func:`rms_norm` with its output in 8 bits, as
    :func:`quantize_fp8` makes it with ``block_rows=1``, from the unrounded
    values.

    Returns ``(data, scale, sum, rstd)`` or, with ``transposed``, ``(data, scale,
    data_t, scale_t, sum, rstd)``.  ``out`` takes the tensors in front of
    ``sum``."""
    lib = _library()
    device = _current_device()
    if dtype not in _FORMAT:
        raise ValueError("dtype %s is not an 8-bit floating type" % dtype)
    d, r, c, sum, rstd = _norm(x, weight, eps, residual, sum, rstd, device, stream)
    if out is None:
        out = _fp8_empty(r, c, 1, dtype, x, stream)
        if transposed:
            out += _fp8_empty(c, r, 1, dtype, x, stream)
    elif len(out) != (4 if transposed else 2):
        raise ValueError("out has %d tensors, expected %d" % (len(out), 4 if transposed else 2))
    q, qr, qc, fmt = _fp8(out[0], out[1], "q", device, 1)
    if qr != r or qc != c or fmt != _FORMAT[dtype]:
        raise ValueError("out: q is %d x %d of %s, expected %d x %d of %s" % (qr, qc, out[0].dtype, r, c, dtype))
    qt = None
    if transposed:
        qt, qr, qc, fmt = _fp8(out[2], out[3], "qt", device, 1)
        if qr != c or qc != r or fmt != _FORMAT[dtype]:
            raise ValueError("out: qt is %d x %d of %s, expected %d x %d of %s" % (qr, qc, out[2].dtype, c, r, dtype))
    _check(lib.apc_rms_norm_fp8(d, q, qt, rstd.data_ptr(), _stream(stream, device)))
    return *out, sum, rstd


def rms_norm_grad(dout, x, weight, rstd, *, dresidual=None, out=None, dweight=None, weight_grad: bool = True, workspace=None,
                  stream=None):
    """Enqueue the gradient of :func:`rms_norm` or :func:`rms_norm_fp8`:
    ``dout`` (``[rows, cols]`` of ``x``'s type) is the output's, ``x`` the norm's
    ``sum``, ``rstd`` its statistics, ``dresidual`` the gradient that reaches
    ``sum`` otherwise.

    Returns ``(dx, dweight)``: the gradient of ``x`` and of the residual alike,
    in ``x``'s type or in ``out`` (which may be ``dout`` or ``dresidual`` itself),
    and the weight's, in its type or in ``dweight``'s; None without
    ``weight_grad``.  ``workspace``: fp32, for a caller that keeps its own, which
    no other call may use at the same time; ``rms_norm_grad_workspace(rows,
    cols)`` elements, none for few rows."""
    lib = _library()
    device = _current_device()
    kind, r, c, pitch = _matrix(x, "x", _DTYPE, device)
    same = {x.dtype: kind}
    dpitch = _sized(dout, "dout", same, device, r, c)[1]
    rpitch = 0 if dresidual is None else _sized(dresidual, "dresidual", same, device, r, c)[1]
    d = _pack_norm_grad(dout.data_ptr(), x.data_ptr(), weight.data_ptr(), 0 if dresidual is None else dresidual.data_ptr(),
                        _vector(rstd, "rstd", _F32, device, r), r, c, dpitch, pitch, rpitch, kind, _weight(weight, "weight", device, c))
    if out is None:
        out = _empty((r, c), x.dtype, x, stream)
    opitch = _sized(out, "out", same, device, r, c)[1]
    handle = _stream(stream, device)
    if not weight_grad:
        if dweight is not None:
            raise ValueError("dweight without weight_grad")
        _check(lib.apc_rms_norm_grad(d, out.data_ptr(), opitch, None, 0, None, handle))
        return out, None
    if dweight is None:
        dweight = _empty((c,), weight.dtype, weight, stream)
    given = d, out.data_ptr(), opitch, dweight.data_ptr(), _weight(dweight, "dweight", device, c)
    size = lib.apc_rms_norm_grad_workspace(r, c)
    if not size:
        _check(lib.apc_rms_norm_grad(*given, None, handle))
    elif workspace is not None:
        if workspace.numel() > size // 4 and workspace.is_contiguous():
            workspace = workspace.view(-1)[:size // 4]
        _check(lib.apc_rms_norm_grad(*given, _vector(workspace, "workspace", _F32, device, size // 4), handle))
    else:
        with _Workspace(size, stream, handle) as work:
            _check(lib.apc_rms_norm_grad(*given, work, handle))
    return out, dweight


def rms_norm_grad_workspace(rows: int, cols: int) -> int:
    """Elements of :func:`rms_norm_grad`'s workspace."""
    return _library().apc_rms_norm_grad_workspace(rows, cols) // 4


def matmul_fp8(a, a_scale, b, b_scale, out=None, out_dtype=torch.bfloat16, stream=None):
    """Enqueue ``out = a b^T`` for 8-bit ``a`` (``[m, k]``) and ``b`` (``[n,
    k]``) with their scales.  Returns ``out`` (``[m, n]`` of ``out_dtype``:
    fp32, bf16 or fp16), or fills the one given, of any row pitch."""
    lib = _library()
    device = _current_device()
    p, m, k, _ = _fp8(a, a_scale, "a", device)
    q, n, kb, _ = _fp8(b, b_scale, "b", device)
    if kb != k:
        raise ValueError("a has %d columns and b has %d" % (k, kb))
    if out is None:
        out = _empty((m, n), out_dtype, a, stream)
    kind, pitch = _sized(out, "out", _DTYPE, device, m, n)
    _check(lib.apc_matmul_fp8(p, q, m, n, k, out.data_ptr(), pitch, kind, _stream(stream, device)))
    return out


def _distill(logits, ids, teacher, temperature, kd_weight, teacher_lse, labels, label_weight, device) -> _Distill:
    kind, rows, vocab, pitch = _matrix(logits, "logits", _DTYPE, device)
    ids_kind, ids_rows, k, ids_pitch = _matrix(ids, "ids", _INDEX, device)
    teacher_kind, teacher_pitch = _sized(teacher, "teacher", _DTYPE, device, rows, k)
    if ids_rows != rows:
        raise ValueError("ids has %d rows and the logits %d" % (ids_rows, rows))
    return _Distill(
        logits.data_ptr(), ids.data_ptr(), teacher.data_ptr(),
        None if teacher_lse is None else _vector(teacher_lse, "teacher_lse", _F32, device, rows),
        None if labels is None else _vector(labels, "labels", _INDEX, device, rows),
        rows, vocab, k, pitch, ids_pitch, teacher_pitch, kind, ids_kind, teacher_kind,
        0 if labels is None else _INDEX[labels.dtype], temperature, kd_weight, label_weight)


def _lse_room(lse, logits, labels, device, rows, stream):
    n = 1 if labels is None else 2
    if lse is None:
        lse = _empty((n, rows), torch.float32, logits, stream)
    return lse, _vector(lse, "lse", _F32, device, n * rows)


def _dlogits_room(out, logits, device, d, stream):
    if out is None:
        out = _empty((d.rows, d.vocab), logits.dtype, logits, stream)
    return out, _sized(out, "out", {logits.dtype: 0}, device, d.rows, d.vocab)[1]


def distill_loss(logits, ids, teacher, *, temperature=1.0, kd_weight=1.0, teacher_lse=None, labels=None,
                 label_weight=0.0, loss=None, lse=None, stream=None):
    """Enqueue each row's distillation loss: ``kd_weight * temperature^2`` times
    the divergence from the teacher's ``k`` largest logits (``teacher``, fp32,
    bf16 or fp16, at the vocabulary's places ``ids``, int32 or int64; ``[rows,
    k]``) to the student's softmax of ``logits`` (``[rows, vocab]``), plus
    ``label_weight`` times the cross entropy of ``labels`` (``[rows]``).

    The teacher is normalised over the row's entries or, with ``teacher_lse``
    (fp32 ``[rows]``: logsumexp of all its logits over the temperature), over
    its whole vocabulary.  Entries whose id lies outside the vocabulary or whose
    logit is -inf do not count, nor do labels outside it.  A row with no logit
    above -1e30 is masked whole: loss 0, gradient 0.

    Returns ``(loss, lse)``: fp32 ``[rows]``, and the statistics that
    :func:`distill_grad` takes, fp32 ``[1 or, with labels, 2, rows]``."""
    lib = _library()
    device = _current_device()
    d = _distill(logits, ids, teacher, temperature, kd_weight, teacher_lse, labels, label_weight, device)
    if loss is None:
        loss = _empty((d.rows,), torch.float32, logits, stream)
    lse, at = _lse_room(lse, logits, labels, device, d.rows, stream)
    _check(lib.apc_distill_loss(ctypes.byref(d), _vector(loss, "loss", _F32, device, d.rows), at, _stream(stream, device)))
    return loss, lse


def distill_grad(logits, ids, teacher, lse, grad_loss, *, temperature=1.0, kd_weight=1.0, teacher_lse=None, labels=None,
                 label_weight=0.0, out=None, stream=None):
    """Enqueue the gradient of the logits: ``grad_loss[t]`` (fp32 ``[rows]``)
    times the gradient of row t's :func:`distill_loss`, whose ``lse`` is given.
    Rows with a ``grad_loss`` of 0 get zeros.  Returns it in the logits' type,
    or in ``out``, which may be ``logits`` itself."""
    lib = _library()
    device = _current_device()
    d = _distill(logits, ids, teacher, temperature, kd_weight, teacher_lse, labels, label_weight, device)
    at = _vector(lse, "lse", _F32, device, (1 if labels is None else 2) * d.rows)
    out, pitch = _dlogits_room(out, logits, device, d, stream)
    _check(lib.apc_distill_grad(ctypes.byref(d), at, _vector(grad_loss, "grad_loss", _F32, device, d.rows), out.data_ptr(),
                                pitch, _stream(stream, device)))
    return out


def distill_loss_grad(logits, ids, teacher, grad_loss, *, temperature=1.0, kd_weight=1.0, teacher_lse=None, labels=None,
                      label_weight=0.0, loss=None, lse=None, out=None, stream=None):
    """Enqueue :func:`distill_loss` and :func:`distill_grad` in one pass over
    the logits, for a ``grad_loss`` known before the loss (a mean's weights, a
    loss scale).  Returns ``(loss, lse, dlogits)``."""
    lib = _library()
    device = _current_device()
    d = _distill(logits, ids, teacher, temperature, kd_weight, teacher_lse, labels, label_weight, device)
    if loss is None:
        loss = _empty((d.rows,), torch.float32, logits, stream)
    lse, at = _lse_room(lse, logits, labels, device, d.rows, stream)
    out, pitch = _dlogits_room(out, logits, device, d, stream)
    _check(lib.apc_distill_loss_grad(ctypes.byref(d), _vector(grad_loss, "grad_loss", _F32, device, d.rows),
                                     _vector(loss, "loss", _F32, device, d.rows), at, out.data_ptr(), pitch,
                                     _stream(stream, device)))
    return loss, lse, out
