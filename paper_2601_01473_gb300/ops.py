"""The operators of a model that is trained on prepared hyperbatches
(include/agnes_ops.h): learned node embeddings with their gradient,
distillation from a teacher's top logits, and feature rows in microscaled 4-bit
floating point.  Argument marshalling only; each call runs the library's CUDA
kernels on the current stream (or ``stream``) and returns without waiting.  Results
are no part of autograd's graph, whatever the arguments require: a training step calls
the gradients itself, or from the backward of its own ``autograd.Function``.

What a kernel finds wrong with its data (an id past the end of its table, a wait
that ran out) is kept on the device, in the int32 tensor ``status`` if one is
given and else in one per device that ``check()`` reads and clears.

With ``stream`` (a Stream or a handle, of the arguments' device), the results
belong to that stream, and the inputs' memory is kept until it has come past the
call; the inputs' values have to be there by then (order the stream after the one
that makes them).
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple

import torch

from .agnes import AgnesError, _stream_of_handle, lib

_FLOATS = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_INDEXES = {torch.int32: 32, torch.int64: 64}
BAD_INDEX, TIMEOUT = 1, 2  # AGNES_OP_*

_status = {}  # device index -> int32 [1]


class RowGrad(NamedTuple):
    """The gradient of the selected rows of a table."""
    ids: torch.Tensor    # int32 [n]: the distinct ids in ascending order, then -1
    rows: torch.Tensor   # [n, dim]: their gradients, then zeros
    count: torch.Tensor  # int32 [1]: how many


def _stream_of(stream, device):
    """``stream``, a Stream or a handle, as a stream of ``device``."""
    if not isinstance(stream, torch.cuda.Stream):
        return _stream_of_handle(int(stream), device)
    if stream.device != device:
        raise ValueError(f"the stream is {stream.device}'s, the arguments are on {device}")
    return stream


def _on_stream(stream, op, *args):
    """op(*args) with ``stream`` current on the arguments' device."""
    tensors = [t for t in args if isinstance(t, torch.Tensor) and t.is_cuda]
    if not tensors:
        return op(*args)  # which refuses them
    stream = _stream_of(stream, tensors[0].device)
    with torch.cuda.stream(stream):
        result = op(*args)
    for t in tensors:
        t.record_stream(stream)
    return result


def _failed(rc: int):
    msg = lib().agnes_last_error(None)
    raise AgnesError(rc, msg.decode() if msg else "")


def _stream(device) -> int | None:
    return torch.cuda.current_stream(device).cuda_stream or None


# the same number without a Stream object around it (2 us of host time a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
if _raw_stream is not None:
    def _stream(device) -> int | None:  # noqa: F811
        return _raw_stream(device.index) or None


def _status_word(status, device) -> int:
    if status is None:
        status = _status.get(device.index)
        if status is None:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("the first call on a device cannot be captured without a "
                                   "status tensor")
            with torch.inference_mode(False):  # else check() may not clear it
                status = torch.zeros(1, dtype=torch.int32, device=device)
            torch.cuda.current_stream(device).synchronize()
            _status[device.index] = status
    elif status.dtype != torch.int32 or status.numel() < 1:
        raise TypeError("status must be an int32 tensor")
    elif status.device != device:
        raise ValueError(f"status must be on {device}")
    return status.data_ptr()


def check(device=None) -> None:
    """Waits for the device and raises AgnesError for what its kernels have found
    wrong since the last check (calls without a ``status`` of their own)."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else \
        torch.device(device)
    index = torch.cuda.current_device() if device.index is None else device.index
    torch.cuda.synchronize(index)
    if index not in _status:
        return
    found = int(_status[index])
    if not found:
        return
    _status[index].zero_()
    torch.cuda.synchronize(index)
    if found & TIMEOUT:
        raise AgnesError(6, "a kernel's bounded wait ran out")
    raise AgnesError(1, "an id or index is at or past the end of its range")


def _rows(name: str, t: torch.Tensor, device=None):
    """(device, rows, columns, row stride) of a matrix of floats whose rows' elements
    are adjacent."""
    if not isinstance(t, torch.Tensor) or t.ndim != 2 or t.dtype not in _FLOATS:
        raise TypeError(f"{name} must be a 2-D float32, float16 or bfloat16 tensor")
    n, dim = t.shape
    step, unit = t.stride()
    if n <= 1:
        step = dim  # there is no next row
    if (unit != 1 and dim > 1 or step < dim) and n and dim:
        raise ValueError(f"{name} must have adjacent elements in each row")
    if device is not None or not t.is_cuda:
        return _on(name, t, device), n, dim, step
    return t.device, n, dim, step


def _on(name: str, t: torch.Tensor, device):
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a CUDA device")
    if device is None:
        return t.device
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    return device


def _ids(name: str, t: torch.Tensor, device) -> int:
    """The bits of a contiguous tensor of indexes."""
    bits = _INDEXES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if bits is None:
        raise TypeError(f"{name} must be an int32 or int64 tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    _on(name, t, device)
    return bits


def _output(out, n, dim, dtype, device):
    """(tensor, its type's code, row stride) of an output [n, dim]: the caller's `out`,
    or a new one of `dtype`."""
    if out is None:
        code = _FLOATS.get(dtype)
        if code is None:
            raise TypeError(f"{dtype} is not float32, float16 or bfloat16")
        return torch.empty((n, dim), dtype=dtype, device=device), code, dim
    _, rows, cols, step = _rows("out", out, device)
    if (rows, cols) != (n, dim):
        raise ValueError(f"out must be {(n, dim)}, not {(rows, cols)}")
    if dtype is not None and dtype != out.dtype:
        raise TypeError("out has another type than out_dtype")
    return out, _FLOATS[out.dtype], step


# ---- embeddings -------------------------------------------------------------------------


def embedding_lookup(table, ids, scale: float = 1.0, out_dtype=None, out=None, status=None,
                     stream=None):
    """``scale * table[ids]`` (agnes_embedding_lookup): the rows of ``table``
    [rows, dim] for ``ids`` of any shape, as [*ids.shape, dim] of ``out_dtype`` (the
    table's by default).  A negative id gives zeros.  ``out``: [ids.numel(), dim],
    its rows adjacent or not, written instead of a new tensor and returned."""
    if stream is not None:
        return _on_stream(stream, embedding_lookup, table, ids, scale, out_dtype, out, status)
    device, rows, dim, step = _rows("table", table)
    bits = _ids("ids", ids, device)
    n = ids.numel()
    if out is None and out_dtype is None:
        out_dtype = table.dtype
    y, code, out_step = _output(out, n, dim, out_dtype, device)
    rc = lib().agnes_embedding_lookup(
        table.data_ptr(), _FLOATS[table.dtype], rows, step, dim, ids.data_ptr(), bits, n, scale,
        y.data_ptr(), code, out_step, _status_word(status, device), _stream(device))
    if rc:
        _failed(rc)
    return y if out is not None or ids.ndim == 1 else y.view(*ids.shape, dim)


@functools.lru_cache(maxsize=1024)
def _grad_workspace(n, dim) -> int:
    need = ctypes.c_int64()
    rc = lib().agnes_embedding_grad_workspace(n, dim, ctypes.byref(need))
    if rc:
        _failed(rc)
    return need.value


def _grad_arguments(grad, ids):
    device, n, dim, step = _rows("grad", grad)
    bits = _ids("ids", ids, device)
    if ids.numel() != n:
        raise ValueError(f"{ids.numel()} ids for {n} rows of grad")
    ws = torch.empty(_grad_workspace(n, dim), dtype=torch.uint8, device=device)
    return device, n, dim, ws, (grad.data_ptr(), _FLOATS[grad.dtype], step, ids.data_ptr(), bits, n)


def embedding_grad(grad, ids, num_rows: int, scale: float = 1.0, out_dtype=None, out=None,
                   status=None, stream=None):
    """The gradient of ``embedding_lookup`` to the whole table (agnes_embedding_grad):
    [num_rows, dim] of ``out_dtype`` (grad's by default), row v the scaled sum of the
    rows of ``grad`` [n, dim] whose id (``ids``, n of any shape) is v, zeros where
    there is none.  ``out``: written instead of a new tensor; contiguous."""
    if stream is not None:
        return _on_stream(stream, embedding_grad, grad, ids, num_rows, scale, out_dtype, out,
                          status)
    device, n, dim, ws, arguments = _grad_arguments(grad, ids)
    if out is None and out_dtype is None:
        out_dtype = grad.dtype
    y, code, step = _output(out, num_rows, dim, out_dtype, device)
    if step != dim:
        raise ValueError("out must be contiguous")
    rc = lib().agnes_embedding_grad(
        *arguments, num_rows, dim, scale, y.data_ptr(), code, ws.data_ptr(), ws.numel(),
        _status_word(status, device), _stream(device))
    if rc:
        _failed(rc)
    return y


def embedding_grad_rows(grad, ids, num_rows: int, scale: float = 1.0, out_dtype=None, status=None,
                        stream=None) -> RowGrad:
    """The same gradient for the selected rows only (agnes_embedding_grad_rows), for
    tables too large for a dense one.  Its shapes do not depend on the ids, so
    ``table.index_add_(0, g.ids.clamp(min=0), g.rows, alpha=-lr)`` needs no read-back:
    the rows past ``count`` are zeros."""
    if stream is not None:
        return _on_stream(stream, embedding_grad_rows, grad, ids, num_rows, scale, out_dtype,
                          status)
    device, n, dim, ws, arguments = _grad_arguments(grad, ids)
    rows, code, _ = _output(None, n, dim, out_dtype or grad.dtype, device)
    out_ids = torch.empty(n, dtype=torch.int32, device=device)
    count = torch.empty(1, dtype=torch.int32, device=device)
    rc = lib().agnes_embedding_grad_rows(
        *arguments, num_rows, dim, scale, out_ids.data_ptr(), rows.data_ptr(), code,
        count.data_ptr(), ws.data_ptr(), ws.numel(), _status_word(status, device),
        _stream(device))
    if rc:
        _failed(rc)
    return RowGrad(out_ids, rows, count)


# ---- distillation -------------------------------------------------------------------------


def _distill_arguments(logits, teacher, index):
    device, n, classes, step = _rows("logits", logits)
    _, rows, top, teacher_step = _rows("teacher", teacher, device)
    bits = _ids("index", index, device)
    if teacher_step != top and rows and top:
        raise ValueError("teacher must be contiguous")
    if rows != n or index.shape != teacher.shape:
        raise ValueError(f"teacher {tuple(teacher.shape)} and index {tuple(index.shape)} must be "
                         f"[{n}, top]")
    return device, n, classes, (
        logits.data_ptr(), _FLOATS[logits.dtype], step, n, classes, teacher.data_ptr(),
        _FLOATS[teacher.dtype], index.data_ptr(), bits, top)


def _weight_arguments(weight, rows, device):
    if not isinstance(weight, torch.Tensor):
        return None, float(weight)
    if weight.dtype != torch.float32 or weight.shape != (rows,) or not weight.is_contiguous():
        raise TypeError(f"weight must be a number or a contiguous float32 tensor [{rows}]")
    _on("weight", weight, device)
    return weight.data_ptr(), 1.0


def distill_loss(logits, teacher, index, temperature: float = 1.0, status=None, stream=None):
    """Each row's loss against the teacher's top logits (agnes_distill_loss):
    ``logits`` [rows, classes], ``teacher`` [rows, top] with their classes ``index``
    (negative: absent).  Returns (loss float32 [rows], stats float32 [rows, 2]);
    ``distill_grad`` takes the stats."""
    if stream is not None:
        return _on_stream(stream, distill_loss, logits, teacher, index, temperature, status)
    device, n, _, arguments = _distill_arguments(logits, teacher, index)
    loss = torch.empty(n, dtype=torch.float32, device=device)
    stats = torch.empty((n, 2), dtype=torch.float32, device=device)
    rc = lib().agnes_distill_loss(*arguments, temperature, loss.data_ptr(), stats.data_ptr(),
                                  _status_word(status, device), _stream(device))
    if rc:
        _failed(rc)
    return loss, stats


def distill_grad(logits, teacher, index, stats, weight=1.0, temperature: float = 1.0,
                 out_dtype=None, out=None, status=None, stream=None):
    """The gradient of sum(weight * loss) to the logits (agnes_distill_grad):
    ``weight`` a number or float32 [rows], ``stats`` from ``distill_loss``.  ``out``:
    written instead of a new tensor of ``out_dtype`` (the logits' by default); it may
    be ``logits``."""
    if stream is not None:
        return _on_stream(stream, distill_grad, logits, teacher, index, stats, weight,
                          temperature, out_dtype, out, status)
    device, n, classes, arguments = _distill_arguments(logits, teacher, index)
    if stats.dtype != torch.float32 or stats.shape != (n, 2) or not stats.is_contiguous():
        raise TypeError("stats must be what distill_loss returned")
    _on("stats", stats, device)
    w, w_scale = _weight_arguments(weight, n, device)
    if out is None and out_dtype is None:
        out_dtype = logits.dtype
    y, code, step = _output(out, n, classes, out_dtype, device)
    rc = lib().agnes_distill_grad(*arguments, temperature, stats.data_ptr(), w, w_scale,
                                  y.data_ptr(), code, step, _status_word(status, device),
                                  _stream(device))
    if rc:
        _failed(rc)
    return y


def distill_loss_grad(logits, teacher, index, weight=1.0, temperature: float = 1.0, out_dtype=None,
                      out=None, status=None, stream=None):
    """(loss, gradient) in one call, the logits read once (agnes_distill_loss_grad);
    arguments as for ``distill_loss`` and ``distill_grad``."""
    if stream is not None:
        return _on_stream(stream, distill_loss_grad, logits, teacher, index, weight, temperature,
                          out_dtype, out, status)
    device, n, classes, arguments = _distill_arguments(logits, teacher, index)
    w, w_scale = _weight_arguments(weight, n, device)
    loss = torch.empty(n, dtype=torch.float32, device=device)
    if out is None and out_dtype is None:
        out_dtype = logits.dtype
    y, code, step = _output(out, n, classes, out_dtype, device)
    rc = lib().agnes_distill_loss_grad(*arguments, temperature, w, w_scale, loss.data_ptr(),
                                       y.data_ptr(), code, step, _status_word(status, device),
                                       _stream(device))
    if rc:
        _failed(rc)
    return loss, y


# ---- 4-bit rows -----------------------------------------------------------------------------


def mx4_row_bytes(dim: int) -> int:
    """Bytes of a 4-bit row of ``dim`` values (agnes_mx4_row_bytes)."""
    need = ctypes.c_int64()
    rc = lib().agnes_mx4_row_bytes(dim, ctypes.byref(need))
    if rc:
        _failed(rc)
    return need.value


def _packed(name, t, dim, device=None):
    """(device, rows, row stride in bytes) of a matrix of 4-bit rows: uint8
    [rows, mx4_row_bytes(dim)], or the same bytes as float16 or float32 "features", as a
    graph gathers them."""
    if not isinstance(t, torch.Tensor) or t.ndim != 2 or \
            t.dtype not in (torch.uint8, torch.float16, torch.float32):
        raise TypeError(f"{name} must be a 2-D tensor of 4-bit rows")
    n, cols = t.shape
    step, unit = t.stride()
    size = t.element_size()
    if dim < 1 or cols * size != ((dim + 31) // 32 * 17 + 15) // 16 * 16:
        raise ValueError(f"{name} has rows of {cols * size} bytes, not those of {dim} values")
    if n <= 1:
        step = cols  # there is no next row
    if (unit != 1 or step < cols) and n:
        raise ValueError(f"{name} must have adjacent bytes in each row")
    return _on(name, t, device), n, step * size


def mx4_quantize(x, out=None, stream=None):
    """Rows of ``x`` [rows, dim] rounded to microscaled 4-bit rows (agnes_mx4_quantize):
    uint8 [rows, mx4_row_bytes(dim)].  ``.view(torch.float16)`` of them makes a graph's
    features."""
    if stream is not None:
        return _on_stream(stream, mx4_quantize, x, out)
    device, rows, dim, step = _rows("x", x)
    if out is None:
        out_step = mx4_row_bytes(dim)
        out = torch.empty((rows, out_step), dtype=torch.uint8, device=device)
    else:
        _, n, out_step = _packed("out", out, dim, device)
        if n != rows:
            raise ValueError(f"out has {n} rows, not {rows}")
    rc = lib().agnes_mx4_quantize(x.data_ptr(), _FLOATS[x.dtype], step, rows, dim,
                                  out.data_ptr(), out_step, _stream(device))
    if rc:
        _failed(rc)
    return out


def mx4_dequantize(x, dim: int, out_dtype=torch.float32, out=None, stream=None):
    """The values [rows, dim] that 4-bit rows stand for (agnes_mx4_dequantize)."""
    if stream is not None:
        return _on_stream(stream, mx4_dequantize, x, dim, out_dtype, out)
    device, rows, step = _packed("x", x, dim)
    y, code, out_step = _output(out, rows, dim, out_dtype if out is None else None, device)
    rc = lib().agnes_mx4_dequantize(x.data_ptr(), step, rows, dim, y.data_ptr(), code, out_step,
                                    _stream(device))
    if rc:
        _failed(rc)
    return y


def mx4_linear(x, w, dim: int, bias=None, out_dtype=torch.float32, out=None, status=None,
               stream=None):
    """``x @ w.T + bias`` of 4-bit rows (agnes_mx4_linear): ``x`` [rows, bytes], for example a
    minibatch's gathered features, ``w`` [width, bytes], both of ``dim`` values a row;
    ``bias`` float32 [width] or None.  Returns [rows, width]."""
    if stream is not None:
        return _on_stream(stream, mx4_linear, x, w, dim, bias, out_dtype, out, status)
    device, rows, step = _packed("x", x, dim)
    _, width, w_step = _packed("w", w, dim, device)
    at = None
    if bias is not None:
        if bias.dtype != torch.float32 or bias.shape != (width,) or not bias.is_contiguous():
            raise TypeError(f"bias must be a contiguous float32 tensor [{width}]")
        _on("bias", bias, device)
        at = bias.data_ptr()
    y, code, out_step = _output(out, rows, width, out_dtype if out is None else None, device)
    rc = lib().agnes_mx4_linear(x.data_ptr(), step, rows, w.data_ptr(), w_step, width, dim, at,
                                y.data_ptr(), code, out_step, _status_word(status, device),
                                _stream(device))
    if rc:
        _failed(rc)
    return y
