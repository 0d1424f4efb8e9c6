"""Embedding lookup, layer / RMS norm and the linear head's cross entropy, with their gradients: argument
marshalling for the operators of the C ABI (include/dte.h says what each computes).

Tensors are CUDA tensors the caller owns; every call enqueues on `stream` (default: the current stream of the
tensors' device) and returns.  A tensor that belongs to another stream is the caller's to order and to
keep alive (torch.Tensor.record_stream), as for every other call of this package.  A refused argument raises
DteError and enqueues nothing.

Matrices may have any shape whose last dimension is contiguous and whose other dimensions can be flattened to
rows a fixed stride apart.  Workspaces are uint8 tensors of at least the bytes the operator's
*_workspace_bytes function gives for the same sizes.
"""
from __future__ import annotations

import struct
from typing import Optional

import torch

from .binding import DTE_OK, DteError, _check, lib

DTE_F32, DTE_BF16, DTE_I32, DTE_I64 = 0, 1, 2, 3
DTE_NORM_LAYER, DTE_NORM_RMS = 0, 1
_INVALID_ARG = 1

_NUMBERS = {torch.float32: DTE_F32, torch.bfloat16: DTE_BF16}
_IDS = {torch.int32: DTE_I32, torch.int64: DTE_I64}


# dte_matrix and dte_ids of the C ABI as packed bytes (natural alignment, no padding): cheaper to make per call than
# a ctypes structure
_pack_matrix = struct.Struct("=QQQQII").pack
_pack_ids = struct.Struct("=QQII").pack
assert struct.calcsize("=QQQQII") == 40 and struct.calcsize("=QQII") == 24


def _refuse(msg: str):
    raise DteError(_INVALID_ARG, msg)


def _device(t: torch.Tensor, name: str) -> int:
    if not isinstance(t, torch.Tensor):
        _refuse(f"{name} must be a tensor")
    device = t.get_device()               # -1 on the CPU
    if device < 0:
        _refuse(f"{name} is not on a CUDA device; there is no CPU fallback")
    return device


def _same_device(t: torch.Tensor, name: str, device: int) -> None:
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        if _device(t, name) != device:
            _refuse(f"{name} is on another device")


def _rows(t: torch.Tensor, name: str):
    """(rows, stride between rows) of a tensor seen as a matrix of its last dimension."""
    shape, stride = t.shape, t.stride()
    n, ld = 1, None
    for d in range(t.dim() - 2, -1, -1):
        if shape[d] == 1:
            continue
        if ld is None:
            ld = stride[d]
        elif stride[d] != ld * n and shape[d] * n > 0:
            _refuse(f"{name}: the leading dimensions cannot be flattened to rows a fixed stride apart")
        n *= shape[d]
    return n, shape[-1] if ld is None else ld


def _matrix(t: torch.Tensor, name: str, device: int):
    """(packed dte_matrix, rows, columns)."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        _same_device(t, name, device)
    dtype = _NUMBERS.get(t.dtype)
    if dtype is None:
        _refuse(f"{name} must be float32 or bfloat16")
    stride = t.stride()
    if len(stride) == 2:
        rows, cols = t.shape
        ld, unit = stride
        if rows == 1:
            ld = cols
    elif stride:
        cols, unit = t.shape[-1], stride[-1]
        rows, ld = _rows(t, name)
    else:
        _refuse(f"{name} needs at least one dimension")
    if unit != 1 and cols != 1:
        _refuse(f"{name}: the last dimension must be contiguous")
    return _pack_matrix(t.data_ptr(), rows, cols, ld, dtype, 0), rows, cols


def _ids(t: torch.Tensor, name: str, device: int):
    """(packed dte_ids, count)."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        _same_device(t, name, device)
    dtype = _IDS.get(t.dtype)
    if dtype is None:
        _refuse(f"{name} must be int32 or int64")
    if not t.is_contiguous():
        _refuse(f"{name} must be contiguous")
    count = t.numel()
    return _pack_ids(t.data_ptr(), count, dtype, 0), count


def _vector(t: Optional[torch.Tensor], name: str, device: int, count: int, dtypes=(torch.float32,)):
    """Address of a contiguous vector of `count` values, or None."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.numel() == count and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    _same_device(t, name, device)
    if t.dtype not in dtypes:
        _refuse(f"{name} must be {' or '.join(str(d).removeprefix('torch.') for d in dtypes)}")
    if t.numel() != count or not t.is_contiguous():
        _refuse(f"{name} must be contiguous with {count} values")
    return t.data_ptr()


def _workspace(t: Optional[torch.Tensor], device: int):
    if t is None:
        return None, 0
    _same_device(t, "workspace", device)
    if not t.is_contiguous():
        _refuse("workspace must be contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def _flags(t: Optional[torch.Tensor], device: int):
    if t is None:
        return None
    _same_device(t, "flags", device)
    if t.dtype != torch.int64 or t.numel() < 1:
        _refuse("flags must be int64")
    return t.data_ptr()


# the current stream's handle without a Stream object around it, where this torch has the call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, device: int) -> int:
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _range(start: int, rows: int, vocab: Optional[int], name: str):
    """(first row, vocabulary size) of a shard."""
    if start < 0 or (vocab is not None and vocab < 0):
        _refuse(f"{name} and vocab must not be negative")
    return start, start + rows if vocab is None else vocab


def _done(status: int) -> None:
    if status != DTE_OK:
        _check(status)


_PARAM_TYPES = (torch.float32, torch.bfloat16)


def _params(weight, bias, device: int, cols: int):
    w = _vector(weight, "weight", device, cols, _PARAM_TYPES)
    b = _vector(bias, "bias", device, cols, _PARAM_TYPES)
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        _refuse("weight and bias must have one type")
    kept = weight if weight is not None else bias
    return w, b, DTE_F32 if kept is None else _NUMBERS[kept.dtype]


def dte_embedding_forward(table: torch.Tensor, ids: torch.Tensor, out: torch.Tensor, scale: float = 1.0, row_start: int = 0,
                          vocab: Optional[int] = None, flags: Optional[torch.Tensor] = None, stream=None) -> None:
    """out[n] = scale * table[ids[n] - row_start], zero for negative ids and ids of other shards."""
    device = _device(table, "table")
    m, rows, _ = _matrix(table, "table", device)
    o, _, _ = _matrix(out, "out", device)
    i, _ = _ids(ids, "ids", device)
    first, total = _range(row_start, rows, vocab, "row_start")
    _done(lib().dte_embedding_forward(m, i, first, total, scale, o, _flags(flags, device), device, _stream(stream, device)))


def dte_embedding_backward_workspace_bytes(n_ids: int, hidden: int) -> int:
    return lib().dte_embedding_backward_workspace_bytes(n_ids, hidden)


def dte_embedding_backward(dout: torch.Tensor, ids: torch.Tensor, dtable: torch.Tensor, workspace: torch.Tensor, scale: float = 1.0,
                           row_start: int = 0, vocab: Optional[int] = None, accumulate: bool = False,
                           flags: Optional[torch.Tensor] = None, stream=None) -> None:
    """dtable[v] (+)= scale * sum of dout[n] over the tokens with ids[n] == row_start + v."""
    device = _device(dtable, "dtable")
    d, _, _ = _matrix(dout, "dout", device)
    m, rows, _ = _matrix(dtable, "dtable", device)
    i, _ = _ids(ids, "ids", device)
    ws, size = _workspace(workspace, device)
    first, total = _range(row_start, rows, vocab, "row_start")
    _done(lib().dte_embedding_backward(d, i, first, total, scale, bool(accumulate), m, ws, size, _flags(flags, device), device,
                                       _stream(stream, device)))


def dte_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor], bias: Optional[torch.Tensor], out: torch.Tensor,
                     mean: Optional[torch.Tensor], rstd: Optional[torch.Tensor], eps: float, rms: bool = False, stream=None) -> None:
    """Layer norm (rms: RMS norm) of every row of x; mean and rstd keep the statistics for the backward pass."""
    device = _device(x, "x")
    m, rows, cols = _matrix(x, "x", device)
    o, _, _ = _matrix(out, "out", device)
    w, b, dtype = _params(weight, bias, device, cols)
    _done(lib().dte_norm_forward(m, w, b, dtype, DTE_NORM_RMS if rms else DTE_NORM_LAYER, eps, o,
                                 _vector(mean, "mean", device, rows), _vector(rstd, "rstd", device, rows), device,
                                 _stream(stream, device)))


def dte_norm_backward_workspace_bytes(rows: int, hidden: int) -> int:
    return lib().dte_norm_backward_workspace_bytes(rows, hidden)


def dte_norm_backward(dout: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: Optional[torch.Tensor],
                      rstd: torch.Tensor, dx: Optional[torch.Tensor], dweight: Optional[torch.Tensor], dbias: Optional[torch.Tensor],
                      workspace: Optional[torch.Tensor], accumulate: bool = False, rms: bool = False, stream=None) -> None:
    """Gradients of dte_norm_forward; dweight and dbias are float32 (accumulate: added to)."""
    device = _device(x, "x")
    d, _, _ = _matrix(dout, "dout", device)
    m, rows, cols = _matrix(x, "x", device)
    o = None if dx is None else _matrix(dx, "dx", device)[0]
    w, _, dtype = _params(weight, None, device, cols)
    ws, size = _workspace(workspace, device)
    _done(lib().dte_norm_backward(d, m, w, dtype, DTE_NORM_RMS if rms else DTE_NORM_LAYER,
                                  _vector(mean, "mean", device, rows), _vector(rstd, "rstd", device, rows), bool(accumulate),
                                  o, _vector(dweight, "dweight", device, cols), _vector(dbias, "dbias", device, cols), ws, size, device, _stream(stream, device)))


def dte_linear_ce_forward_workspace_bytes(tokens: int, vocab_rows: int, hidden: int) -> int:
    return lib().dte_linear_ce_forward_workspace_bytes(tokens, vocab_rows, hidden)


def dte_linear_ce_forward(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                          target_logit: Optional[torch.Tensor], loss: Optional[torch.Tensor], workspace: torch.Tensor,
                          logit_scale: float = 1.0, vocab_start: int = 0, vocab: Optional[int] = None,
                          flags: Optional[torch.Tensor] = None, stream=None) -> None:
    """lse, target logit and loss of every token for the head rows [vocab_start, vocab_start + rows)."""
    device = _device(x, "x")
    m, _, _ = _matrix(x, "x", device)
    w, rows, _ = _matrix(weight, "weight", device)
    t, n = _ids(targets, "targets", device)
    ws, size = _workspace(workspace, device)
    first, total = _range(vocab_start, rows, vocab, "vocab_start")
    _done(lib().dte_linear_ce_forward(m, w, t, first, total, logit_scale,
                                      _vector(lse, "lse", device, n), _vector(target_logit, "target_logit", device, n),
                                      _vector(loss, "loss", device, n), ws, size, _flags(flags, device), device,
                                      _stream(stream, device)))


def dte_linear_ce_backward_workspace_bytes(tokens: int, vocab_rows: int, hidden: int) -> int:
    return lib().dte_linear_ce_backward_workspace_bytes(tokens, vocab_rows, hidden)


def dte_linear_ce_backward_workspace_min_bytes(tokens: int, vocab_rows: int, hidden: int) -> int:
    return lib().dte_linear_ce_backward_workspace_min_bytes(tokens, vocab_rows, hidden)


def dte_linear_ce_backward(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, dloss: torch.Tensor,
                           dx: Optional[torch.Tensor], dweight: Optional[torch.Tensor], workspace: torch.Tensor,
                           logit_scale: float = 1.0, vocab_start: int = 0, vocab: Optional[int] = None, accumulate: bool = False,
                           flags: Optional[torch.Tensor] = None, stream=None) -> None:
    """dx and dweight for a given dloss per token; lse over the whole vocabulary."""
    device = _device(x, "x")
    m, _, _ = _matrix(x, "x", device)
    w, rows, _ = _matrix(weight, "weight", device)
    t, n = _ids(targets, "targets", device)
    d = None if dx is None else _matrix(dx, "dx", device)[0]
    g = None if dweight is None else _matrix(dweight, "dweight", device)[0]
    ws, size = _workspace(workspace, device)
    first, total = _range(vocab_start, rows, vocab, "vocab_start")
    _done(lib().dte_linear_ce_backward(m, w, t, first, total, logit_scale,
                                       _vector(lse, "lse", device, n), _vector(dloss, "dloss", device, n),
                                       bool(accumulate), d, g, ws,
                                       size, _flags(flags, device), device, _stream(stream, device)))
