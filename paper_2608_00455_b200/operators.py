"""Embedding lookup, layer / RMS norm, rotary positions, causal attention over packed sequences and the linear head's
cross entropy, with their gradients, and the global gradient norm with clipping: argument marshalling for the
operators of the C ABI (include/dte.h says what each computes).

Tensors are CUDA tensors the caller owns; every call enqueues on `stream` (default: the current stream of the
tensors' device) and returns.  A tensor that belongs to another stream is the caller's to order and to
keep alive (torch.Tensor.record_stream), as for every other call of this package.  A refused argument raises
DteError and enqueues nothing.

Matrices may have any shape whose last dimension is contiguous and whose other dimensions can be flattened to
rows a fixed stride apart.  Workspaces are uint8 tensors of at least the bytes the operator's
*_workspace_bytes function gives for the same sizes.
"""
from __future__ import annotations

import array
import ctypes
import struct
from typing import Optional, Sequence, Tuple

import torch

from .binding import DTE_OK, DteError, _check, lib

DTE_F32, DTE_BF16, DTE_I32, DTE_I64 = 0, 1, 2, 3
DTE_NORM_LAYER, DTE_NORM_RMS = 0, 1
DTE_ROPE_HALF, DTE_ROPE_INTERLEAVED = 0, 1
DTE_ROPE_PLAIN, DTE_ROPE_LINEAR, DTE_ROPE_BASE, DTE_ROPE_RAMP = 0, 1, 2, 3
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


def _heads(t: torch.Tensor, name: str, device: int):
    """(packed dte_matrix, tokens, heads, head_dim) of a tensor (tokens, heads, head_dim) whose heads lie side by side."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        _same_device(t, name, device)
    dtype = _NUMBERS.get(t.dtype)
    if dtype is None:
        _refuse(f"{name} must be float32 or bfloat16")
    if t.dim() != 3:
        _refuse(f"{name} must be tokens x heads x head_dim")
    tokens, heads, dim = t.shape
    if dim == 0:
        _refuse(f"{name}: head_dim must not be 0")
    ld, step, unit = t.stride()
    if (unit != 1 and dim != 1) or (step != dim and heads != 1):
        _refuse(f"{name}: the heads of a token must lie side by side")
    return _pack_matrix(t.data_ptr(), tokens, heads * dim, heads * dim if tokens == 1 else ld, dtype, 0), tokens, heads, dim


def dte_rope_frequencies(rot: int, base: float, scaling: int = DTE_ROPE_PLAIN, factor: float = 1.0, original_positions: float = 0.0,
                         fast_turns: float = 32.0, slow_turns: float = 1.0) -> Tuple[torch.Tensor, float]:
    """(radians per position of each of the rot / 2 pairs: a float64 tensor on the CPU, amplitude)."""
    if not 0 <= rot < 2 ** 32 or not 0 <= scaling < 2 ** 32:
        _refuse("rot and scaling must not be negative")
    f, amplitude = (ctypes.c_double * max(1, min(rot, 1024) // 2))(), ctypes.c_double()
    _done(lib().dte_rope_frequencies(rot, base, scaling, factor, original_positions, fast_turns, slow_turns, f, ctypes.byref(amplitude)))
    return torch.tensor(list(f), dtype=torch.float64), amplitude.value


def dte_rope(q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, frequencies: torch.Tensor,
             q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, interleaved: bool = False,
             amplitude: float = 1.0, inverse: bool = False, stream=None) -> None:
    """Turns the first 2 * len(frequencies) columns of every head of q and k (tokens, heads, head_dim) by positions * frequencies,
    in place where no output is given; inverse: the gradient."""
    device = _device(q, "q")
    m, rows, heads, dim = _heads(q, "q", device)
    o = m
    if q_out is not None:
        o, r, h, d = _heads(q_out, "q_out", device)
        if d != dim or h != heads or r != rows:
            _refuse("q_out must have its input's shape")
    mk = ok = None
    if k is not None:
        mk, rows, heads, dim_k = _heads(k, "k", device)
        if dim_k != dim:
            _refuse("q and k must have one head_dim")
        ok = mk
        if k_out is not None:
            ok, r, h, d = _heads(k_out, "k_out", device)
            if d != dim or h != heads or r != rows:
                _refuse("k_out must have its input's shape")
    elif k_out is not None:
        _refuse("k_out without k")
    p, _ = _ids(positions, "positions", device)
    if not isinstance(frequencies, torch.Tensor) or frequencies.dim() != 1:
        _refuse("frequencies must be a vector")
    pairs = frequencies.numel()
    f = _vector(frequencies, "frequencies", device, pairs, (torch.float64,))
    _done(lib().dte_rope(m, mk, dim, p, f, 2 * pairs, DTE_ROPE_INTERLEAVED if interleaved else DTE_ROPE_HALF, amplitude, bool(inverse),
                         o, ok, device, _stream(stream, device)))


def dte_attention_plan_bytes(tokens: int, n_sequences: int) -> int:
    return lib().dte_attention_plan_bytes(tokens, n_sequences)


def dte_attention_plan(starts: torch.Tensor, tokens: int, plan: torch.Tensor, flags: Optional[torch.Tensor] = None, stream=None) -> None:
    """Leaves in plan the order of work on sequences starts[s] .. starts[s + 1] - 1 of a batch of `tokens` rows."""
    device = _device(starts, "starts")
    if tokens < 0:
        _refuse("tokens must not be negative")
    i, _ = _ids(starts, "starts", device)
    ws, size = _workspace(plan, device)
    _done(lib().dte_attention_plan(i, tokens, ws, size, _flags(flags, device), device, _stream(stream, device)))


def _per_head(t: Optional[torch.Tensor], name: str, device: int, heads: int, tokens: int):
    if t is not None and tuple(t.shape) != (heads, tokens):
        _refuse(f"{name} must be heads x tokens")
    return _vector(t, name, device, heads * tokens)


def dte_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, plan: torch.Tensor, out: torch.Tensor,
                          lse: Optional[torch.Tensor], scale: Optional[float] = None, flags: Optional[torch.Tensor] = None,
                          stream=None) -> None:
    """Causal attention of q (tokens, heads, head_dim) over k and v (tokens, key heads, head_dim) of its sequence; lse (heads,
    tokens) is what the backward pass reads.  scale: 1 / sqrt(head_dim) unless given."""
    device = _device(q, "q")
    m, tokens, heads, dim = _heads(q, "q", device)
    mk, mv, mo = (_heads(t, name, device) for t, name in ((k, "k"), (v, "v"), (out, "out")))
    if not dim == mk[3] == mv[3] == mo[3]:
        _refuse("q, k, v and out must have one head_dim")
    ws, size = _workspace(plan, device)
    _done(lib().dte_attention_forward(m, mk[0], mv[0], dim, ws, size, dim ** -0.5 if scale is None else scale, mo[0],
                                      _per_head(lse, "lse", device, heads, tokens), _flags(flags, device), device,
                                      _stream(stream, device)))


def dte_attention_backward_workspace_bytes(tokens: int, heads: int) -> int:
    return lib().dte_attention_backward_workspace_bytes(tokens, heads)


def dte_attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor,
                           plan: torch.Tensor, dq: torch.Tensor, dk: torch.Tensor, dv: torch.Tensor, workspace: torch.Tensor,
                           scale: Optional[float] = None, flags: Optional[torch.Tensor] = None, stream=None) -> None:
    """Gradients of dte_attention_forward from its outputs and dout."""
    device = _device(q, "q")
    m, tokens, heads, dim = _heads(q, "q", device)
    others = [_heads(t, name, device) for t, name in ((k, "k"), (v, "v"), (out, "out"), (dout, "dout"), (dq, "dq"), (dk, "dk"), (dv, "dv"))]
    if any(o[3] != dim for o in others):
        _refuse("all matrices must have one head_dim")
    mk, mv, mo, md, gq, gk, gv = (o[0] for o in others)
    ws, size = _workspace(plan, device)
    scratch, scratch_size = _workspace(workspace, device)
    _done(lib().dte_attention_backward(m, mk, mv, dim, mo, _per_head(lse, "lse", device, heads, tokens), md, ws, size,
                                       dim ** -0.5 if scale is None else scale, gq, gk, gv, scratch, scratch_size,
                                       _flags(flags, device), device, _stream(stream, device)))


def _tensors(tensors: Sequence[torch.Tensor], name: str, device: int) -> bytes:
    """Packed dte_tensor array."""
    flat = []
    for t in tensors:
        if not isinstance(t, torch.Tensor) or t.get_device() != device:
            _same_device(t, name, device)
        dtype = _NUMBERS.get(t.dtype)
        if dtype is None:
            _refuse(f"{name} must be float32 or bfloat16")
        if not t.is_contiguous():
            _refuse(f"{name} must be contiguous")
        flat += (t.data_ptr(), t.numel(), dtype)       # dtype and the reserved word as one number: both little-endian
    return array.array("Q", flat).tobytes()


def dte_grad_sum_squares_workspace_bytes(n_tensors: int) -> int:
    return lib().dte_grad_sum_squares_workspace_bytes(n_tensors)


def dte_grad_sum_squares(tensors: Sequence[torch.Tensor], sum_squares: torch.Tensor, workspace: torch.Tensor, accumulate: bool = False,
                         stream=None) -> None:
    """sum_squares (one float64) = sum of the squares of all elements of all tensors (accumulate: added to it)."""
    device = _device(sum_squares, "sum_squares")
    ws, size = _workspace(workspace, device)
    _done(lib().dte_grad_sum_squares(_tensors(tensors, "tensors", device), len(tensors), bool(accumulate),
                                     _vector(sum_squares, "sum_squares", device, 1, (torch.float64,)), ws, size, device,
                                     _stream(stream, device)))


def dte_grad_clip(tensors: Sequence[torch.Tensor], sum_squares: torch.Tensor, max_norm: float, norm: Optional[torch.Tensor] = None,
                  outs: Optional[Sequence[torch.Tensor]] = None, stream=None) -> None:
    """Every element times max_norm / norm where norm = sqrt(sum_squares) is larger, and finite in float32; into outs, or in place."""
    device = _device(sum_squares, "sum_squares")
    if outs is not None and len(outs) != len(tensors):
        _refuse("outs must have one tensor per tensor")
    _done(lib().dte_grad_clip(_tensors(tensors, "tensors", device), len(tensors),
                              _vector(sum_squares, "sum_squares", device, 1, (torch.float64,)), max_norm,
                              None if outs is None else _tensors(outs, "outs", device), _vector(norm, "norm", device, 1), device,
                              _stream(stream, device)))
