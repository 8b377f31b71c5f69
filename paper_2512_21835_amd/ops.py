"""Binding of include/stage_ops.h: operators around a layer's projections, on torch tensors.

Argument marshalling and the checks that need the tensors' shapes; the library checks the rest.  A call
runs on the current torch stream of its tensors' device unless ``stream`` (a torch stream of it) is given,
and returns the tensor that it writes.  With ``stream`` the tensors' memory is kept until the call is done there, as by
Tensor.record_stream; waiting for their contents is the caller's.  Where a call needs a workspace and none is given, one is
taken from torch's allocator, on that stream.  The operators have no backward pass: where gradients are being recorded,
tensors that require one are refused.
"""
from __future__ import annotations

import ctypes
import struct
from ctypes import c_float, c_int32, c_int64, c_void_p
from typing import Optional, Sequence, Tuple

import torch

from .stage import STAGE_BF16, STAGE_F32, _check, lib

_TYPES = {torch.float32: STAGE_F32, torch.bfloat16: STAGE_BF16}


class StageBatch(ctypes.Structure):
    """stage_batch of include/stage_ops.h; stage_batch() makes one and keeps its tensors."""
    _fields_ = [("n_seqs", c_int32), ("max_rows", c_int32), ("max_len", c_int32), ("max_blocks", c_int32),
                ("row_start", c_void_p), ("length", c_void_p), ("block_table", c_void_p)]


class StageCache(ctypes.Structure):
    _fields_ = [("pool", c_void_p), ("n_blocks", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32),
                ("type", c_int32)]


class StageAppendArgs(ctypes.Structure):
    _fields_ = [("device", c_int32), ("batch", StageBatch), ("cache", StageCache), ("rows", c_int32),
                ("n_q_heads", c_int32), ("qkv", c_void_p), ("q_out", c_void_p), ("qkv_ld", c_int64), ("q_ld", c_int64),
                ("qkv_type", c_int32), ("q_type", c_int32), ("q_gain", c_void_p), ("k_gain", c_void_p),
                ("eps", c_float), ("n_angles", c_int32), ("cos", c_void_p), ("sin", c_void_p),
                ("positions", c_void_p), ("n_axes", c_int32), ("section", c_int32 * 3)]


class StageWindowArgs(ctypes.Structure):
    _fields_ = [("device", c_int32), ("batch", StageBatch), ("cache", StageCache), ("rows", c_int32),
                ("n_q_heads", c_int32), ("window", c_int32), ("sinks", c_int32), ("scale", c_float), ("q", c_void_p),
                ("out", c_void_p), ("q_ld", c_int64), ("out_ld", c_int64), ("type", c_int32)]


class StageAdapterArgs(ctypes.Structure):
    _fields_ = [("device", c_int32), ("rows", c_int32), ("k", c_int32), ("n", c_int32), ("n_adapters", c_int32),
                ("max_rank", c_int32), ("type", c_int32), ("x", c_void_p), ("base", c_void_p), ("out", c_void_p),
                ("x_ld", c_int64), ("base_ld", c_int64), ("out_ld", c_int64), ("a", c_void_p), ("b", c_void_p),
                ("ids", c_void_p), ("ranks", c_void_p), ("scales", c_void_p)]


# A call's argument struct as one pack() (a tenth of the time of filling a ctypes structure field by field; the
# classes above are the same layouts for programs that call the library themselves).  "40s" is a StageBatch.
_BATCH = struct.Struct("@iiiiPPP")
_APPEND = struct.Struct("@i4x40sPiiii ii PP qq ii PP fi PPP iiii")
_WINDOW = struct.Struct("@i4x40sPiiii ii iif4x PP qq i4x")
_ADAPTER = struct.Struct("@iiiiiii4x PPP qqq PPP PP")


_recording = torch.is_grad_enabled


def _no_backward() -> ValueError:
    return ValueError("the operators have no backward pass: a tensor that requires a gradient is taken under torch.no_grad() only")


def _device(t: torch.Tensor) -> int:
    device = t.get_device()
    if device < 0:
        raise ValueError("tensors must be on a GPU")
    return device


def _type(t: torch.Tensor) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"float32 or bfloat16 is needed, got {t.dtype}")
    return kind


def _plain(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, shape: Tuple[int, ...], device: int) -> int:
    """Address of a contiguous tensor of this type, shape and device; 0 for none."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {shape} on the call's device, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _row_stride(t: torch.Tensor, name: str, device: int) -> int:
    """Elements from row to row of [rows, width] or [rows, heads, head_dim], whose rows are each contiguous."""
    shape = t.shape
    if t.get_device() != device:
        raise ValueError(f"{name} is on another device")
    width = shape[-1] if len(shape) == 2 else shape[1] * shape[2]
    if t.is_contiguous():
        return width
    stride = t.stride()
    if (stride[-1] != 1 and shape[-1] != 1) or (len(shape) == 3 and stride[1] != shape[2] and shape[1] != 1):
        raise ValueError(f"the rows of {name} must be contiguous")
    return stride[0] if shape[0] > 1 else width


def _cache(pool: torch.Tensor, device: int) -> Tuple[int, int, int, int, int]:
    shape = pool.shape
    if len(shape) != 5 or shape[1] != 2 or shape[3] != 16 or not pool.is_contiguous() or pool.get_device() != device:
        raise ValueError("pool must be a contiguous tensor [n_blocks, 2, n_kv_heads, 16, head_dim] on the call's device")
    return pool.data_ptr(), shape[0], shape[2], shape[4], _type(pool)


def _batch(batch: StageBatch, device: int) -> bytes:
    if batch.device != device:
        raise ValueError("the batch is on another device")
    return batch.raw


def _workspace(size, args: bytes, device: int, given: Optional[torch.Tensor], stream):
    """Address and bytes of the workspace of a call, and what keeps it."""
    if given is not None:
        if not given.is_contiguous() or given.get_device() != device:
            raise ValueError("the workspace must be a contiguous tensor on the call's device")
        return given.data_ptr(), given.nbytes, given
    need = c_int64()
    rc = size(args, ctypes.byref(need))
    if rc:
        _check(rc)
    if need.value == 0:
        return None, 0, None
    if stream is None:
        given = torch.empty(need.value, dtype=torch.uint8, device=device)
    else:
        with torch.cuda.stream(stream):
            given = torch.empty(need.value, dtype=torch.uint8, device=device)
    return given.data_ptr(), need.value, given


def _handle(stream, device: int) -> int:
    if stream is None:
        return _current_stream(device)
    if stream.device.index != device:
        raise ValueError("the stream is on another device")
    return stream.cuda_stream


def _keep(stream, *tensors: Optional[torch.Tensor]) -> None:
    """The tensors' memory goes to nobody else before what is enqueued on `stream` is done."""
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def _current_stream(device: int) -> int:
    return torch.cuda.current_stream(device).cuda_stream


if hasattr(torch._C, "_cuda_getCurrentRawStream"):   # (the same handle, without a stream object)
    _current_stream = torch._C._cuda_getCurrentRawStream  # noqa: F811


def stage_batch(row_start: torch.Tensor, length: torch.Tensor, block_table: torch.Tensor, max_rows: int,
                max_len: int) -> StageBatch:
    """The sequences of a call: int32 row_start [n + 1], length [n] and block_table [n, max_blocks]; no sequence
    has more than max_rows rows or holds more than max_len tokens."""
    device, n = _device(row_start), length.shape[0]
    blocks = block_table.shape[-1]
    raw = _BATCH.pack(n, max_rows, max_len, blocks, _plain(row_start, "row_start", torch.int32, (n + 1,), device),
                      _plain(length, "length", torch.int32, (n,), device),
                      _plain(block_table, "block_table", torch.int32, (n, blocks), device))
    b = StageBatch.from_buffer_copy(raw)
    b.raw, b.device, b.tensors = raw, device, (row_start, length, block_table)
    return b


def stage_norm_rope_append(qkv: torch.Tensor, q_out: torch.Tensor, pool: torch.Tensor, batch: StageBatch,
                           cos: torch.Tensor, sin: torch.Tensor, q_gain: Optional[torch.Tensor] = None,
                           k_gain: Optional[torch.Tensor] = None, eps: float = 1e-5,
                           positions: Optional[torch.Tensor] = None, sections: Optional[Sequence[int]] = None,
                           stream=None) -> torch.Tensor:
    """Norm of the query and key heads of qkv [rows, Hq + 2 Hkv, d], rotation, append to pool; queries to q_out [rows, Hq,
    d].  positions int32 [rows], or [3, rows] with the pairs per axis in ``sections``."""
    if _recording() and (qkv.requires_grad or q_out.requires_grad or pool.requires_grad or cos.requires_grad or sin.requires_grad or
                         (q_gain is not None and q_gain.requires_grad) or (k_gain is not None and k_gain.requires_grad)):
        raise _no_backward()
    device = _device(qkv)
    cache = _cache(pool, device)
    d, hkv = cache[3], cache[2]
    if qkv.dim() != 3 or q_out.dim() != 3:
        raise ValueError("qkv and q_out have three dimensions: rows, heads, head_dim")
    rows, hq, angles = qkv.shape[0], q_out.shape[1], cos.shape[0]
    if qkv.shape != (rows, hq + 2 * hkv, d) or q_out.shape != (rows, hq, d):
        raise ValueError(f"qkv {tuple(qkv.shape)}, q_out {tuple(q_out.shape)} and pool {tuple(pool.shape)} do not fit")
    axes = 1 if positions is None or positions.dim() == 1 else 3
    if positions is not None and (axes == 3) != (sections is not None):
        raise ValueError("positions of three axes come with the pairs of each in sections")
    if sections is not None and (positions is None or len(sections) != 3):
        raise ValueError("sections are three numbers, and come with positions [3, rows]")
    args = _APPEND.pack(
        device, _batch(batch, device), *cache, rows, hq, qkv.data_ptr(), q_out.data_ptr(),
        _row_stride(qkv, "qkv", device), _row_stride(q_out, "q_out", device), _type(qkv), _type(q_out),
        _plain(q_gain, "q_gain", torch.bfloat16, (d,), device), _plain(k_gain, "k_gain", torch.bfloat16, (d,), device),
        eps, angles, _plain(cos, "cos", torch.float32, (angles, d // 2), device),
        _plain(sin, "sin", torch.float32, (angles, d // 2), device),
        _plain(positions, "positions", torch.int32, (rows,) if axes == 1 else (3, rows), device), axes,
        *(sections or (d // 2, 0, 0)))
    if rows:
        rc = lib().stage_norm_rope_append(args, _handle(stream, device))
        if rc:
            _check(rc)
        _keep(stream, qkv, q_out, pool, cos, sin, q_gain, k_gain, positions, *batch.tensors)
    return q_out


def _window_args(q, out, pool, batch, window, sinks, scale):
    if _recording() and (q.requires_grad or out.requires_grad or pool.requires_grad):
        raise _no_backward()
    device = _device(q)
    cache = _cache(pool, device)
    shape = q.shape
    if len(shape) != 3 or out.shape != shape or q.dtype is not out.dtype or shape[2] != cache[3]:
        raise ValueError(f"q {tuple(q.shape)} {q.dtype}, out {tuple(out.shape)} {out.dtype} and pool {tuple(pool.shape)} do not fit")
    return device, _WINDOW.pack(device, _batch(batch, device), *cache, shape[0], shape[1], window, sinks, scale,
                                q.data_ptr(), out.data_ptr(), _row_stride(q, "q", device),
                                _row_stride(out, "out", device), _type(q))


def stage_window_workspace(q: torch.Tensor, out: torch.Tensor, pool: torch.Tensor, batch: StageBatch, window: int = 0,
                           sinks: int = 0) -> int:
    """Bytes of workspace that stage_window_attention takes with these arguments."""
    need = c_int64()
    _check(lib().stage_window_workspace(_window_args(q, out, pool, batch, window, sinks, 0.0)[1], ctypes.byref(need)))
    return need.value


def stage_window_attention(q: torch.Tensor, out: torch.Tensor, pool: torch.Tensor, batch: StageBatch, window: int = 0,
                           sinks: int = 0, scale: float = 0.0, workspace: Optional[torch.Tensor] = None,
                           stream=None) -> torch.Tensor:
    """Attention of q [rows, Hq, d] over pool: positions of the last ``window`` tokens (0: all) and the first ``sinks``."""
    device, args = _window_args(q, out, pool, batch, window, sinks, scale)
    if q.shape[0]:
        L = lib()
        ws, size, keep = _workspace(L.stage_window_workspace, args, device, workspace, stream)
        rc = L.stage_window_attention(args, ws, size, _handle(stream, device))
        if rc:
            _check(rc)
        _keep(stream, q, out, pool, workspace, *batch.tensors)
    return out


def _adapter_args(x, base, out, a, b, ids, ranks, scales):
    if _recording() and (x.requires_grad or base.requires_grad or out.requires_grad or a.requires_grad or b.requires_grad or
                         (scales is not None and scales.requires_grad)):
        raise _no_backward()
    device = _device(x)
    if x.dim() != 2 or base.dim() != 2 or base.shape != out.shape or base.shape[0] != x.shape[0] or \
            not x.dtype is base.dtype is out.dtype or a.dim() != 3:
        raise ValueError(f"x {tuple(x.shape)} {x.dtype}, base {tuple(base.shape)} {base.dtype} and out {tuple(out.shape)} "
                         f"{out.dtype} do not fit")
    (rows, k), n, (count, rank, _) = x.shape, base.shape[1], a.shape
    return device, _ADAPTER.pack(
        device, rows, k, n, count, rank, _type(x), x.data_ptr(), base.data_ptr(), out.data_ptr(),
        _row_stride(x, "x", device), _row_stride(base, "base", device), _row_stride(out, "out", device),
        _plain(a, "a", torch.bfloat16, (count, rank, k), device), _plain(b, "b", torch.bfloat16, (count, n, rank), device),
        _plain(ids, "ids", torch.int32, (rows,), device), _plain(ranks, "ranks", torch.int32, (count,), device),
        _plain(scales, "scales", torch.float32, (count,), device))


def stage_adapter_workspace(x, base, out, a, b, ids, ranks=None, scales=None) -> int:
    """Bytes of workspace that stage_adapter_add takes with these arguments."""
    need = c_int64()
    args = _adapter_args(x, base, out, a, b, ids, ranks, scales)[1]
    _check(lib().stage_adapter_workspace(args, ctypes.byref(need)))
    return need.value


def stage_adapter_add(x: torch.Tensor, base: torch.Tensor, out: torch.Tensor, a: torch.Tensor, b: torch.Tensor,
                      ids: torch.Tensor, ranks: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out [rows, n] = base + scales[i] * b[i] (a[i] x), i = ids of the row: x [rows, k], a [n_adapters, max_rank, k], b
    [n_adapters, n, max_rank]; ids out of range: no adapter."""
    device, args = _adapter_args(x, base, out, a, b, ids, ranks, scales)
    if x.shape[0]:
        L = lib()
        ws, size, keep = _workspace(L.stage_adapter_workspace, args, device, workspace, stream)
        rc = L.stage_adapter_add(args, ws, size, _handle(stream, device))
        if rc:
            _check(rc)
        _keep(stream, x, base, out, a, b, ids, ranks, scales, workspace)
    return out
