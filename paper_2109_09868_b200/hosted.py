"""Binding of the hosted-model operators: linear, per-head norm with rotary positions, attention over a paged cache.

Marshalling only, as in ``binding.py``: tensors become device pointers and element strides in one packed struct (one
foreign-function argument keeps the host time of a single-token call low), and the C entry point of the same name is
called.  There is no fallback: a missing library, a CPU tensor or a layout the library cannot take raises.
"""
from __future__ import annotations

import math
import struct
from typing import Optional

import torch

from .binding import OK, ApproxiferError, load

TYPE_BF16, TYPE_F32 = 0, 1
_TYPES = {torch.bfloat16: TYPE_BF16, torch.float32: TYPE_F32}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
ST_POSITION, ST_SLOT = 32, 64

_LINEAR = struct.Struct("@qqqPqPqPPqPqii")
_NORM_ROPE = struct.Struct("@qiiiiiiPqqPqqPqqPPPqPPqqPqqqPqqqqPifP")
_ATTENTION = struct.Struct("@qiiiiiiiifiPqqPqqqPqqqqPqqPPPqqPq")
_WORKSPACE = struct.Struct("@Pq")  # the last two fields of the attention arguments

_entry = {}


def _call(name: str, packed: bytes, device: torch.device, stream) -> None:
    fn = _entry.get(name)
    if fn is None:
        fn = _entry[name] = getattr(load(), name)
    if device.index != torch.cuda.current_device():
        raise ValueError("%s: the tensors must be on the current CUDA device" % name)
    handle = torch._C._cuda_getCurrentRawStream(device.index) if stream is None else int(stream.cuda_stream)
    rc = fn(packed, handle)
    if rc != OK:
        raise ApproxiferError(rc, name)


def _new(shape, like: torch.Tensor, dtype, stream) -> torch.Tensor:
    """An output tensor; where it is written on another stream than the current one, the allocator is told."""
    out = torch.empty(shape, dtype=dtype, device=like.device)
    if stream is not None:
        out.record_stream(stream)
    return out


def _check(t: torch.Tensor, dtype, shape, name: str, device: torch.device) -> int:
    """A CUDA tensor of this type and shape on this device, innermost dimension contiguous; its address."""
    if t.device != device or t.dtype != dtype or t.shape != shape or (shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError("%s must be %s %s on %s with a contiguous innermost dimension, got %s %s on %s with strides %s"
                         % (name, dtype, list(shape), device, t.dtype, list(t.shape), t.device, t.stride()))
    return t.data_ptr()


def _vector(t: torch.Tensor, dtype, n: int, name: str, device: torch.device) -> int:
    if t.device != device or t.dtype != dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of %d elements on %s" % (name, dtype, n, device))
    return t.data_ptr()


def approxifer_linear(X: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, activation: str = "none",
                      residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                      Y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """act(X weight^T + bias) + residual: X [M][K], weight [N][K], bias [N] bfloat16; residual, Y [M][N] of out_dtype
    (bfloat16, the default, or float32).  activation: one of ACTIVATIONS.  Y may be the residual itself."""
    if not X.is_cuda:
        raise ValueError("X must be a CUDA tensor (the library has no CPU path)")
    if X.dim() != 2 or weight.dim() != 2:
        raise ValueError("X must be [M][K] and weight [N][K]")
    (M, K), N, dev = X.shape, weight.shape[0], X.device
    if out_dtype is None:
        out_dtype = torch.bfloat16 if Y is None else Y.dtype
    kind, act = _TYPES.get(out_dtype), ACTIVATIONS.get(activation)
    if kind is None or act is None:
        raise ValueError("out_dtype must be torch.bfloat16 or torch.float32, activation one of %s" % sorted(ACTIVATIONS))
    if Y is None:
        Y = _new((M, N), X, out_dtype, stream)
    xp = _check(X, torch.bfloat16, (M, K), "X", dev)
    wp = _check(weight, torch.bfloat16, (N, K), "weight", dev)
    yp = _check(Y, out_dtype, (M, N), "Y", dev)
    bp = 0 if bias is None else _vector(bias, torch.bfloat16, N, "bias", dev)
    rp, rs = (0, 0) if residual is None else (_check(residual, out_dtype, (M, N), "residual", dev), _row(residual, N))
    _call("approxifer_linear", _LINEAR.pack(M, N, K, xp, _row(X, K), wp, _row(weight, K), bp, rp, rs, yp, _row(Y, N), act, kind), dev, stream)
    return Y


def _row(t: torch.Tensor, length: int) -> int:
    """Row stride; of a single row, whose stride says nothing, its length rounded up to whole 16 bytes."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), (length + 7) // 8 * 8)


def approxifer_qk_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], v: Optional[torch.Tensor], q_weight: Optional[torch.Tensor],
                            k_weight: Optional[torch.Tensor], cos_sin: torch.Tensor, positions: torch.Tensor,
                            k_cache: Optional[torch.Tensor], v_cache: Optional[torch.Tensor], slots: Optional[torch.Tensor],
                            q_out: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                            status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Norm of every head of q [T][Hq][D] and k [T][Hkv][D], then the rotation of positions [T] int32 by the table
    cos_sin [positions][rot] fp32 (rot/2 cosines, then sines); the turned queries are returned, the turned keys and the
    values v are written to slots [T] int64 of k_cache, v_cache [pages][Hkv][page][D] (a negative slot is skipped)."""
    if not q.is_cuda:
        raise ValueError("q must be a CUDA tensor (the library has no CPU path)")
    if q.dim() != 3 or cos_sin.dim() != 2:
        raise ValueError("q must be [T][Hq][D] and cos_sin [positions][rot]")
    (T, Hq, D), dev, dt = q.shape, q.device, q.dtype
    kind = _TYPES.get(dt)
    if kind is None:
        raise ValueError("q must be torch.bfloat16 or torch.float32")
    if (k is None) != (k_cache is None) or (v is None) != (v_cache is None):
        raise ValueError("k comes with k_cache and v with v_cache")
    if q_out is None:
        q_out = _new((T, Hq, D), q, dt, stream)
    cache = k_cache if k_cache is not None else v_cache
    if cache is not None and (cache.dim() != 4 or slots is None):
        raise ValueError("the caches must be [pages][Hkv][page][D], with slots")
    pages, Hkv, page = (0, 1, 1) if cache is None else cache.shape[:3]
    if not cos_sin.is_contiguous():
        raise ValueError("cos_sin must be contiguous")
    parts = [_check(q, dt, (T, Hq, D), "q", dev), q.stride(0), q.stride(1)]
    for x, name in ((k, "k"), (v, "v")):
        parts += [0, 0, 0] if x is None else [_check(x, dt, (T, Hkv, D), name, dev), x.stride(0), x.stride(1)]
    parts += [0 if w is None else _vector(w, dt, D, "weight", dev) for w in (q_weight, k_weight)]
    parts += [_check(cos_sin, torch.float32, cos_sin.shape, "cos_sin", dev), cos_sin.shape[0], _vector(positions, torch.int32, T, "positions", dev)]
    parts += [_check(q_out, dt, (T, Hq, D), "q_out", dev), q_out.stride(0), q_out.stride(1)]
    for x, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        parts += [0, 0, 0, 0] if x is None else [_check(x, dt, (pages, Hkv, page, D), name, dev), x.stride(0), x.stride(1), x.stride(2)]
    parts += [pages, 0 if slots is None else _vector(slots, torch.int64, T, "slots", dev), page, eps,
              0 if status is None else _vector(status, torch.int32, T, "status", dev)]
    _call("approxifer_qk_norm_rope", _NORM_ROPE.pack(T, Hq, Hkv, D, cos_sin.shape[1], 1 if interleaved else 0, kind, *parts), dev, stream)
    return q_out


def approxifer_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor, q_start: torch.Tensor,
                         kv_len: torch.Tensor, max_q: int, window: int = 0, sinks: int = 0, scale: Optional[float] = None,
                         out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of the packed queries q [T][Hq][D] over caches [pages][Hkv][page][D]: sequence b has the queries
    q_start[b] .. q_start[b+1]-1 at the last of its kv_len[b] positions, held by the pages block_table[b] (a negative
    entry: a page that was freed).  A query sees the last `window` positions up to its own (0: all) and the first
    `sinks`.  max_q: an upper bound on the queries of a sequence."""
    if not q.is_cuda:
        raise ValueError("q must be a CUDA tensor (the library has no CPU path)")
    if q.dim() != 3 or k_cache.dim() != 4 or block_table.dim() != 2:
        raise ValueError("q must be [T][Hq][D], the caches [pages][Hkv][page][D], block_table [batch][pages]")
    (T, Hq, D), dev = q.shape, q.device
    pages, Hkv, page, _ = k_cache.shape
    batch, table_pages = block_table.shape
    shape = (pages, Hkv, page, D)
    if out is None:
        out = _new((T, Hq, D), q, torch.bfloat16, stream)
    qp, op = _check(q, torch.bfloat16, (T, Hq, D), "q", dev), _check(out, torch.bfloat16, (T, Hq, D), "out", dev)
    kp, vp = _check(k_cache, torch.bfloat16, shape, "k_cache", dev), _check(v_cache, torch.bfloat16, shape, "v_cache", dev)
    tp = _check(block_table, torch.int32, (batch, table_pages), "block_table", dev)
    sp, lp = _vector(q_start, torch.int32, batch + 1, "q_start", dev), _vector(kv_len, torch.int32, batch, "kv_len", dev)
    qs, ks, vs, os = q.stride(), k_cache.stride(), v_cache.stride(), out.stride()
    packed = _ATTENTION.pack(T, batch, max_q, Hq, Hkv, D, page, window, sinks, 1 / math.sqrt(D) if scale is None else scale, 0, qp, qs[0], qs[1],
                             kp, ks[0], ks[1], ks[2], vp, vs[0], vs[1], vs[2], pages, tp, block_table.stride(0), table_pages, sp, lp, op, os[0], os[1], 0, 0)
    if max_q == 1:
        need = load().approxifer_attention_workspace(packed)
        if need > 0:
            room = _new((need,), q, torch.uint8, stream)
            packed = packed[:-_WORKSPACE.size] + _WORKSPACE.pack(room.data_ptr(), need)
    _call("approxifer_attention", packed, dev, stream)
    return out
