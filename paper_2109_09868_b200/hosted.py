"""Binding of the hosted-model operators: linear, per-head norm with rotary positions, attention over a paged cache.

Marshalling only, as in ``binding.py``: tensors become device pointers and element strides in one packed struct (one
foreign-function argument keeps the host time of a single-token call low), and the C entry point of the same name is
called.  There is no fallback: a missing library, a CPU tensor or a layout the library cannot take raises.
"""
from __future__ import annotations

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


def _call(name: str, packed: bytes, device: int, stream) -> None:
    fn = _entry.get(name)
    if fn is None:
        fn = _entry[name] = getattr(load(), name)
    if device != torch._C._cuda_getDevice():
        raise ValueError("%s: the tensors must be on the current CUDA device" % name)
    rc = fn(packed, torch._C._cuda_getCurrentRawStream(device) if stream is None else int(stream.cuda_stream))
    if rc != OK:
        raise ApproxiferError(rc, name)


def _new(like: torch.Tensor, shape, dtype, stream) -> torch.Tensor:
    """An output tensor; where it is written on another stream than the current one, the allocator is told."""
    out = like.new_empty(shape, dtype=dtype)
    if stream is not None:
        out.record_stream(stream)
    return out


def _array(t: torch.Tensor, dtype, shape, name: str, device: int):
    """Address and strides of a CUDA tensor of this type and shape on this device, innermost dimension contiguous."""
    strides = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or (strides[-1] != 1 and shape[-1] > 1):
        raise ValueError("%s must be %s %s on CUDA device %d with a contiguous innermost dimension, got %s %s on %s with strides %s"
                         % (name, dtype, list(shape), device, t.dtype, list(t.shape), t.device, strides))
    return t.data_ptr(), strides


def _vector(t: torch.Tensor, dtype, n: int, name: str, device: int) -> int:
    if t.dtype is not dtype or t.shape != (n,) or t.get_device() != device or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of %d elements on CUDA device %d" % (name, dtype, n, device))
    return t.data_ptr()


def _device(t: torch.Tensor, name: str) -> int:
    device = t.get_device()
    if device < 0 or not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor (the library has no CPU path)" % name)
    return device


def approxifer_linear(X: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, activation: str = "none",
                      residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                      Y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """act(X weight^T + bias) + residual: X [M][K], weight [N][K], bias [N] bfloat16; residual, Y [M][N] of out_dtype
    (bfloat16, the default, or float32).  activation: one of ACTIVATIONS.  Y may be the residual itself."""
    dev = _device(X, "X")
    if X.dim() != 2 or weight.dim() != 2:
        raise ValueError("X must be [M][K] and weight [N][K]")
    M, K = X.shape
    N = weight.shape[0]
    if out_dtype is None:
        out_dtype = torch.bfloat16 if Y is None else Y.dtype
    kind, act = _TYPES.get(out_dtype), ACTIVATIONS.get(activation)
    if kind is None or act is None:
        raise ValueError("out_dtype must be torch.bfloat16 or torch.float32, activation one of %s" % sorted(ACTIVATIONS))
    if Y is None:
        Y = _new(X, (M, N), out_dtype, stream)
    xp, xs = _array(X, torch.bfloat16, (M, K), "X", dev)
    wp, ws = _array(weight, torch.bfloat16, (N, K), "weight", dev)
    yp, ys = _array(Y, out_dtype, (M, N), "Y", dev)
    bp = 0 if bias is None else _vector(bias, torch.bfloat16, N, "bias", dev)
    rp, rs = (0, (0, 1)) if residual is None else _array(residual, out_dtype, (M, N), "residual", dev)
    if M == 1:  # (the row stride of a single row says nothing)
        xs, ys, rs = (max(xs[0], K), 1), (max(ys[0], N), 1), (max(rs[0], N), 1)
    _call("approxifer_linear", _LINEAR.pack(M, N, K, xp, xs[0], wp, max(ws[0], K) if N == 1 else ws[0], bp, rp, rs[0], yp, ys[0], act, kind), dev, stream)
    return Y


def approxifer_qk_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], v: Optional[torch.Tensor], q_weight: Optional[torch.Tensor],
                            k_weight: Optional[torch.Tensor], cos_sin: torch.Tensor, positions: torch.Tensor,
                            k_cache: Optional[torch.Tensor], v_cache: Optional[torch.Tensor], slots: Optional[torch.Tensor],
                            q_out: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                            status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Norm of every head of q [T][Hq][D] and k [T][Hkv][D], then the rotation of positions [T] int32 by the table
    cos_sin [positions][rot] fp32 (rot/2 cosines, then sines); the turned queries are returned, the turned keys and the
    values v are written to slots [T] int64 of k_cache, v_cache [pages][Hkv][page][D] (a negative slot is skipped)."""
    dev = _device(q, "q")
    if q.dim() != 3 or cos_sin.dim() != 2 or not cos_sin.is_contiguous():
        raise ValueError("q must be [T][Hq][D] and cos_sin a contiguous [positions][rot]")
    dt = q.dtype
    T, Hq, D = shape = q.shape
    kind = _TYPES.get(dt)
    if kind is None:
        raise ValueError("q must be torch.bfloat16 or torch.float32")
    if (k is None) != (k_cache is None) or (v is None) != (v_cache is None):
        raise ValueError("k comes with k_cache and v with v_cache")
    cache = k_cache if k_cache is not None else v_cache
    if cache is not None and (cache.dim() != 4 or slots is None):
        raise ValueError("the caches must be [pages][Hkv][page][D], with slots")
    if q_out is None:
        q_out = _new(q, shape, dt, stream)
    pages, Hkv, page = (0, 1, 1) if cache is None else cache.shape[:3]
    qp, qs = _array(q, dt, shape, "q", dev)
    op, os = _array(q_out, dt, shape, "q_out", dev)
    kp, ks = (0, (0, D, 1)) if k is None else _array(k, dt, (T, Hkv, D), "k", dev)
    vp, vs = (0, (0, D, 1)) if v is None else _array(v, dt, (T, Hkv, D), "v", dev)
    kcp, kc = (0, (0, 0, 0, 1)) if k is None else _array(k_cache, dt, (pages, Hkv, page, D), "k_cache", dev)
    vcp, vc = (0, (0, 0, 0, 1)) if v is None else _array(v_cache, dt, (pages, Hkv, page, D), "v_cache", dev)
    rows, rot = cos_sin.shape
    packed = _NORM_ROPE.pack(T, Hq, Hkv, D, rot, 1 if interleaved else 0, kind, qp, qs[0], qs[1], kp, ks[0], ks[1], vp, vs[0], vs[1],
                             0 if q_weight is None else _vector(q_weight, dt, D, "q_weight", dev),
                             0 if k_weight is None else _vector(k_weight, dt, D, "k_weight", dev),
                             _array(cos_sin, torch.float32, (rows, rot), "cos_sin", dev)[0], rows, _vector(positions, torch.int32, T, "positions", dev),
                             op, os[0], os[1], kcp, kc[0], kc[1], kc[2], vcp, vc[0], vc[1], vc[2], pages,
                             0 if slots is None else _vector(slots, torch.int64, T, "slots", dev), page, eps,
                             0 if status is None else _vector(status, torch.int32, T, "status", dev))
    _call("approxifer_qk_norm_rope", packed, dev, stream)
    return q_out


def approxifer_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor, q_start: torch.Tensor,
                         kv_len: torch.Tensor, max_q: int, window: int = 0, sinks: int = 0, scale: Optional[float] = None,
                         out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of the packed queries q [T][Hq][D] over caches [pages][Hkv][page][D]: sequence b has the queries
    q_start[b] .. q_start[b+1]-1 at the last of its kv_len[b] positions, held by the pages block_table[b] (a negative
    entry: a page that was freed).  A query sees the last `window` positions up to its own (0: all) and the first
    `sinks`.  max_q: an upper bound on the queries of a sequence."""
    dev = _device(q, "q")
    if q.dim() != 3 or k_cache.dim() != 4 or block_table.dim() != 2:
        raise ValueError("q must be [T][Hq][D], the caches [pages][Hkv][page][D], block_table [batch][pages]")
    T, Hq, D = q_shape = q.shape
    pages, Hkv, page, _ = k_cache.shape
    batch, table_pages = block_table.shape
    if out is None:
        out = _new(q, q_shape, torch.bfloat16, stream)
    qp, qs = _array(q, torch.bfloat16, q_shape, "q", dev)
    op, os = _array(out, torch.bfloat16, q_shape, "out", dev)
    kp, ks = _array(k_cache, torch.bfloat16, (pages, Hkv, page, D), "k_cache", dev)
    vp, vs = _array(v_cache, torch.bfloat16, (pages, Hkv, page, D), "v_cache", dev)
    tp, ts = _array(block_table, torch.int32, (batch, table_pages), "block_table", dev)
    packed = _ATTENTION.pack(T, batch, max_q, Hq, Hkv, D, page, window, sinks, D ** -0.5 if scale is None else scale, 0, qp, qs[0], qs[1],
                             kp, ks[0], ks[1], ks[2], vp, vs[0], vs[1], vs[2], pages, tp, ts[0], table_pages,
                             _vector(q_start, torch.int32, batch + 1, "q_start", dev), _vector(kv_len, torch.int32, batch, "kv_len", dev),
                             op, os[0], os[1], 0, 0)
    if max_q == 1:
        need = load().approxifer_attention_workspace(packed)
        if need > 0:
            room = _new(q, (need,), torch.uint8, stream)
            packed = packed[:-_WORKSPACE.size] + _WORKSPACE.pack(room.data_ptr(), need)
    _call("approxifer_attention", packed, dev, stream)
    return out
