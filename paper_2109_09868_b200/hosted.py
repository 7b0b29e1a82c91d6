"""Hosted-model operators: linear, per-head norm with rotary positions, attention over a paged cache, also behind a common prefix,
norms around a block, 4-bit microscaled arrays and products.

The calls go through ``_hosted`` (``csrc/hosted_binding.cpp``), which marshals tensors into the C structs of
``include/approxifer.h`` and calls the C entry point of the same name: in C++, because a single-token call is short enough
for marshalling in Python to cost more than the call.  There is no fallback: a missing library, a CPU tensor or a layout the
library cannot take raises.

``stream``: the stream that the work is enqueued on (None: the current one).  As everywhere in CUDA it is the caller who makes it
wait for what the inputs come from, and who waits for it before the outputs are used elsewhere.  An output that is not given is
allocated on that stream, so its memory is free there, and kept for the current stream too.  The operators serve: they compute no
gradients, and their outputs have none, whatever the inputs ask for.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import shutil
from typing import Optional

import torch

from . import build as _build
from .binding import ApproxiferError, load

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
NORMS = {None: 0, "rms": 1, "layer": 2}
GATE_ACTIVATIONS = {"none": 0, "sigmoid": 1, "tanh": 2}
ST_POSITION, ST_SLOT = 32, 64

_native = None


def _load():
    """The native binding, with the loaded library's entry points."""
    global _native
    lib = load()
    have_compilers = shutil.which("g++") is not None and (shutil.which("nvcc") is not None or os.path.exists("/usr/local/cuda/bin/nvcc"))
    if have_compilers and _build.binding_is_stale():
        _build.build_binding()
    if not os.path.exists(_build.BINDING):
        raise RuntimeError("_hosted.so is missing and cannot be built (no g++ or no CUDA headers): run `python -m paper_2109_09868_b200.build`")
    loader = importlib.machinery.ExtensionFileLoader("_hosted", _build.BINDING)
    module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_hosted", loader))
    loader.exec_module(module)
    entries = (lib.approxifer_linear, lib.approxifer_qk_norm_rope, lib.approxifer_attention, lib.approxifer_attention_workspace, lib.approxifer_block_norm,
               lib.approxifer_mx_quantize, lib.approxifer_mx_dequantize, lib.approxifer_mx_linear, lib.approxifer_mx_linear_workspace,
               lib.approxifer_prefix_attention, lib.approxifer_prefix_attention_workspace)
    module.bind(ApproxiferError, *[ctypes.cast(f, ctypes.c_void_p).value for f in entries])
    _native = module
    return module


def _on(stream, call, given, *args) -> torch.Tensor:
    """``call`` on a stream that need not be the current one.  A new output is taken from that stream's memory: a block of the
    current stream's may still be in use there by work that `stream` does not wait for."""
    if given is not None:
        return call(*args, int(stream.cuda_stream))
    user = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        out = call(*args, int(stream.cuda_stream))
    out.record_stream(user)  # (it is used there: its memory goes back to `stream` only after that)
    return out


def _all_on(stream, call, given, *args):
    """As `_on`, for calls that may allocate more than one output, or a workspace (which the allocator's order on that stream then
    makes safe).  `given`: the outputs that the caller brought, None for each of the others."""
    user = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        out = call(*args, int(stream.cuda_stream))
    for tensor, brought in zip(out if isinstance(out, tuple) else (out,), given):
        if tensor is not None and brought is None:
            tensor.record_stream(user)
    return out


def _code(names, name, what):
    code = names.get(name)
    if code is None:
        raise ValueError("%s must be one of %s" % (what, sorted(names, key=str)))
    return code


def approxifer_linear(X: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, activation: str = "none",
                      residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                      Y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """act(X weight^T + bias) + residual: X [M][K], weight [N][K], bias [N] bfloat16; residual, Y [M][N] of out_dtype
    (bfloat16, the default, or float32).  activation: one of ACTIVATIONS.  Y may be the residual itself."""
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError("activation must be one of %s" % sorted(ACTIVATIONS))
    args = (X, weight, bias, act, residual, out_dtype, Y)
    if stream is None:
        return (_native or _load()).linear(*args, None)
    return _on(stream, (_native or _load()).linear, Y, *args)


def approxifer_qk_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], v: Optional[torch.Tensor], q_weight: Optional[torch.Tensor],
                            k_weight: Optional[torch.Tensor], cos_sin: torch.Tensor, positions: torch.Tensor,
                            k_cache: Optional[torch.Tensor], v_cache: Optional[torch.Tensor], slots: Optional[torch.Tensor],
                            q_out: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                            status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Norm of every head of q [T][Hq][D] and k [T][Hkv][D], then the rotation of positions [T] int32 by the table
    cos_sin [positions][rot] fp32 (rot/2 cosines, then sines); the turned queries are returned, the turned keys and the
    values v are written to slots [T] int64 of k_cache, v_cache [pages][Hkv][page][D] (a negative slot is skipped)."""
    args = (q, k, v, q_weight, k_weight, cos_sin, positions, k_cache, v_cache, slots, q_out, eps, interleaved, status)
    if stream is None:
        return (_native or _load()).norm_rope(*args, None)
    return _on(stream, (_native or _load()).norm_rope, q_out, *args)


def approxifer_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor, q_start: torch.Tensor,
                         kv_len: torch.Tensor, max_q: int, window: int = 0, sinks: int = 0, scale: Optional[float] = None,
                         out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of the packed queries q [T][Hq][D] over caches [pages][Hkv][page][D]: sequence b has the queries
    q_start[b] .. q_start[b+1]-1 at the last of its kv_len[b] positions, held by the pages block_table[b] (a negative
    entry: a page that was freed).  A query sees the last `window` positions up to its own (0: all) and the first
    `sinks`.  max_q: an upper bound on the queries of a sequence.  workspace: CUDA memory for large single-token calls
    (allocated where it is needed and not given, except with `stream`: such a call runs without it)."""
    args = (q, k_cache, v_cache, block_table, q_start, kv_len, max_q, window, sinks, scale, out, workspace)
    if stream is None:
        return (_native or _load()).attention(*args, None)
    return _on(stream, (_native or _load()).attention, out, *args)


def approxifer_prefix_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, prefix_table: torch.Tensor, prefix_len: int,
                                block_table: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, max_q: int, scale: Optional[float] = None,
                                out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """As approxifer_attention, for sequences that begin with the same prefix of `prefix_len` positions, which lies in the pages
    prefix_table [pages] int32 once and, but in small calls, is read once for all.  block_table and kv_len say of each sequence what follows the
    prefix; every query sees the prefix and its sequence's own positions up to itself.  workspace: CUDA memory (allocated
    where it is not given)."""
    args = (q, k_cache, v_cache, prefix_table, prefix_len, block_table, q_start, kv_len, max_q, scale, out, workspace)
    if stream is None:
        return (_native or _load()).prefix_attention(*args, None)
    return _all_on(stream, (_native or _load()).prefix_attention, (out,), *args)


def approxifer_block_norm(residual: torch.Tensor, block: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                          block_weight: Optional[torch.Tensor] = None, block_bias: Optional[torch.Tensor] = None, next_weight: Optional[torch.Tensor] = None,
                          next_bias: Optional[torch.Tensor] = None, after: Optional[str] = None, before: Optional[str] = "rms", gate_activation: str = "none",
                          residual_scale: float = 1.0, block_scale: float = 1.0, eps: float = 1e-6, residual_out: Optional[torch.Tensor] = None,
                          next_out: Optional[torch.Tensor] = None, stream=None):
    """r' = residual_scale residual + block_scale act(gate) norm_after(block) and x = norm_before(r') -> (r', x).
    residual [T][N] bfloat16 or float32; block [T][N], the weights and biases [N] and the gate ([N], [T][1] or [T][N]) bfloat16 or
    float32, all alike, as is x.  after, before: "rms", "layer" or None (no such norm; without the second x is None).  Without a block
    r' is `residual` itself.  residual_out may be `residual`, next_out may be `block`."""
    args = (residual, block, gate, block_weight, block_bias, next_weight, next_bias, _code(NORMS, after, "after"), _code(NORMS, before, "before"),
            _code(GATE_ACTIVATIONS, gate_activation, "gate_activation"), residual_scale, block_scale, eps, residual_out, next_out)
    if stream is None:
        return (_native or _load()).block_norm(*args, None)
    return _all_on(stream, (_native or _load()).block_norm, (residual if block is None else residual_out, next_out), *args)


def approxifer_mx_quantize(X: torch.Tensor, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None, stream=None):
    """The 4-bit microscaled form of X [M][K] bfloat16 or float32, K a multiple of 32 -> (codes [M][K/2] uint8, scales
    [ceil(M/128)][ceil(K/128)][512] uint8): 32 neighbours share a power of two, an element is 0, 0.5, 1, 1.5, 2, 3, 4 or 6 times it.
    Given codes must have rows of whole 16 bytes."""
    if stream is None:
        return (_native or _load()).mx_quantize(X, codes, scales, None)
    return _all_on(stream, (_native or _load()).mx_quantize, (codes, scales), X, codes, scales)


def approxifer_mx_dequantize(codes: torch.Tensor, scales: torch.Tensor, out_dtype: Optional[torch.dtype] = None, X: Optional[torch.Tensor] = None,
                             stream=None) -> torch.Tensor:
    """What approxifer_mx_quantize's codes and scales stand for: [M][K] of out_dtype (bfloat16, the default, or float32)."""
    if stream is None:
        return (_native or _load()).mx_dequantize(codes, scales, out_dtype, X, None)
    return _all_on(stream, (_native or _load()).mx_dequantize, (X,), codes, scales, out_dtype, X)


def approxifer_mx_linear(X: torch.Tensor, weight: torch.Tensor, weight_scales: torch.Tensor, bias: Optional[torch.Tensor] = None, activation: str = "none",
                         residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None, Y: Optional[torch.Tensor] = None,
                         x_scales: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """act(Q(X) weight^T + bias) + residual with both operands in the 4-bit form of approxifer_mx_quantize: weight [N][K/2] codes
    with weight_scales; X [M][K] bfloat16, brought into that form within the call, or, with x_scales, [M][K/2] codes.  The rest as
    for approxifer_linear.  workspace: CUDA memory (allocated where it is needed and not given)."""
    args = (X, weight, weight_scales, x_scales, bias, _code(ACTIVATIONS, activation, "activation"), residual, out_dtype, Y, workspace)
    if stream is None:
        return (_native or _load()).mx_linear(*args, None)
    return _all_on(stream, (_native or _load()).mx_linear, (Y,), *args)
