"""Hosted-model operators: linear, per-head norm with rotary positions, attention over a paged cache.

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
    entries = (lib.approxifer_linear, lib.approxifer_qk_norm_rope, lib.approxifer_attention, lib.approxifer_attention_workspace)
    module.bind(*[ctypes.cast(f, ctypes.c_void_p).value for f in entries], ApproxiferError)
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
