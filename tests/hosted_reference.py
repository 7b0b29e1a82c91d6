"""Plain 64-bit forms of the hosted-model operators (CPU, double), with the bounds their tests allow.

Bounds, from the arithmetic alone (u16 = 2^-8: half a unit in the last of bfloat16's 8 significant bits, relative; u32 =
2^-23: one fp32 operation, whichever way it rounds):
  linear     |err| <= round(|y|) + L (K + 8) u32 S,   S = sum_k |x_k w_k| + |bias| + |r|; each of the K products and sums in
             fp32 errs by at most u32 of a partial sum that S bounds; the activations' slopes are at most L = 1.13 (gelu);
             their own fp32 evaluation is covered by 8 u32 S plus 4 u32 (|z| + 1).
  norm_rope  |err| <= round(|y|) + (D/32 + 32) u32 (|a| + |b|) with a, b the two turned elements: the sum of squares errs by
             at most (D/32 + 6) u32 relative, its root halves that, and scaling, weighting and turning take under 10 more.
  attention  |err| <= u16 |o| + (u16 + 2 d) sum_j p_j |v_j|, d = the error of a score times 2: (D + 8) u32 scale sum |q k| + 4 u32
             |s|; p is rounded to bfloat16 (u16), its exponential's error is below u16.
"""
import math

import torch

U16, U32 = 2.0 ** -8, 2.0 ** -23


def rounding(y, dtype):
    return (U16 if dtype == torch.bfloat16 else U32) * y.abs() + 2.0 ** -130


def linear(x, w, bias, act, residual, out_dtype):
    x, w = x.double(), w.double()
    z, size = x @ w.T, x.abs() @ w.abs().T
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    y = {"none": lambda t: t, "relu": lambda t: t.clamp_min(0), "gelu": lambda t: t * 0.5 * (1 + torch.erf(t / math.sqrt(2))),
         "gelu_tanh": lambda t: 0.5 * t * (1 + torch.tanh(math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3))),
         "silu": lambda t: t * torch.sigmoid(t)}[act](z)
    if residual is not None:
        y, size = y + residual.double(), size + residual.double().abs()
    return y, rounding(y, out_dtype) + 1.13 * (x.shape[1] + 8) * U32 * size + 4 * U32 * (z.abs() + 1)


def norm_rope_rows(x, weight, cos_sin, positions, eps, interleaved):
    """One array of heads [T][H][D] -> (result, bound)."""
    T, H, D = x.shape
    dtype, x = x.dtype, x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    rot = cos_sin.shape[1]
    half = rot // 2
    y, size = x.clone(), x.abs()
    if rot:
        cs = cos_sin.double()[positions.long()]
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            c, s = cs[:, i, None], cs[:, half + i, None]
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., b] * c + x[..., a] * s
            size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, rounding(y, dtype) + (D / 32 + 32) * U32 * size


def attention(q, k_cache, v_cache, block_table, q_start, kv_len, window, sinks, scale):
    """One query and head at a time, only over what it sees -> (result, bound)."""
    T, Hq, D = q.shape
    pages, Hkv, page, _ = k_cache.shape
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    bound = torch.zeros_like(out)
    for b in range(block_table.shape[0]):
        s0, s1, n = int(q_start[b]), int(q_start[b + 1]), int(kv_len[b])
        for t in range(s0, s1):
            p = n - (s1 - t)
            seen = [j for j in range(p + 1) if (window == 0 or j > p - window or j < sinks) and j // page < block_table.shape[1]
                    and 0 <= int(block_table[b, j // page]) < pages]
            if not seen:
                continue
            at = torch.tensor(seen)
            pg, row = block_table[b].long()[at // page], at % page
            for hk in range(Hkv):
                k, v = k_cache[pg, hk, row].double(), v_cache[pg, hk, row].double()
                hs = slice(hk * (Hq // Hkv), (hk + 1) * (Hq // Hkv))
                qq = q[t, hs].double()
                s = qq @ k.T * scale
                w = torch.softmax(s, -1)
                o = w @ v
                d = (D + 8) * U32 * abs(scale) * (qq.abs() @ k.abs().T) + 4 * U32 * s.abs()
                out[t, hs] = o
                bound[t, hs] = U16 * o.abs() + (U16 + 2 * d.amax(-1, keepdim=True)) * (w @ v.abs()) + 2.0 ** -130
    return out, bound
