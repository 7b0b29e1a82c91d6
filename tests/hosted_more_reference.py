"""Plain 64-bit forms of block_norm, the 4-bit arrays and their product, and the attention behind a prefix (CPU, double), with the
bounds their tests allow.

Bounds, from the arithmetic alone (U16 = 2^-8, U32 = 2^-23 as in hosted_reference):
  block_norm  a row's sum is made of at most 16 terms a thread and ten levels of pairs: 26 U32 relative for squares, half of that
              after the root; with the root itself (2 units), the mean and two or three products less than 24 U32 |z|.  A layer norm's
              mean errs by 27 U32 A, A = the mean magnitude, and the difference is rounded: 30 U32 (A + |x|) k |w| more.  The gate's
              function errs by less than 6 U32 relative, the sum a r + b g u by 4 U32 of its terms.  An error e of r' moves the second
              norm's result by at most k |w| (e + mean e + |c| |e + mean e|_2 / |c|_2), c the (centred) row.
  mx_linear   as hosted_reference.linear: products of 4-bit values and powers of two are exact.
  prefix      as hosted_reference.attention; joining a few partial results adds less than 16 U32 (|o| + sum_j p_j |v_j|).
The 4-bit form itself has no bound: it is compared bit for bit.
"""
import math

import torch

from hosted_reference import U16, U32, linear, rounding  # noqa: F401

VALUES = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def row_norm(x, e, kind, w, b, eps):
    """The norm of x, known up to e -> (result, bound)."""
    if kind is None:
        return x, e
    w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w.double()
    mean = x.mean(-1, keepdim=True) if kind == "layer" else 0.0
    c = x - mean
    k = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    z = c * k * w
    e = e + e.mean(-1, keepdim=True) if kind == "layer" else e
    size = torch.sqrt((c * c).sum(-1, keepdim=True) + x.shape[-1] * eps).clamp_min(1e-300)
    moved = k * w.abs() * (e + c.abs() * torch.sqrt((e * e).sum(-1, keepdim=True)) / size)
    own = 24 * U32 * z.abs()
    if kind == "layer":
        own = own + 30 * U32 * (x.abs().mean(-1, keepdim=True) + x.abs()) * k * w.abs()
    y = z if b is None else z + b.double()
    return y, moved + own + 2 * U32 * (z.abs() + y.abs())


def block_norm(residual, block, gate, block_weight, block_bias, next_weight, next_bias, after, before, gate_activation, residual_scale, block_scale, eps):
    """-> ((r', bound), (x, bound) or None), the bounds without the last rounding of x but with that of r'."""
    r = residual.double()
    zero = torch.zeros_like(r)
    if block is None:
        total, e = r, zero
    else:
        u, eu = row_norm(block.double(), zero, after, block_weight, block_bias, eps)
        g, eg = torch.ones((), dtype=torch.float64), 0.0
        if gate is not None:
            g = {"none": lambda t: t, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[gate_activation](gate.double())
            eg = 6 * U32 if gate_activation != "none" else 0.0
        total = residual_scale * r + block_scale * g * u
        e = abs(block_scale) * g.abs() * (eu + eg * u.abs()) + 4 * U32 * ((residual_scale * r).abs() + (block_scale * g * u).abs())
    first = (total, e + rounding(total, residual.dtype) + U32 * total.abs())
    if before is None:
        return first, None
    x, ex = row_norm(total, e, before, next_weight, next_bias, eps)
    dtype = residual.dtype if block is None and next_weight is None else (block if block is not None else next_weight).dtype
    return first, (x, ex + rounding(x, dtype))


def mx_quantize(x):
    """-> codes [M][K/2], scales [ceil(M/128)][ceil(K/128)][512], byte for byte."""
    m, k = x.shape
    rows, cols = (m + 127) // 128, (k + 127) // 128
    codes = torch.zeros((m, k), dtype=torch.uint8)
    scales = torch.zeros((rows, cols, 512), dtype=torch.uint8)
    x = x.double()
    for g in range(k // 32):
        v = x[:, 32 * g: 32 * g + 32]
        top = v.abs().amax(1)
        byte = torch.zeros(m, dtype=torch.int64)
        for i in range(m):
            t = float(top[i])
            byte[i] = 255 if not math.isfinite(t) else 0 if t == 0 else max(0, math.frexp(t)[1] - 3 + 127)
        unit = torch.pow(torch.tensor(2.0, dtype=torch.float64), byte.double() - 127)[:, None]
        d = ((v / unit).abs()[..., None] - VALUES).abs()
        near = d == d.amin(-1, keepdim=True)
        idx = near.int().argmax(-1)                       # the lower of two that are equally near ...
        other = 7 - near.flip(-1).int().argmax(-1)        # ... and the upper
        idx = torch.where((idx != other) & (idx % 2 == 1), other, idx)
        c = (idx + 8 * torch.signbit(v).long()).to(torch.uint8)
        codes[:, 32 * g: 32 * g + 32] = torch.where((byte == 255)[:, None], torch.zeros_like(c), c)
        for i in range(m):
            scales[i // 128, g // 4, (i % 32) * 16 + (i // 32) % 4 * 4 + g % 4] = int(byte[i])
    return codes[:, 0::2] | (codes[:, 1::2] << 4), scales


def mx_values(codes, scales):
    m, k = codes.shape[0], 2 * codes.shape[1]
    c = torch.stack([codes & 15, codes >> 4], -1).view(m, k).long()
    row, group = torch.arange(m)[:, None], torch.arange(k // 32)
    byte = scales[row // 128, group // 4, (row % 32) * 16 + (row // 32) % 4 * 4 + group % 4].double()
    unit = torch.pow(torch.tensor(2.0, dtype=torch.float64), byte - 127)
    unit[byte == 255] = float("nan")
    return torch.where(c >= 8, -1.0, 1.0) * VALUES[c % 8] * unit.repeat_interleave(32, 1)


def prefix_attention(q, k_cache, v_cache, prefix_table, prefix_len, block_table, q_start, kv_len, scale):
    """One query and head at a time, only over what it sees -> (result, bound)."""
    T, Hq, D = q.shape
    pages, Hkv, page, _ = k_cache.shape
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    bound = torch.zeros_like(out)

    def places(table, count):
        at = torch.arange(min(count, table.shape[0] * page))
        at = at[(table.long()[at // page] >= 0) & (table.long()[at // page] < pages)]
        return table.long()[at // page], at % page

    common = places(prefix_table, prefix_len)
    for b in range(block_table.shape[0]):
        s0, s1, n = int(q_start[b]), int(q_start[b + 1]), int(kv_len[b])
        for t in range(s0, s1):
            p = n - (s1 - t)
            if p < 0:
                continue
            mine = places(block_table[b], p + 1)
            pg, row = torch.cat([common[0], mine[0]]), torch.cat([common[1], mine[1]])
            if len(pg) == 0:
                continue
            for hk in range(Hkv):
                k, v = k_cache[pg, hk, row].double(), v_cache[pg, hk, row].double()
                hs = slice(hk * (Hq // Hkv), (hk + 1) * (Hq // Hkv))
                qq = q[t, hs].double()
                s = qq @ k.T * scale
                w = torch.softmax(s, -1)
                o = w @ v
                d = (D + 8) * U32 * abs(scale) * (qq.abs() @ k.abs().T) + 4 * U32 * s.abs()
                size = w @ v.abs()
                out[t, hs] = o
                bound[t, hs] = U16 * o.abs() + (U16 + 2 * d.amax(-1, keepdim=True)) * size + 16 * U32 * (o.abs() + size) + 2.0 ** -130
    return out, bound
