"""Measured cases of further operators of a hosted decoder model.

Beside its projections, its rotation and its attention over a cache, a worker's time in a hosted decoder goes into

  norm     r' = a r + b act(gate) norm_after(y),  x = norm_before(r')    between two blocks: the end of one, the start of the next
  mx_round the 4-bit microscaled form of an array (32 elements share a power of two) and the values that it stands for
  mx       Y = act(Q(X) Q(W)^T + b) + R with both operands in that form      a projection whose weights are held in 4 bits
  prefix   attention of a batch of sequences that begin with the same long prefix, which lies in the cache once

A prefix that all K queries of a group share is the same in every coded query, since the encoder's weights sum to one: all
workers' sequences share it.  `run` computes the operators in plain elementary operations in 32 bits, or, where `own` is true,
through the package.
"""
import math

import torch

own = False

NORM = dict(op="norm", tokens=1, width=8, stream="bf16", dtype="bf16", after="rms", before="rms", gate="none", gate_act="none", bias=False, a=1.0, b=1.0)
MX_ROUND = dict(op="mx_round", m=1, k=32, dtype="bf16")
MX = dict(op="mx", m=1, n=1, k=32, coded=False, bias=False, act="none", residual=False, out="bf16")
PREFIX = dict(op="prefix", batch=1, q=1, prefix=1, kv=1, ragged=False, hq=1, hkv=1, d=128, page=16)


def listed():
    return [
        # one token between two blocks, normed on both sides and gated: latency
        dict(NORM, name="norm_one_token", width=4096, gate="column"),
        # odd token count and width, layer norms with biases, a gate for every element, fp32
        dict(NORM, name="norm_odd_fp32", tokens=1237, width=1003, stream="fp32", dtype="fp32", after="layer", before="layer", gate="element", gate_act="sigmoid",
             bias=True, a=0.5),
        # a batch of prompts, the stream of residuals held in fp32
        dict(NORM, name="norm_prompts", tokens=16384, width=4096, stream="fp32", gate="column", gate_act="tanh", b=0.7),
        # the rows of a ragged batch, fp32
        dict(MX_ROUND, name="mx_round_ragged_fp32", m=1237, k=2080, dtype="fp32"),
        # a layer's weights
        dict(MX_ROUND, name="mx_round_weights", m=16384, k=4096),
        # one token of one coded sequence through an output projection: latency
        dict(MX, name="mx_one_token", m=1, n=4096, k=4096, residual=True),
        # 20 workers' sequences on one GPU, one token each, through the widening product: reading the weights
        dict(MX, name="mx_20_tokens", m=20, n=16384, k=4096, bias=True, act="gelu"),
        # odd numbers of rows and columns, operands that are both in 4 bits already, fp32 out
        dict(MX, name="mx_odd_coded", m=333, n=1003, k=2080, coded=True, bias=True, out="fp32"),
        # a batch of prompts through the widening product: the largest ordinary matrix product
        dict(MX, name="mx_prompts", m=8192, n=16384, k=4096, bias=True, act="gelu_tanh"),
        # five workers' sequences, one token each, behind a short prefix that ends inside a page, heads of 64
        dict(PREFIX, name="prefix_5_tokens", batch=5, prefix=1003, kv=77, ragged=True, hq=8, hkv=2, d=64),
        # 96 sequences, one token each, behind a long common prefix
        dict(PREFIX, name="prefix_96_tokens", batch=96, prefix=32768, kv=700, ragged=True, hq=32, hkv=8),
        # the workers' own prompts behind a common one
        dict(PREFIX, name="prefix_prompts", batch=8, q=300, prefix=4096, kv=300, ragged=True, hq=32, hkv=8, page=64),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "norm", "mx_round", "mx", "mx", "mx", "prefix", "prefix", "prefix"))
    if op == "norm":
        dtype = rng.choice(("bf16", "bf16", "fp32"))
        after, before = rng.choice((("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("rms", "none"), ("none", "layer")))
        width = rng.choice((8 * _log(rng, 8, 1024), _log(rng, 33, 4096)))
        gate = rng.choice(("none", "column", "token", "element"))
        return dict(NORM, tokens=_log(rng, 1, 8192), width=width, dtype=dtype, stream="fp32" if rng.random() < 0.3 else dtype, after=after, before=before,
                    gate=gate, gate_act="none" if gate == "none" else rng.choice(("none", "sigmoid", "tanh")), bias=rng.random() < 0.5,
                    a=rng.choice((1.0, 0.5, 0.9)), b=rng.choice((1.0, 0.7)))
    if op == "mx_round":
        return dict(MX_ROUND, m=_log(rng, 1, 8192), k=32 * _log(rng, 1, 256), dtype=rng.choice(("bf16", "bf16", "fp32")))
    if op == "mx":
        return dict(MX, m=_log(rng, 1, 8192), n=_log(rng, 10, 16384), k=32 * _log(rng, 2, 128), coded=rng.random() < 0.3, bias=rng.random() < 0.5,
                    act=rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")), residual=rng.random() < 0.5, out=rng.choice(("bf16", "bf16", "fp32")))
    hkv = rng.choice((1, 2, 4, 8))
    case = dict(PREFIX, hkv=hkv, hq=hkv * rng.choice((1, 2, 3, 4, 8)), d=rng.choice((64, 80, 96, 128)), page=rng.choice((16, 32, 64)), ragged=rng.random() < 0.7,
                prefix=_log(rng, 64, 16384))
    if rng.random() < 0.6:  # serving: one token for each sequence
        case.update(batch=_log(rng, 1, 96), kv=_log(rng, 1, 2048))
    else:  # prompts behind the prefix, whole or the last chunk of one
        case.update(batch=rng.choice((2, 3, 5, 8)), q=_log(rng, 2, 300))
        case["kv"] = case["q"] + rng.choice((0, 0, _log(rng, 1, 1024)))
        case["prefix"] = min(case["prefix"], 4096)
    return case


def _lengths(case):
    """Each sequence's own tokens in the cache and its new ones: all alike, or spread down to about a third."""
    kv, q, n = case["kv"], case["q"], case["batch"]
    if not case["ragged"]:
        return [kv] * n, [q] * n
    kvs = [max(1, kv - (b * 7919 * max(1, kv // 97)) % max(1, (2 * kv) // 3)) for b in range(n)]
    return kvs, [min(q, x) for x in kvs]


def _size(name):
    return 4 if name == "fp32" else 2


def _dtype(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def work(case):
    if case["op"] == "norm":
        t, n, s, size = case["tokens"], case["width"], _size(case["stream"]), _size(case["dtype"])
        gate = {"none": 0, "column": n, "token": t, "element": t * n}[case["gate"]]
        vectors = ((case["after"] != "none") + (case["before"] != "none")) * (1 + case["bias"]) * n
        return {"bytes": t * n * (2 * s + size * (1 + (case["before"] != "none"))) + (gate + vectors) * size, "flops": t * n * 14}
    if case["op"] == "mx_round":
        m, k = case["m"], case["k"]
        return {"bytes": m * k * (_size(case["dtype"]) + 2) + m * k // 32, "flops": m * k * 4}
    if case["op"] == "mx":
        m, n, k = case["m"], case["n"], case["k"]
        x = m * k // 2 + m * k // 32 if case["coded"] else 2 * m * k
        return {"bytes": x + n * k // 2 + n * k // 32 + 2 * n * case["bias"] + m * n * _size(case["out"]) * (1 + case["residual"]), "flops": 2 * m * n * k}
    kvs, qs = _lengths(case)
    pairs = sum(q * case["prefix"] + sum(range(kv - q + 1, kv + 1)) for kv, q in zip(kvs, qs))
    rows = case["prefix"] + sum(kvs)  # the prefix is read once for all
    return {"bytes": 2 * 2 * rows * case["hkv"] * case["d"] + 2 * 2 * sum(qs) * case["hq"] * case["d"], "flops": 4 * pairs * case["hq"] * case["d"]}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, std=1.0):
        return torch.empty(shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=g)

    def activations(m, k, dtype=torch.bfloat16):
        """Rows of differing size, a few columns much larger than the others."""
        x = normal(m, k, dtype=dtype)
        x *= torch.exp(normal(m, 1, dtype=torch.float32)).to(dtype)
        x[:, torch.randint(0, k, (max(1, k // 200),), device="cuda", generator=g)] *= 20
        return x

    st = dict(case)
    if case["op"] == "norm":
        t, n, dt = case["tokens"], case["width"], _dtype(case["dtype"])
        st.update(r=normal(t, n, dtype=_dtype(case["stream"]), std=3.0), y=activations(t, n, dt), eps=1e-6)
        for name in ("after", "before"):
            there = case[name] != "none"
            st[name + "_w"] = 1 + normal(n, dtype=dt, std=0.1) if there else None
            st[name + "_b"] = normal(n, dtype=dt, std=0.1) if there and case["bias"] else None
        shape = {"none": None, "column": (n,), "token": (t, 1), "element": (t, n)}[case["gate"]]
        st["g"] = None if shape is None else normal(*shape, dtype=dt)
        return st
    if case["op"] == "mx_round":
        st["x"] = activations(case["m"], case["k"], _dtype(case["dtype"]))
        return st
    if case["op"] == "mx":
        m, n, k = case["m"], case["n"], case["k"]
        out = _dtype(case["out"])
        st.update(x=activations(m, k), xs=None, out_dtype=out)
        st["w"], st["ws"] = _plain_quantize(normal(n, k, std=1 / math.sqrt(k)))
        if case["coded"]:
            st["x"], st["xs"] = _plain_quantize(st["x"])
        st["bias_row"] = normal(n) if case["bias"] else None
        st["r"] = normal(m, n, dtype=out) if case["residual"] else None
        return st
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    kvs, qs = _lengths(case)
    held = [(n + page - 1) // page for n in [case["prefix"]] + kvs]
    order = torch.randperm(sum(held) + 1, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(kvs), max(held[1:])), -1, device="cuda", dtype=torch.int32)
    at = held[0]
    for b, n in enumerate(held[1:]):
        table[b, :n] = order[at: at + n]
        at += n
    starts = [0]
    for q in qs:
        starts.append(starts[-1] + q)
    pages = sum(held) + 1
    st.update(query=normal(starts[-1], hq, d), k_cache=normal(pages, hkv, page, d), v_cache=normal(pages, hkv, page, d), prefix_table=order[: held[0]].clone(),
              table=table, q_start=torch.tensor(starts, device="cuda", dtype=torch.int32), kv_len=torch.tensor(kvs, device="cuda", dtype=torch.int32),
              max_q=max(qs), max_kv=max(kvs), scale=1 / math.sqrt(d))
    return st


def _activation(x, act):
    if act == "relu":
        return x.clamp_min(0)
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    if act == "sigmoid":
        return 1 / (1 + torch.exp(-x))
    if act == "tanh":
        return torch.tanh(x)
    return x


def _plain_row_norm(x, kind, w, b, eps):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + eps) * w.float()
    return x if b is None else x + b.float()


def _plain_norm(st):
    u = _plain_row_norm(st["y"].float(), st["after"], st["after_w"], st["after_b"], st["eps"])
    if st["g"] is not None:
        u = u * _activation(st["g"].float(), st["gate_act"])
    r = st["a"] * st["r"].float() + st["b"] * u
    out = {"residual": r.to(st["r"].dtype)}
    if st["before"] != "none":
        out["next"] = _plain_row_norm(r, st["before"], st["before_w"], st["before_b"], st["eps"]).to(st["y"].dtype)
    return out


# The 4-bit form: of every 32 neighbours in a row, with 2^e <= largest magnitude < 2^(e+1), the scale is 2^(e-2) (the byte e - 2 + 127)
# and each element the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale, ties to the even code, at most 6; two to a byte, the
# first in the low half.  Scales lie in blocks of 128 rows x 4 groups, row r, group k at byte (r % 32) * 16 + (r / 32) * 4 + k.
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _plain_quantize(x):
    m, k = x.shape
    x = x.float().view(m, k // 32, 32)
    top = x.abs().amax(dim=-1)
    byte = torch.where(top > 0, (torch.frexp(top)[1] - 3 + 127).clamp_min(0), 0)
    v = torch.ldexp(x, (127 - byte)[..., None])
    a = v.abs()
    code = (a > 0.25).to(torch.uint8)
    for inclusive, border in ((True, 0.75), (False, 1.25), (True, 1.75), (False, 2.5), (True, 3.5), (False, 5.0)):
        code += (a >= border) if inclusive else (a > border)
    code += 8 * torch.signbit(v)
    code = code.view(m, k // 2, 2)
    codes = code[..., 0] | (code[..., 1] << 4)
    rows, cols = (m + 127) // 128, (k // 32 + 3) // 4
    scales = torch.zeros((rows * 128, cols * 4), device=x.device, dtype=torch.uint8)
    scales[:m, : k // 32] = byte.to(torch.uint8)
    return codes, scales.view(rows, 4, 32, cols, 4).permute(0, 3, 2, 1, 4).reshape(rows, cols, 512)


def _plain_values(codes, scales):
    m, k = codes.shape[0], 2 * codes.shape[1]
    table = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=codes.device)
    v = table[torch.stack([codes & 15, codes >> 4], dim=-1).int()].view(m, k // 32, 32)
    rows, cols = scales.shape[:2]
    byte = scales.view(rows, cols, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rows * 128, cols * 4)[:m, : k // 32]
    return torch.ldexp(v, byte.int()[..., None] - 127).view(m, k)


def _plain_mx(st):
    x = _plain_values(*(_plain_quantize(st["x"]) if st["xs"] is None else (st["x"], st["xs"])))
    y = x @ _plain_values(st["w"], st["ws"]).t()
    if st["bias_row"] is not None:
        y = y + st["bias_row"].float()
    y = _activation(y, st["act"])
    if st["r"] is not None:
        y = y + st["r"].float()
    return y.to(st["out_dtype"])


def _plain_prefix(st):
    batch, hq, hkv, d, page, nq, n = st["batch"], st["hq"], st["hkv"], st["d"], st["page"], st["max_q"], st["prefix"]
    dev, g = st["query"].device, hq // hkv
    kv_len, q_start = st["kv_len"].long(), st["q_start"].long()
    q_len = q_start[1:] - q_start[:-1]
    at = torch.arange(n, device=dev)
    pages = st["prefix_table"].long()[at // page]
    pk, pv = (st[c][pages, :, at % page].float().permute(1, 0, 2) for c in ("k_cache", "v_cache"))  # [hkv][prefix][d]
    at = torch.arange(st["max_kv"], device=dev)
    pages = st["table"].long()[:, at // page].clamp_min(0)
    k, v = (st[c][pages, :, (at % page).expand(batch, -1)].float().transpose(1, 2) for c in ("k_cache", "v_cache"))  # [batch][hkv][own][d]
    token = torch.arange(nq, device=dev)
    q = st["query"][(q_start[:-1, None] + token).clamp_max(st["query"].shape[0] - 1)].float() * st["scale"]  # [batch][nq][hq][d]
    q = q.view(batch, nq, hkv, g, d).permute(2, 0, 3, 1, 4)  # [hkv][batch][g][nq][d]
    common = (q.reshape(hkv, -1, d) @ pk.transpose(1, 2)).view(hkv, batch, g, nq, n)
    mine = (q.reshape(hkv, batch, -1, d) @ k.permute(1, 0, 3, 2)).view(hkv, batch, g, nq, -1)
    pos = (kv_len - q_len)[:, None] + token
    mine = mine.masked_fill_((at > pos[..., None])[None, :, None], -math.inf)
    top = torch.maximum(common.amax(dim=-1, keepdim=True), mine.amax(dim=-1, keepdim=True))
    common, mine = torch.exp_(common.sub_(top)), torch.exp_(mine.sub_(top))
    total = common.sum(dim=-1, keepdim=True) + mine.sum(dim=-1, keepdim=True)
    o = (common.view(hkv, -1, n) @ pv).view(hkv, batch, g, nq, d)
    o += (mine.view(hkv, batch, g * nq, -1) @ v.transpose(0, 1)).view(hkv, batch, g, nq, d)
    o = (o / total).permute(1, 3, 0, 2, 4).reshape(batch, nq, hq, d)
    each = torch.arange(st["query"].shape[0], device=dev)
    seq = torch.bucketize(each, q_start[1:], right=True)
    return o[seq, each - q_start[seq]].to(st["query"].dtype)


def run(st):
    if not own:
        if st["op"] == "mx_round":
            codes, scales = _plain_quantize(st["x"])
            return {"values": _plain_values(codes, scales).to(torch.bfloat16), "scales": scales.view(torch.float8_e8m0fnu)}
        return {"norm": _plain_norm, "mx": _plain_mx, "prefix": _plain_prefix}[st["op"]](st)
    import paper_2109_09868_b200 as ap

    if st["op"] == "norm":
        residual, following = ap.approxifer_block_norm(
            st["r"], st["y"], gate=st["g"], after=None if st["after"] == "none" else st["after"], before=None if st["before"] == "none" else st["before"],
            block_weight=st["after_w"], block_bias=st["after_b"], next_weight=st["before_w"], next_bias=st["before_b"], gate_activation=st["gate_act"],
            residual_scale=st["a"], block_scale=st["b"], eps=st["eps"])
        return {"residual": residual} if following is None else {"residual": residual, "next": following}
    if st["op"] == "mx_round":
        codes, scales = ap.approxifer_mx_quantize(st["x"])
        return {"values": ap.approxifer_mx_dequantize(codes, scales), "scales": scales.view(torch.float8_e8m0fnu)}
    if st["op"] == "mx":
        return ap.approxifer_mx_linear(st["x"], st["w"], st["ws"], x_scales=st["xs"], bias=st["bias_row"], activation=st["act"], residual=st["r"],
                                       out_dtype=st["out_dtype"])
    return ap.approxifer_prefix_attention(st["query"], st["k_cache"], st["v_cache"], st["prefix_table"], st["prefix"], st["table"], st["q_start"],
                                          st["kv_len"], st["max_q"], scale=st["scale"])


def _exact_values(x):
    """The values of the 4-bit form and the scales, by search among all the values that a group can take."""
    m, k = x.shape
    x = x.double().view(-1, 32)
    exponent = (x.abs().amax(dim=1, keepdim=True).view(torch.int64) >> 52) - 1023  # (a 64-bit number's own, by its bits)
    scale = (((exponent - 2).clamp_min(-127) + 1023) << 52).view(torch.float64)
    grid = torch.tensor(_VALUES, device=x.device, dtype=torch.float64)
    a = x.abs() / scale
    hi = torch.bucketize(a, grid).clamp_max(7)  # the first value that is not less
    lo = (hi - 1).clamp_min(0)
    down, up = a - grid[lo], grid[hi] - a
    nearest = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return (torch.where(x < 0, -1.0, 1.0) * grid[nearest] * scale).view(m, k), scale.view(m, -1)


def exact(case, seed):
    """The definitions in 64 bits, written apart from the plain forms."""
    st = prepare(case, seed)
    if case["op"] == "norm":
        def norm(x, kind, w, b):
            if kind == "none":
                return x
            var, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
            if kind == "rms":
                var, mean = var + mean ** 2, 0.0
            return torch.addcmul(torch.zeros((), device="cuda", dtype=torch.float64) if b is None else b.double(), (x - mean) / torch.sqrt(var + st["eps"]), w.double())

        gate = 1.0 if st["g"] is None else {"none": lambda t: t, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[case["gate_act"]](st["g"].double())
        r = case["a"] * st["r"].double() + case["b"] * gate * norm(st["y"].double(), case["after"], st["after_w"], st["after_b"])
        return {"residual": r, **({} if case["before"] == "none" else {"next": norm(r, case["before"], st["before_w"], st["before_b"])})}
    if case["op"] == "mx_round":
        values, scale = _exact_values(st["x"])
        m, groups = scale.shape
        tiles = torch.full(((m + 127) // 128, (groups + 3) // 4, 512), 2.0 ** -127, device="cuda", dtype=torch.float64)
        row, group = torch.arange(m, device="cuda")[:, None], torch.arange(groups, device="cuda")
        tiles[row // 128, group // 4, (row % 32) * 16 + (row // 32) % 4 * 4 + group % 4] = scale
        return {"values": values, "scales": tiles}
    if case["op"] == "mx":
        m, n, k = case["m"], case["n"], case["k"]
        if m * n * k > 1 << 38:
            return None  # 64-bit products of this size would take too long
        w = _plain_values(st["w"], st["ws"]).double()
        x = _exact_values(st["x"])[0] if st["xs"] is None else _plain_values(st["x"], st["xs"]).double()
        y = torch.nn.functional.linear(x, w, None if st["bias_row"] is None else st["bias_row"].double())
        y = {"none": lambda t: t, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
             "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[case["act"]](y)
        return y if st["r"] is None else y + st["r"].double()
    kvs, qs = _lengths(case)
    g, page = case["hq"] // case["hkv"], case["page"]
    if sum(q * (case["prefix"] + kv) for kv, q in zip(kvs, qs)) * case["hq"] * case["d"] > 1 << 37:
        return None  # 64-bit products of this size would take too long
    out, at = torch.empty(st["query"].shape, device="cuda", dtype=torch.float64), 0
    first = torch.arange(case["prefix"], device="cuda")
    for b, (kv, q) in enumerate(zip(kvs, qs)):
        j = torch.arange(kv, device="cuda")
        pages = torch.cat([st["prefix_table"].long()[first // page], st["table"][b].long()[j // page]])
        rows = torch.cat([first % page, j % page])
        place = torch.arange(case["prefix"] + kv, device="cuda")
        hidden = place > torch.arange(case["prefix"] + kv - q, case["prefix"] + kv, device="cuda")[:, None]
        for h in range(case["hkv"]):
            k, v = (st[c][:, h][pages, rows].double() for c in ("k_cache", "v_cache"))
            for i in range(h * g, h * g + g):
                s = (st["query"][at: at + q, i].double() @ k.T) * st["scale"]
                out[at: at + q, i] = torch.softmax(s.masked_fill(hidden, -torch.inf), dim=-1) @ v
        at += q
    return out
