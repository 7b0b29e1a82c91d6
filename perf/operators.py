"""Measured cases of the operators of a hosted decoder model.

The coded queries of a group go to W workers that all host the same model.  Where that model is a decoder over
sequences, a coded query is a sequence of embeddings and the worker's time goes into three operators:

  linear     Y = act(X W^T + b) + R                    every projection, and the head that gives the predictions
  norm_rope  per-head norm of queries and keys, position rotation, keys and values written to the paged cache
  attention  attention over the paged cache with a sliding window and a few first tokens that stay visible

`run` computes them in plain elementary operations in 32 bits, or, where `own` is true, through the package.
"""
import math

import torch

own = False

LINEAR = dict(op="linear", m=1, n=1, k=8, bias=False, act="none", residual=False, out="bf16")
NORM_ROPE = dict(op="norm_rope", tokens=1, hq=1, hkv=1, d=128, rot=128, interleaved=False, page=16, dtype="bf16")
ATTENTION = dict(op="attention", batch=1, q=1, kv=1, ragged=False, hq=1, hkv=1, d=128, page=16, window=0, sinks=0)


def listed():
    return [
        # one token of one coded sequence through an output projection: the latency of a layer's smallest product
        dict(LINEAR, name="linear_one_token", m=1, n=4096, k=4096, residual=True),
        # 20 workers' sequences on one GPU, one token each, through the widening product: reading the weights
        dict(LINEAR, name="linear_20_tokens", m=20, n=16384, k=4096, bias=True, act="gelu"),
        # the linear stand-in model of the 1x28x28 workload: 256 groups x 5 workers, 784 -> 10 classes in fp32
        dict(LINEAR, name="linear_784_to_10", m=1280, n=10, k=784, bias=True, out="fp32"),
        # a batch of prompts through the widening product: the largest ordinary matrix product
        dict(LINEAR, name="linear_prompts", m=8192, n=16384, k=4096, bias=True, act="gelu_tanh"),
        # one token: latency
        dict(NORM_ROPE, name="norm_rope_one_token", tokens=1, hq=32, hkv=8),
        # odd token count and head counts, partial rotation of neighbouring pairs, fp32
        dict(NORM_ROPE, name="norm_rope_partial_fp32", tokens=1237, hq=15, hkv=5, d=80, rot=48, interleaved=True, dtype="fp32"),
        # a batch of prompts
        dict(NORM_ROPE, name="norm_rope_prompts", tokens=16384, hq=32, hkv=8),
        # one token of one sequence just past its window: latency
        dict(ATTENTION, name="attention_one_token", kv=1500, hq=32, hkv=8, window=1024, sinks=4),
        # 48 sequences of up to 32,768 tokens, one token each, pages that left the window already freed
        dict(ATTENTION, name="attention_48_tokens_window", batch=48, kv=32768, ragged=True, hq=32, hkv=8, window=4096, sinks=4),
        # few long contexts read whole: the work has to be split along the context
        dict(ATTENTION, name="attention_long_context", batch=4, kv=131072, ragged=True, hq=16, hkv=2, d=64, page=64),
        # prompts of odd lengths under a window shorter than they are
        dict(ATTENTION, name="attention_prompts_window", batch=4, q=4096, kv=4096, ragged=True, hq=32, hkv=8, d=64, window=1024, sinks=4),
        # long prompts, causal only: the largest attention
        dict(ATTENTION, name="attention_prompts_long", batch=2, q=8192, kv=8192, hq=32, hkv=4, page=64),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("linear", "linear", "norm_rope", "attention", "attention"))
    if op == "linear":
        case = dict(LINEAR, m=_log(rng, 1, 8192), n=_log(rng, 10, 16384), k=8 * _log(rng, 8, 512), bias=rng.random() < 0.5,
                    act=rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")), residual=rng.random() < 0.5,
                    out=rng.choice(("bf16", "bf16", "fp32")))
        return case
    if op == "norm_rope":
        d = rng.choice((64, 80, 96, 128))
        return dict(NORM_ROPE, tokens=_log(rng, 1, 8192), hq=(hkv := rng.choice((1, 2, 4, 5, 8))) * rng.choice((1, 2, 3, 4)), hkv=hkv, d=d,
                    rot=rng.choice((d, d // 2)), interleaved=rng.random() < 0.3, page=rng.choice((16, 32, 64)),
                    dtype=rng.choice(("bf16", "bf16", "fp32")))
    hkv = rng.choice((1, 2, 4, 8))
    case = dict(ATTENTION, hkv=hkv, hq=hkv * rng.choice((1, 2, 3, 4, 8)), d=rng.choice((64, 80, 96, 128)), page=rng.choice((16, 32, 64)),
                window=rng.choice((0, _log(rng, 64, 4096))), sinks=rng.choice((0, 1, 4, 16)), ragged=rng.random() < 0.7)
    if rng.random() < 0.6:  # serving: one token for each sequence
        case.update(batch=_log(rng, 1, 64), kv=_log(rng, 1, 32768))
    else:  # prompts, whole or the last chunk of one
        case.update(batch=rng.choice((1, 2, 3)), q=_log(rng, 2, 2048))
        case["kv"] = case["q"] + rng.choice((0, 0, _log(rng, 1, 4096)))
    return case


def _lengths(case):
    """Tokens in the cache and new tokens of each sequence: all alike, or spread down to about a third."""
    kv, q, n = case["kv"], case["q"], case["batch"]
    if not case["ragged"]:
        return [kv] * n, [q] * n
    kvs = [max(q if q == 1 else 1, kv - (b * 7919 * max(1, kv // 97)) % max(1, (2 * kv) // 3)) for b in range(n)]
    return kvs, [min(q, x) for x in kvs]


def _visible(case, position):
    """How many cached tokens the query at `position` sees."""
    n, w, s = position + 1, case["window"], case["sinks"]
    return n if not w or n <= w else w + min(s, n - w)


def work(case):
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": 2 * (m * k + n * k) + 2 * n * case["bias"] + m * n * out * (1 + case["residual"]), "flops": 2 * m * n * k}
    if case["op"] == "norm_rope":
        size = 4 if case["dtype"] == "fp32" else 2
        t, heads, d = case["tokens"], case["hq"] + 2 * case["hkv"], case["d"]
        return {"bytes": 2 * t * heads * d * size + 2 * d * size + t * (case["rot"] * 4 + 12), "flops": t * heads * d * 7}
    kvs, qs = _lengths(case)
    read = pairs = 0
    for kv, q in zip(kvs, qs):
        read += min(kv, _visible(case, kv - q) + q - 1 if case["window"] else kv)
        pairs += sum(_visible(case, p) for p in range(kv - q, kv))
    return {"bytes": 2 * 2 * read * case["hkv"] * case["d"] + 2 * 2 * sum(qs) * case["hq"] * case["d"], "flops": 4 * pairs * case["hq"] * case["d"]}


def _dtype(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, std=1.0):
        return torch.empty(shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=g)

    st = dict(case)
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        out = _dtype(case["out"])
        st.update(x=normal(m, k), w=normal(n, k, std=1 / math.sqrt(k)), out_dtype=out)
        st["b"] = normal(n) if case["bias"] else None
        st["r"] = normal(m, n, dtype=out) if case["residual"] else None
        return st
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    if case["op"] == "norm_rope":
        t, dt, longest = case["tokens"], _dtype(case["dtype"]), 32768
        qkv = normal(t, (hq + 2 * hkv) * d, dtype=dt)  # one projection's output; the three parts are views of it
        q, k, v = qkv.split([hq * d, hkv * d, hkv * d], dim=1)
        pages = (t + page - 1) // page + 3
        angle = torch.arange(longest, device="cuda", dtype=torch.float64)[:, None] * (
            10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"]))
        st.update(q=q.view(t, hq, d), k=k.view(t, hkv, d), v=v.view(t, hkv, d), eps=1e-6,
                  qw=1 + normal(d, dtype=dt, std=0.1), kw=1 + normal(d, dtype=dt, std=0.1),
                  cos_sin=torch.cat([angle.cos(), angle.sin()], dim=1).float(),
                  positions=torch.randint(0, longest, (t,), device="cuda", dtype=torch.int32, generator=g),
                  slots=torch.randperm(pages * page, device="cuda", generator=g)[:t],
                  k_cache=normal(pages, hkv, page, d, dtype=dt), v_cache=normal(pages, hkv, page, d, dtype=dt))
        return st
    kvs, qs = _lengths(case)
    # pages of positions that no query of the call sees any more are freed: their entries hold -1
    held = []
    for kv, q in zip(kvs, qs):
        first = 0 if not case["window"] else max(0, kv - q + 1 - case["window"])
        held.append([p for p in range((kv + page - 1) // page) if (p + 1) * page > first or p * page < case["sinks"]])
    pages = sum(map(len, held)) + 1
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    at, rows, cols = 0, [], []
    for b, ps in enumerate(held):
        rows += [b] * len(ps)
        cols += ps
    table = torch.full((len(kvs), (max(kvs) + page - 1) // page), -1, device="cuda", dtype=torch.int32)
    table[torch.tensor(rows, device="cuda"), torch.tensor(cols, device="cuda")] = order[: len(rows)]
    starts = [0]
    for q in qs:
        starts.append(starts[-1] + q)
    st.update(query=normal(starts[-1], hq, d), k_cache=normal(pages, hkv, page, d), v_cache=normal(pages, hkv, page, d), table=table,
              q_start=torch.tensor(starts, device="cuda", dtype=torch.int32), kv_len=torch.tensor(kvs, device="cuda", dtype=torch.int32),
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
    return x


def _plain_linear(st):
    y = st["x"].float() @ st["w"].float().t()
    if st["b"] is not None:
        y = y + st["b"].float()
    y = _activation(y, st["act"])
    if st["r"] is not None:
        y = y + st["r"].float()
    return y.to(st["out_dtype"])


def _plain_norm_rope_rows(x, w, cos, sin, st):
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + st["eps"]) * w.float()
    rot, half = st["rot"], st["rot"] // 2
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if st["interleaved"] else (x[..., :half], x[..., half:rot])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], dim=-1).flatten(-2) if st["interleaved"] else torch.cat([u, v], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_norm_rope(st):
    cos, sin = st["cos_sin"][st["positions"].long()][:, None, :].chunk(2, dim=-1)
    q = _plain_norm_rope_rows(st["q"], st["qw"], cos, sin, st).to(st["q"].dtype)
    k = _plain_norm_rope_rows(st["k"], st["kw"], cos, sin, st).to(st["k"].dtype)
    page, row = st["slots"] // st["page"], st["slots"] % st["page"]
    st["k_cache"][page, :, row] = k
    st["v_cache"][page, :, row] = st["v"]
    return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _plain_attention(st):
    batch, hq, hkv, d, page = st["table"].shape[0], st["hq"], st["hkv"], st["d"], st["page"]
    window, sinks, nq, dev = st["window"], st["sinks"], st["max_q"], st["query"].device
    kv_len, q_start = st["kv_len"].long(), st["q_start"].long()
    q_len = q_start[1:] - q_start[:-1]
    # the span of positions that any query of a sequence sees: the window of its first one up to its last, and the sinks
    if window and window + nq - 1 + sinks < st["max_kv"]:
        first = (kv_len - q_len + 1 - window).clamp_min(sinks)
        at = first[:, None] + torch.arange(window + nq - 1, device=dev)
        at = torch.cat([torch.arange(sinks, device=dev).expand(batch, sinks), at], dim=1)
    else:
        at = torch.arange(st["max_kv"], device=dev).expand(batch, st["max_kv"])
    pages = st["table"].long().gather(1, (at // page).clamp_max(st["table"].shape[1] - 1))
    there = (at < kv_len[:, None]) & (pages >= 0)
    pages, row = pages.clamp_min(0), at % page
    k = st["k_cache"][pages, :, row].float().permute(0, 2, 3, 1)  # [batch][hkv][d][span]
    v = st["v_cache"][pages, :, row].float().transpose(1, 2)  # [batch][hkv][span][d]
    token = torch.arange(nq, device=dev)
    q = st["query"][(q_start[:-1, None] + token).clamp_max(st["query"].shape[0] - 1)].float()  # [batch][nq][hq][d]
    q = q.view(batch, nq, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(batch, hkv, -1, d)
    s = ((q * st["scale"]) @ k).view(batch, hkv, hq // hkv, nq, -1)
    pos = (kv_len - q_len)[:, None] + token  # [batch][nq]
    seen = there[:, None, :] & (at[:, None, :] <= pos[:, :, None])
    if window:
        seen &= (at[:, None, :] > pos[:, :, None] - window) | (at[:, None, :] < sinks)
    seen = seen[:, None, None]
    s = s.masked_fill_(~seen, -math.inf)
    p = torch.exp_(s.sub_(s.amax(dim=-1, keepdim=True).clamp_min_(-3e38)))
    total = p.sum(dim=-1, keepdim=True)
    o = (p.view(batch, hkv, -1, p.shape[-1]) @ v).view(batch, hkv, hq // hkv, nq, d) / total.clamp_min(1e-37)
    o = o.permute(0, 3, 1, 2, 4).reshape(batch, nq, hq, d)
    each = torch.arange(st["query"].shape[0], device=dev)
    seq = torch.bucketize(each, q_start[1:], right=True)
    return o[seq, each - q_start[seq]].to(st["query"].dtype)


def run(st):
    if not own:
        return {"linear": _plain_linear, "norm_rope": _plain_norm_rope, "attention": _plain_attention}[st["op"]](st)
    import paper_2109_09868_b200 as ap

    if st["op"] == "linear":
        return ap.approxifer_linear(st["x"], st["w"], bias=st["b"], activation=st["act"], residual=st["r"], out_dtype=st["out_dtype"])
    if st["op"] == "norm_rope":
        q = ap.approxifer_qk_norm_rope(st["q"], st["k"], st["v"], st["qw"], st["kw"], st["cos_sin"], st["positions"], st["k_cache"],
                                       st["v_cache"], st["slots"], eps=st["eps"], interleaved=st["interleaved"])
        return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    return ap.approxifer_attention(st["query"], st["k_cache"], st["v_cache"], st["table"], st["q_start"], st["kv_len"], st["max_q"],
                                   window=st["window"], sinks=st["sinks"], scale=st["scale"])


def exact(case, seed):
    """The definitions in 64 bits, written apart from the plain forms: row blocks, complex rotations, one sequence and head at a time."""
    st = prepare(case, seed)
    if case["op"] == "linear":
        w = st["w"].double()
        y = torch.cat([torch.nn.functional.linear(x.double(), w, None if st["b"] is None else st["b"].double()) for x in st["x"].split(1024)])
        y = {"none": lambda t: t, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
             "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[case["act"]](y)
        return y if st["r"] is None else y + st["r"].double()
    if case["op"] == "norm_rope":
        half = case["rot"] // 2
        turn = torch.complex(st["cos_sin"][:, :half].double(), st["cos_sin"][:, half:].double())[st["positions"].long()][:, None]

        def rows(x, w):
            x = x.double()
            x = x / torch.linalg.vector_norm(x, dim=-1, keepdim=True).pow(2).div(x.shape[-1]).add(st["eps"]).sqrt() * w.double()
            z = x[..., : case["rot"]]
            z = torch.view_as_complex(z.unflatten(-1, (-1, 2)).contiguous()) if case["interleaved"] else torch.complex(z[..., :half], z[..., half:])
            z = z * turn
            z = torch.view_as_real(z).flatten(-2) if case["interleaved"] else torch.cat([z.real, z.imag], -1)
            return torch.cat([z, x[..., case["rot"]:]], -1)

        caches = {}
        for name, new in (("k_cache", rows(st["k"], st["kw"])), ("v_cache", st["v"].double())):
            flat = st[name].double().transpose(1, 2).flatten(0, 1)  # [slot][hkv][d]
            flat[st["slots"]] = new
            caches[name] = flat.unflatten(0, (-1, case["page"])).transpose(1, 2).contiguous()
        return {"q": rows(st["q"], st["qw"]), **caches}
    kvs, qs = _lengths(case)
    g, window, sinks, page = case["hq"] // case["hkv"], case["window"], case["sinks"], case["page"]
    if sum(kv * q for kv, q in zip(kvs, qs)) * case["hq"] > 1 << 33:
        return None  # 64-bit products of the longest prompts would take too long
    out, at = torch.empty(st["query"].shape, device="cuda", dtype=torch.float64), 0
    for b, (kv, q) in enumerate(zip(kvs, qs)):
        lo = max(0, kv - q + 1 - window) if window else 0
        keep = torch.tensor([j for j in range(min(sinks, lo))] + list(range(lo, kv)), device="cuda")
        slot = st["table"][b].long()[keep // page], keep % page
        pos = torch.arange(kv - q, kv, device="cuda")[:, None]
        hidden = keep > pos
        if window:
            hidden |= (keep <= pos - window) & (keep >= sinks)
        for h in range(case["hkv"]):
            k, v = (st[c][:, h][slot].double() for c in ("k_cache", "v_cache"))
            for i in range(h * g, h * g + g):
                s = (st["query"][at: at + q, i].double() @ k.T) * st["scale"]
                out[at: at + q, i] = torch.softmax(s.masked_fill(hidden, -torch.inf), dim=-1) @ v
        at += q
    return out
