"""approxifer_prefix_attention against its 64-bit plain form: prefix and own lengths, head layouts, pages, tables, strides."""
import pytest
import torch

import hosted_more_reference as ref
import paper_2109_09868_b200 as ap

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def normal(shape, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(BF)


def problem(prefix, kv, qs, Hq, Hkv, D, page, seed=0, spare=3, short=()):
    """Queries, caches and tables; `short`: pages (prefix pages first, then each sequence's) whose entry says that nothing is there."""
    g = torch.Generator().manual_seed(seed)
    held = [(n + page - 1) // page for n in [prefix] + kv]
    pages = sum(held) + spare
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(kv), max(held[1:] + [1])), -1, dtype=torch.int32)
    at = held[0]
    for b, n in enumerate(held[1:]):
        table[b, :n] = order[at: at + n]
        at += n
    first = order[: held[0]].clone()
    for where, entry, value in short:
        (first if where < 0 else table[where])[entry] = value
    start = torch.tensor([0] + list(torch.tensor(qs).cumsum(0)), dtype=torch.int32)
    return dict(q=normal((int(start[-1]), Hq, D), seed + 1), k_cache=normal((pages, Hkv, page, D), seed + 2), v_cache=normal((pages, Hkv, page, D), seed + 3),
                prefix_table=first, prefix_len=prefix, block_table=table, q_start=start, kv_len=torch.tensor(kv, dtype=torch.int32))


def run(p, max_q=None, scale=0.1, **more):
    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in p.items()}
    qs = (p["q_start"][1:] - p["q_start"][:-1]).max() if max_q is None else max_q
    return ap.approxifer_prefix_attention(**dev, max_q=int(qs), scale=scale, **more)


def check(got, want, bound):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    over = ((got - want).abs() - bound).max()
    assert over <= 0, float(over)
    assert ap.device_wait_timeouts() == 0


CASES = [  # prefix, own lengths, new tokens, Hq, Hkv, D, page
    (1, [1], [1], 1, 1, 8, 16),
    (1003, [77, 5, 31, 1, 50], [1] * 5, 8, 2, 64, 16),
    (1000, [1, 2, 3], [1, 1, 1], 4, 4, 128, 16),
    (4096, [300] * 7, [1] * 7, 32, 4, 128, 64),
    (5000, [700, 1, 20], [1, 1, 1], 15, 5, 80, 32),
    (127, [33, 90], [1, 1], 6, 2, 96, 8),
    (128, [33, 90], [1, 1], 6, 2, 96, 128),
    (129, [1, 1], [1, 1], 8, 1, 72, 256),
    (0, [33, 90], [1, 1], 6, 2, 64, 16),
    (3000, [100] * 40, [1] * 40, 4, 1, 64, 16),         # rows of several tiles for one key head
    (2500, [40] * 70, [1] * 70, 8, 2, 128, 16),
    (700, [20, 130, 300], [20, 130, 200], 8, 2, 64, 16),  # prompts
    (700, [20, 130, 300], [20, 130, 200], 8, 2, 128, 64),
    (260, [1, 5, 40, 64], [1, 3, 40, 2], 5, 1, 40, 8),
    (1500, [600], [500], 4, 2, 128, 32),
    (64, [2, 1, 9], [2, 1, 9], 24, 1, 128, 16),
    (300, [12, 7], [1, 0], 4, 2, 64, 16),                # a sequence without a new token
    (300, [5, 7, 0], [1, 1, 1], 4, 2, 64, 16),           # and one without a cached one
    (300, [5, 7, 2], [3, 9, 2], 4, 2, 64, 16),           # fewer cached tokens than new ones
    (50, [13, 29], [1, 1], 3, 3, 33, 5),                 # odd heads and pages: the element-wise kernel
    (50, [13, 29], [4, 29], 3, 1, 33, 7),
    (90, [13, 29], [4, 2], 2, 1, 200, 16),
]


@pytest.mark.parametrize("prefix,kv,qs,Hq,Hkv,D,page", CASES)
def test_prefix_attention_matches_the_plain_form(prefix, kv, qs, Hq, Hkv, D, page):
    p = problem(prefix, kv, qs, Hq, Hkv, D, page)
    want, bound = ref.prefix_attention(**p, scale=0.1)
    check(run(p), want, bound)
    check(run(p, max_q=max(qs) + 3), want, bound)  # a loose bound on the queries


@pytest.mark.parametrize("qs", [[1, 1, 1], [1, 40, 9]])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
def test_prefix_attention_scales(qs, scale):
    p = problem(400, [60, 90, 33], qs, 8, 2, 64, 16)
    want, bound = ref.prefix_attention(**p, scale=scale)
    check(run(p, scale=scale), want, bound)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("qs", [[1, 1, 1], [1, 40, 9]])
def test_prefix_attention_pages_that_hold_nothing(qs, D):
    for short in ([(-1, 3, -1), (-1, 10, 1000000), (0, 1, -5)], [(-1, i, -1) for i in range(25)], [(0, i, -1) for i in range(4)] + [(2, i, -7) for i in range(3)],
                  [(-1, i, -1) for i in range(25)] + [(0, i, -1) for i in range(4)]):
        p = problem(400, [60, 90, 33], qs, 8, 2, D, 16, short=short)
        p["block_table"][p["block_table"] == -1] = -1
        want, bound = ref.prefix_attention(**p, scale=0.1)
        check(run(p), want, bound)
    # tables that end early, and a prefix longer than its table
    p = problem(400, [60, 90, 33], qs, 8, 2, D, 16)
    p["prefix_table"], p["block_table"] = p["prefix_table"][:7], p["block_table"][:, :2].contiguous()
    want, bound = ref.prefix_attention(**p, scale=0.1)
    check(run(p), want, bound)
    p["prefix_table"], p["prefix_len"] = p["prefix_table"][:0], 0
    want, bound = ref.prefix_attention(**p, scale=0.1)
    check(run(p), want, bound)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("qs", [[1, 1, 1], [1, 40, 9]])
def test_prefix_attention_what_is_not_seen_has_no_influence(qs, D):
    """NaN and infinities behind the prefix's end in its last page, behind the sequences' ends, and in pages that no table names."""
    p = problem(403, [60, 90, 33], qs, 8, 2, D, 16)
    want, bound = ref.prefix_attention(**p, scale=0.1)
    named = torch.zeros(p["k_cache"].shape[0], 16, dtype=torch.bool)
    for table, n in [(p["prefix_table"], 403)] + [(p["block_table"][b], int(p["kv_len"][b])) for b in range(3)]:
        at = torch.arange(n)
        named[table.long()[at // 16], at % 16] = True
    for name, bad in (("k_cache", float("nan")), ("v_cache", float("inf"))):
        c = p[name].transpose(1, 2)
        c[~named] = bad
    check(run(p), want, bound)
    # a NaN that is seen reaches those that see it: of the prefix all, of a sequence its own from there on
    p["v_cache"][p["prefix_table"][5], 1, 3, 2] = float("nan")
    got = run(p).double().cpu()
    assert torch.isnan(got[:, 4:, 2]).all() and not torch.isnan(got[:, :4]).any() and not torch.isnan(got[:, :, 3:]).any()


@pytest.mark.parametrize("D,page", [(64, 16), (128, 32), (128, 16)])
@pytest.mark.parametrize("qs", [[1] * 6, [30] * 6])
def test_prefix_attention_strides_and_guards(qs, D, page):
    p = problem(800, [60, 90, 33, 47, 31, 100], qs, 8, 2, D, page)
    want, bound = ref.prefix_attention(**p, scale=0.1)
    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in p.items()}
    T = p["q"].shape[0]
    for pad in (8, 3):
        q = torch.full((T, 8, D + pad), float("nan"), dtype=BF, device="cuda")
        q[..., :D] = dev["q"]
        kv = torch.full(p["k_cache"].shape[:1] + (page, 2, 2, D), float("nan"), dtype=BF, device="cuda")  # keys and values side by side, heads within a row
        kv[:, :, 0], kv[:, :, 1] = dev["k_cache"].transpose(1, 2), dev["v_cache"].transpose(1, 2)
        out = torch.full((T + 2, 8, D + pad), 7.0, dtype=BF, device="cuda")
        view = out[1:-1, :, :D]
        table = torch.full((6, p["block_table"].shape[1] + 3), 12345678, dtype=torch.int32, device="cuda")
        table[:, :-3] = dev["block_table"]
        got = ap.approxifer_prefix_attention(q[..., :D], kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2), dev["prefix_table"], 800, table[:, :-3], dev["q_start"],
                                             dev["kv_len"], max(qs), scale=0.1, out=view)
        assert got is view
        check(view, want, bound)
        view.fill_(7.0)
        assert bool((out == 7.0).all())


def test_prefix_attention_large_scores():
    """Scores of some thousand: the maxima of the prefix and of a sequence's own keys lie far apart either way."""
    for qs in ([1, 1], [40, 3]):
        p = problem(300, [60, 90], qs, 4, 1, 64, 16)
        p["q"] = p["q"] * 16
        for part, factor in ((p["prefix_table"], 30.0), (p["block_table"][p["block_table"] >= 0], 30.0)):
            p2 = dict(p, k_cache=p["k_cache"].clone())
            p2["k_cache"][part.long()] *= factor
            want, bound = ref.prefix_attention(**p2, scale=0.5)
            check(run(p2, scale=0.5), want, bound)


@pytest.mark.parametrize("qs", [[1] * 9, [25] * 9])
def test_prefix_attention_is_repeatable_and_runs_on_a_stream_and_in_a_graph(qs):
    p = problem(3000, [60, 90, 33, 47, 31, 100, 28, 64, 65], qs, 16, 4, 128, 16)
    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in p.items()}
    first = ap.approxifer_prefix_attention(**dev, max_q=max(qs))
    for _ in range(3):
        assert torch.equal(ap.approxifer_prefix_attention(**dev, max_q=max(qs)), first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = ap.approxifer_prefix_attention(**dev, max_q=max(qs), stream=s)
    s.synchronize()
    assert torch.equal(y, first)
    out = torch.zeros_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ap.approxifer_prefix_attention(**dev, max_q=max(qs), out=out)
        ap.approxifer_prefix_attention(**dev, max_q=max(qs), out=out)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)


def test_prefix_attention_equals_attention_over_the_whole():
    """Pages of the prefix at the head of every sequence's own table: approxifer_attention computes the same."""
    for qs in ([1, 1, 1], [30, 1, 64]):
        p = problem(512, [60, 90, 64], qs, 8, 2, 128, 16)
        both = dict(p, block_table=torch.cat([p["prefix_table"].expand(3, -1), p["block_table"]], 1).contiguous(), kv_len=p["kv_len"] + 512)
        dev = {n: t.cuda() for n, t in both.items() if isinstance(t, torch.Tensor) and n != "prefix_table"}
        want, bound = ref.prefix_attention(**p, scale=0.1)
        check(ap.approxifer_attention(**dev, max_q=max(qs), scale=0.1), want, bound)
        check(run(p), want, bound)


def test_prefix_attention_of_no_tokens_and_offsets_beyond_32_bits():
    p = problem(64, [5], [0], 4, 2, 64, 16)
    assert run(p, max_q=1).shape == (0, 4, 64)
    # pages beyond 2^32 elements from the base
    page, D, Hkv = 64, 128, 8
    pages = 2 ** 32 // (page * D * Hkv) + 40
    k, v = (torch.empty((pages, Hkv, page, D), dtype=BF, device="cuda") for _ in range(2))
    for qs in ([1, 1], [20, 3]):
        p = problem(1500, [60, 90], qs, 16, Hkv, D, page)
        far = pages - 40
        some = p["k_cache"].shape[0]
        k[far: far + some], v[far: far + some] = p["k_cache"].cuda(), p["v_cache"].cuda()
        want, bound = ref.prefix_attention(**p, scale=0.1)
        moved = dict(p, prefix_table=p["prefix_table"] + far, block_table=torch.where(p["block_table"] < 0, -1, p["block_table"] + far).int())
        dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in moved.items() if n not in ("k_cache", "v_cache")}
        check(ap.approxifer_prefix_attention(**dev, k_cache=k, v_cache=v, max_q=max(qs), scale=0.1), want, bound)


def test_prefix_attention_refuses_what_the_library_cannot_take():
    p = problem(64, [5, 9], [1, 1], 4, 2, 64, 16)
    dev = dict({n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in p.items()}, max_q=1)
    for bad in (dict(q=dev["q"].float()), dict(prefix_table=dev["prefix_table"].long()), dict(prefix_table=dev["prefix_table"][None]), dict(prefix_table=p["prefix_table"]),
                dict(block_table=dev["block_table"][0]), dict(kv_len=dev["kv_len"][:1]), dict(v_cache=dev["v_cache"][:, :1]), dict(out=dev["q"][:1])):
        with pytest.raises(ValueError):
            ap.approxifer_prefix_attention(**dict(dev, **bad))
    for bad in (dict(prefix_len=-1), dict(prefix_len=2 ** 31), dict(max_q=0), dict(scale=float("nan")), dict(q=dev["q"][:, :3].contiguous())):
        with pytest.raises(ap.ApproxiferError):
            ap.approxifer_prefix_attention(**dict(dev, **bad))
    assert ap.load().approxifer_prefix_attention(None, None) == ap.load().approxifer_attention(None, None)
