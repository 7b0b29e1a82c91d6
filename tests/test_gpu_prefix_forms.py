"""approxifer_prefix_attention in each of its forms (told by how many kernels a call launches): the prefix walked by every sequence, or in
a step of its own, cut into parts, shared by clusters, joined on the way or by a kernel for it."""
import pytest
import torch

import hosted_more_reference as ref
import paper_2109_09868_b200 as ap
from test_gpu_prefix import check, problem, run

pytestmark = pytest.mark.gpu

CASES = [  # launches, prefix, own lengths, new tokens, Hq, Hkv, D, page
    (1, 1003, [77, 5, 31, 1, 50], [1] * 5, 8, 2, 64, 16),                  # single tokens, each through the prefix
    (1, 2000, [900, 3], [1, 1], 16, 4, 128, 32),                           # ... a cluster of CTAs to a sequence
    (1, 501, [40, 3, 9], [1, 1, 1], 6, 2, 96, 8),                          # ... pages shorter than a chunk
    (2, 600, [600] * 16, [1] * 16, 16, 8, 64, 16),                         # in two steps, few parts, joined on the way
    (2, 700, [500] * 16, [1] * 16, 32, 8, 128, 16),
    (3, 3000, [100] * 40, [1] * 40, 4, 1, 64, 16),                         # many parts, joined by a kernel
    (3, 9000, [100, 3, 50, 70] * 4, [1] * 16, 8, 1, 128, 32),
    (3, 900, [600, 20, 300] * 10, [1] * 30, 32, 8, 64, 16),                # equal runs over warps, joined with the prefix's parts
    (3, 900, [600, 20, 300] * 10, [1] * 30, 32, 8, 128, 16),
    (2, 20573, [9] * 46, [1] * 46, 16, 1, 64, 64),                         # a long prefix: parts shared by clusters
    (3, 35031, [5, 2], [1, 1], 2, 1, 128, 64),
    (1, 108, [100, 178, 30], [100, 178, 20], 12, 4, 96, 32),               # prompts through the prefix
    (1, 200, [40, 300], [40, 90], 8, 2, 64, 16),
    (1, 1500, [1500], [60], 2, 1, 128, 16),                                # ... shared by a cluster
    (1, 1500, [1500], [60], 2, 1, 64, 16),
    (2, 5000, [50, 47, 60, 50, 44, 50, 50, 52], [50, 47, 48, 50, 44, 50, 50, 50], 128, 8, 128, 64),  # in two steps, some blocks uncut
    (2, 5000, [56, 55, 60, 56, 54, 56, 56, 58], [56, 55, 54, 56, 54, 56, 54, 53], 128, 8, 64, 32),
    (3, 4096, [9, 5, 40], [8, 5, 8], 12, 4, 128, 16),                      # many parts
    (1, 50, [13, 29, 8], [4, 20, 2], 3, 1, 33, 7),                          # odd layouts: element by element
    (3, 30000, [9, 2000, 40], [8, 5, 8], 4, 2, 64, 16),                    # ... long tables of their own: the own keys shared by a cluster
]


@pytest.mark.parametrize("launches,prefix,kv,qs,Hq,Hkv,D,page", CASES)
def test_each_form_matches_the_plain_form(launches, prefix, kv, qs, Hq, Hkv, D, page):
    p = problem(prefix, kv, qs, Hq, Hkv, D, page)
    want, bound = ref.prefix_attention(**p, scale=0.1)
    before = ap.launch_count()
    got = run(p)
    assert ap.launch_count() - before == launches
    check(got, want, bound)


@pytest.mark.parametrize("case", [0, 3, 5, 7, 10, 12, 13, 15, 17, 18])
def test_each_form_with_rows_that_see_less(case):
    """Pages that hold nothing, sequences without a new token, without a place for it, and tokens behind the last sequence, whose rows
    stay as they are."""
    _, prefix, kv, qs, Hq, Hkv, D, page = CASES[case]
    kv, qs = list(kv), list(qs)
    if len(qs) > 2:
        kv[1], qs[2] = 0, 0
    p = problem(prefix, kv, qs, Hq, Hkv, D, page, short=[(-1, 1, -1), (-1, (prefix - 1) // page, 10 ** 6)] + ([(0, 0, -3)] if kv[0] else []))
    want, bound = ref.prefix_attention(**p, scale=0.1)
    T = p["q"].shape[0]
    p["q"] = torch.cat([p["q"], torch.randn((3, Hq, D), generator=torch.Generator().manual_seed(9)).bfloat16()])  # three tokens of no sequence
    max_q = max(max(qs), -(-(T + 3) // len(qs)))
    if max(qs) == 1 and max_q > 1:
        max_q = 1
        p["q"] = p["q"][:T]  # (a bound of one leaves no room for them unless some sequence has none)
        if T < len(qs):
            p["q"] = torch.cat([p["q"], p["q"][:1]])
    out = torch.full((p["q"].shape[0], Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    run(p, max_q=max_q, out=out)
    check(out[:T], want, bound)
    assert bool((out[T:] == 7.0).all())


@pytest.mark.parametrize("case", [1, 3, 5, 7, 9, 12, 13, 15, 17, 18, 19])
def test_each_form_keeps_infinities_and_nan_apart(case):
    _, prefix, kv, qs, Hq, Hkv, D, page = CASES[case]
    p = problem(prefix - 5, kv, qs, Hq, Hkv, D, page)
    want, bound = ref.prefix_attention(**p, scale=0.1)
    named = torch.zeros(p["k_cache"].shape[0], page, dtype=torch.bool)
    for table, n in [(p["prefix_table"], prefix - 5)] + [(p["block_table"][b], n) for b, n in enumerate(kv)]:
        at = torch.arange(n)
        named[table.long()[at // page], at % page] = True
    for name, bad in (("k_cache", float("nan")), ("v_cache", float("inf"))):
        p[name].transpose(1, 2)[~named] = bad
    check(run(p), want, bound)
    # an infinity among the last of the prefix's values that is seen: all rows of its head see it
    p["v_cache"][p["prefix_table"][(prefix - 6) // page], 0, (prefix - 6) % page, 1] = float("inf")
    got = run(p).double().cpu()
    group = Hq // Hkv
    assert not torch.isfinite(got[:, :group, 1]).any()
    keep = torch.ones(Hq, D, dtype=torch.bool)
    keep[:group, 1] = False
    check(got[:, keep], want[:, keep], bound[:, keep])


@pytest.mark.parametrize("case", [3, 5, 7, 15, 17])
def test_forms_that_share_a_workspace_follow_each_other(case):
    """Two calls on one stream with one workspace, captured and replayed: the second waits for the first's last kernel."""
    _, prefix, kv, qs, Hq, Hkv, D, page = CASES[case]
    a, b = (problem(prefix, kv, qs, Hq, Hkv, D, page, seed=s) for s in (0, 10))
    room = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    dev = [{n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in p.items()} for p in (a, b)]
    want = [ap.approxifer_prefix_attention(**d, max_q=max(qs)) for d in dev]
    got = [torch.zeros_like(w) for w in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            for d, o in zip(dev, got):
                ap.approxifer_prefix_attention(**d, max_q=max(qs), workspace=room, out=o)
    for _ in range(3):
        for o in got:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
