"""approxifer_prefix_attention of single tokens in the layouts that approxifer_attention runs on the tensor cores and prompts cannot have:
pages of any size, queries and outputs at 4 bytes, many query heads to a key head.  They run the same kernel: behind a prefix of whole
chunks and pages, which approxifer_attention sees at the head of each sequence's own table, both give the same bits."""
import pytest
import torch

import hosted_more_reference as ref
import paper_2109_09868_b200 as ap
from test_gpu_prefix import check, problem, run

pytestmark = pytest.mark.gpu

CASES = [  # prefix, own lengths, Hq, Hkv, D, page, distance of the queries from 16 bytes (elements), more elements to a row of them
    (4032, [77, 5, 31, 1, 50, 300], 8, 2, 64, 24, 0, 0),
    (960, [40, 3, 9], 6, 2, 96, 24, 0, 0),
    (960, [40, 3, 9], 4, 4, 128, 5, 0, 0),
    (960, [40, 3, 9], 4, 1, 40, 4, 0, 0),
    (64, [7, 2], 2, 1, 8, 1, 0, 0),
    (960, [40, 3, 9], 8, 2, 64, 16, 2, 0),
    (960, [40, 3, 9], 8, 2, 128, 32, 0, 2),
    (960, [40, 3, 9], 8, 2, 80, 40, 6, 6),
    (480, [40, 3], 260, 2, 64, 16, 0, 0),
]


def placed(t, at, more):
    """t [T][H][D] in the middle of a larger array, its base `at` elements from 16 bytes, its rows `more` elements longer."""
    T, H, D = t.shape
    room = torch.full((T * H * (D + more) + 16,), 7.0, dtype=t.dtype, device="cuda")
    view = room[at: at + T * H * (D + more)].view(T, H, D + more)[..., :D]
    view.copy_(t)
    return room, view


@pytest.mark.parametrize("prefix,kv,Hq,Hkv,D,page,at,more", CASES)
def test_single_tokens_run_the_same_kernel_as_attention(prefix, kv, Hq, Hkv, D, page, at, more):
    p = problem(prefix, kv, [1] * len(kv), Hq, Hkv, D, page)
    want, bound = ref.prefix_attention(**p, scale=0.1)
    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in p.items()}
    _, dev["q"] = placed(dev["q"], at, more)
    room, out = placed(torch.full_like(p["q"], 7.0).cuda(), at, more)
    before = ap.launch_count()
    assert ap.approxifer_prefix_attention(**dev, max_q=1, scale=0.1, out=out) is out
    assert ap.launch_count() - before == 1
    check(out, want, bound)
    table = torch.cat([dev["prefix_table"].expand(len(kv), -1), dev["block_table"]], 1).contiguous()
    whole = ap.approxifer_attention(dev["q"], dev["k_cache"], dev["v_cache"], table, dev["q_start"], dev["kv_len"] + prefix, 1, scale=0.1)
    assert torch.equal(out, whole)
    out.fill_(7.0)
    assert bool((room == 7.0).all())


@pytest.mark.parametrize("kv,page,D", [([300, 5, 77], 24, 64), ([2000] * 70, 24, 128), ([2000] * 70, 4, 64)])
def test_single_tokens_without_a_prefix_are_attentions(kv, page, D):
    p = problem(0, kv, [1] * len(kv), 8, 2, D, page)
    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in p.items()}
    own = [dev[n] for n in ("q", "k_cache", "v_cache", "block_table", "q_start", "kv_len")]
    before = ap.launch_count()
    want = ap.approxifer_attention(*own, 1, scale=0.1)
    launches = ap.launch_count() - before
    got = ap.approxifer_prefix_attention(**dev, max_q=1, scale=0.1)
    assert ap.launch_count() - before == 2 * launches
    assert torch.equal(got, want)


def test_rows_that_see_less():
    """Pages that hold nothing in the prefix and behind it, a prefix longer than its table, sequences without a new token and without a place for
    it, infinities and NaN behind every end."""
    p = problem(403, [60, 0, 90, 33], [1, 1, 0, 1], 8, 2, 64, 24, short=[(-1, 3, -1), (-1, 10, 10 ** 6), (0, 1, -5)])
    named = torch.zeros(p["k_cache"].shape[0], 24, dtype=torch.bool)
    for table, n in [(p["prefix_table"], 403)] + [(p["block_table"][b], int(p["kv_len"][b])) for b in range(4)]:
        at = torch.arange(n)
        page = table.long()[at // 24]
        there = (page >= 0) & (page < named.shape[0])
        named[page[there], at[there] % 24] = True
    for name, bad in (("k_cache", float("nan")), ("v_cache", float("inf"))):
        p[name].transpose(1, 2)[~named] = bad
    for count in (403, 10 ** 6):  # (the table has 408 positions)
        q = dict(p, prefix_len=count)
        if count > 403:
            q["k_cache"], q["v_cache"] = (c.nan_to_num(0.0, 0.0, 0.0) for c in (p["k_cache"], p["v_cache"]))
        want, bound = ref.prefix_attention(**q, scale=0.1)
        check(run(q, max_q=1), want, bound)
