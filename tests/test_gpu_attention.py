"""approxifer_attention against its 64-bit plain form: one token and chunks of prompts, windows, sinks, lengths of zero and one,
pages that end inside a tile, freed pages, NaN wherever nothing may be read, strides."""
import pytest
import torch

import hosted_reference as ref
import paper_2109_09868_b200 as ap
from test_hosted_cpu import ATTENTION

pytestmark = pytest.mark.gpu


def inputs(qs, kvs, Hq, Hkv, D, page, seed=0, dirty=True):
    """Packed queries and a cache whose pages are shuffled; slots that hold no token are NaN."""
    g = torch.Generator().manual_seed(seed)
    per = [(n + page - 1) // page for n in kvs]
    pages = sum(per) + 2
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(kvs), max(max(per), 1)), -1, dtype=torch.int32)
    used, at = torch.zeros((pages, page), dtype=torch.bool), 0
    for b, (n, m) in enumerate(zip(kvs, per)):
        table[b, :m] = order[at: at + m]
        for j in range(n):
            used[table[b, j // page].long(), j % page] = True
        at += m
    starts = torch.tensor([sum(qs[:i]) for i in range(len(qs) + 1)], dtype=torch.int32)
    rnd = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
    q, k, v = rnd(sum(qs), Hq, D), rnd(pages, Hkv, page, D), rnd(pages, Hkv, page, D)
    if dirty:
        for c in (k, v):
            c.transpose(1, 2)[~used] = float("nan")
    return q, k, v, table, starts, torch.tensor(kvs, dtype=torch.int32)


def run(x, max_q, window, sinks, scale):
    return ap.approxifer_attention(*[t.cuda() for t in x], max_q, window=window, sinks=sinks, scale=scale)


def check(got, want, bound):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    over = ((got - want).abs() - bound).max()
    assert over <= 0, float(over)


CASES = [  # queries, cached tokens, Hq, Hkv, D, page, window, sinks
    # one token for each sequence
    ([1], [1], 1, 1, 64, 16, 0, 0),
    ([1, 1, 1], [1, 17, 300], 8, 2, 128, 16, 0, 0),
    ([1, 1, 1, 1], [5, 128, 129, 1000], 8, 8, 64, 16, 64, 4),
    ([1, 1], [700, 3], 16, 1, 128, 32, 100, 1),
    ([1, 1], [1500, 2100], 4, 1, 128, 16, 0, 0),
    ([1, 1, 1], [90, 91, 92], 6, 2, 80, 8, 17, 3),
    ([1, 1], [333, 64], 9, 3, 96, 64, 0, 0),
    ([1], [500], 40, 2, 64, 16, 200, 16),      # 20 query heads share a key head
    ([1, 1], [77, 400], 4, 2, 72, 24, 50, 2),  # a page size that is no power of two
    ([1, 1], [0, 40], 4, 2, 64, 16, 8, 2),     # a sequence with nothing cached: its row is zero
    ([1, 1], [130, 260], 2, 2, 40, 16, 1, 0),  # a window of the token itself
    ([1], [260], 2, 1, 64, 16, 100, 300),      # more sinks than tokens before the window
    ([1] * 40, [37 * i for i in range(40)], 4, 1, 64, 16, 0, 0),                # many sequences of all lengths, the first empty
    ([1] * 35, [1 + 61 * (i % 7) for i in range(35)], 2, 2, 128, 8, 90, 3),
    ([1, 0, 1, 1], [300, 50, 0, 4100], 20, 1, 64, 64, 0, 0),                    # a sequence without a new token; two row tiles
    # prompts and chunks
    ([5], [5], 1, 1, 64, 16, 0, 0),
    ([130], [130], 4, 2, 128, 16, 0, 0),
    ([300, 1, 129], [300, 200, 129], 4, 1, 64, 16, 0, 0),
    ([257], [257], 2, 2, 128, 64, 100, 4),
    ([200, 64], [513, 700], 8, 2, 64, 32, 130, 5),
    ([150, 3], [400, 3], 6, 2, 80, 16, 64, 1),
    ([90], [600], 3, 1, 96, 8, 0, 0),
    ([70], [70], 16, 1, 128, 128, 20, 2),
    ([2, 2], [300, 2], 4, 4, 128, 16, 0, 0),
    ([33, 7], [20, 7], 4, 2, 64, 16, 0, 0),    # fewer cached tokens than queries: the first rows see nothing
    ([20], [200], 10, 2, 64, 16, 16, 0),       # 5 query heads share a key head
    ([40], [120], 4, 2, 72, 24, 50, 2),
    ([140], [140], 2, 1, 256, 16, 0, 0),
    ([6], [50], 2, 1, 33, 16, 10, 1),
    ([400], [400], 2, 1, 128, 16, 5, 40),      # sinks that reach past the window's start
    # few queries at long contexts: the keys are cut over a cluster
    ([7], [3000], 2, 1, 96, 16, 0, 0),
    ([2], [1100], 4, 4, 64, 64, 0, 0),
    ([33, 100], [1700, 2500], 8, 2, 64, 16, 0, 0),
    ([160], [2600], 4, 2, 128, 32, 900, 5),
    ([90, 2, 0], [1600, 900, 70], 6, 2, 128, 16, 1000, 20),
    ([20], [10], 2, 2, 128, 16, 0, 0),
]


@pytest.mark.parametrize("qs,kvs,Hq,Hkv,D,page,window,sinks", CASES)
def test_attention_matches_the_plain_form(qs, kvs, Hq, Hkv, D, page, window, sinks):
    x = inputs(qs, kvs, Hq, Hkv, D, page, seed=sum(kvs) + D)
    scale = D ** -0.5
    want, bound = ref.attention(*x, window, sinks, scale)
    check(run(x, max(qs), window, sinks, scale), want, bound)


def test_attention_scale_sign_and_large_scores():
    x = inputs([1, 140], [300, 140], 4, 2, 64, 16, seed=9)
    for scale in (-0.3, 0.0, 4.0):
        want, bound = ref.attention(*x, 0, 0, scale)
        check(run(x, 140, 0, 0, scale), want, bound)
        one = (x[0][:1], x[1], x[2], x[3][:1], x[4][:2], x[5][:1])
        check(run(one, 1, 0, 0, scale), want[:1], bound[:1])


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 2), (128, 8, 1)])
def test_attention_freed_pages_and_foreign_tokens_are_not_seen(D, Hq, Hkv):
    """Pages that left the window are freed and given to others: their entries are -1, out of range, or their content is NaN."""
    window, sinks, page, n = 100, 4, 16, 700
    for nq in (1, 90):
        x = list(inputs([nq], [n], Hq, Hkv, D, page, seed=5))
        want, bound = ref.attention(*x, window, sinks, D ** -0.5)
        first = n - nq + 1 - window  # the first position any query's window holds
        gone = [p for p in range(1, n // page) if (p + 1) * page <= first]
        for c in (1, 2):
            x[c] = x[c].clone()
            x[c][x[3][0, gone].long()] = float("nan")
            head = x[c].transpose(1, 2)[x[3][0, 0].long()]  # the sinks' page, beyond the sinks
            head[sinks:] = float("nan")
        check(run(x, nq, window, sinks, D ** -0.5), want, bound)
        x[3] = x[3].clone()
        x[3][0, gone] = torch.tensor([(-1, 10 ** 6, -7)[i % 3] for i in range(len(gone))], dtype=torch.int32)
        check(run(x, nq, window, sinks, D ** -0.5), want, bound)
        # a page inside the window that is gone too: its positions are left out
        x[3][0, n // page - 2] = -1
        want, bound = ref.attention(*x, window, sinks, D ** -0.5)
        check(run(x, nq, window, sinks, D ** -0.5), want, bound)
        x[3][:] = -1
        assert not run(x, nq, window, sinks, D ** -0.5).any()


def test_attention_later_and_earlier_tokens_cannot_reach_a_row():
    """Infinities and NaN in a key or a value change exactly the rows that see them."""
    for D, page in ((64, 16), (128, 32)):
        n, window, sinks = 300, 90, 2
        x = list(inputs([n], [n], 4, 2, D, page, seed=3))
        want, bound = ref.attention(*x, window, sinks, D ** -0.5)
        for at, bad in ((40, float("nan")), (140, float("inf")), (299, float("-inf")), (1, float("nan"))):
            for which in (1, 2):
                y = list(x)
                y[which] = x[which].clone()
                y[which][x[3][0, at // page].long(), 1, at % page, 3] = bad
                got = run(y, n, window, sinks, D ** -0.5).double().cpu()
                sees = torch.tensor([at <= p and (at > p - window or at < sinks) for p in range(n)])
                check(got[~sees], want[~sees], bound[~sees])
                check(got[:, :2], want[:, :2], bound[:, :2])  # the other key head
                if which == 2:  # a value: that element of the rows that see it, no other
                    assert not torch.isfinite(got[sees][:, 2:, 3]).any()
                    rest = [d for d in range(D) if d != 3]
                    check(got[sees][:, 2:][..., rest], want[sees][:, 2:][..., rest], bound[sees][:, 2:][..., rest])
                elif bad != bad:
                    assert torch.isnan(got[sees][:, 2:]).all()


def test_attention_strides_guards_streams_and_repeatability():
    for qs, kvs in (([1, 1], [100, 333]), ([77, 130], [100, 333])):
        q, k, v, table, start, lens = inputs(qs, kvs, 4, 2, 128, 16, seed=11)
        want, bound = ref.attention(q, k, v, table, start, lens, 60, 4, 0.1)
        T = q.shape[0]
        wide = torch.zeros((T, 9, 136), dtype=torch.bfloat16, device="cuda")
        wide[:, 2:6, 8:] = q.cuda()
        token_major = [c.cuda().transpose(1, 2).contiguous().transpose(1, 2) for c in (k, v)]  # rows of a page before its heads
        out = torch.full((T + 2, 4, 136), 7.0, dtype=torch.bfloat16, device="cuda")
        rest = [t.cuda() for t in (table, start, lens)]
        args = dict(window=60, sinks=4, scale=0.1)
        got = ap.approxifer_attention(wide[:, 2:6, 8:], *token_major, *rest, max(qs), out=out[1:-1, :, :128], **args)
        check(got, want, bound)
        first = got.clone()
        got.fill_(7.0)
        assert bool((out == 7.0).all())
        for _ in range(3):
            assert torch.equal(ap.approxifer_attention(q.cuda(), *token_major, *rest, max(qs), **args), first)
        s = torch.cuda.Stream()
        qd = q.cuda()
        s.wait_stream(torch.cuda.current_stream())
        y = ap.approxifer_attention(qd, *token_major, *rest, max(qs), stream=s, **args)
        s.synchronize()
        assert torch.equal(y, first)
        # a looser bound on the queries of a sequence may choose another kernel, with other roundings
        check(ap.approxifer_attention(qd, *token_major, *rest, max(qs) + 5, **args), want, bound)
        # bases and rows that are not whole 16 bytes
        odd = torch.zeros((T, 4, 131), dtype=torch.bfloat16, device="cuda")
        odd[:, :, 1:129] = q.cuda()
        yo = torch.zeros((T, 4, 129), dtype=torch.bfloat16, device="cuda")
        check(ap.approxifer_attention(odd[:, :, 1:129], *token_major, *rest, max(qs), out=yo[:, :, 1:], **args), want, bound)


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 4, 1), (64, 20, 1), (96, 2, 2)])
def test_attention_single_tokens_with_and_without_workspace(D, Hq, Hkv):
    """The balanced form (with the workspace the library asks for) and the cluster form (without) agree with the plain form.  The
    table is much wider than the sequences are long, so that the library expects a large call."""
    kvs = [5, 700, 0, 333, 64, 1, 1500, 16, 15, 17, 800]
    q, k, v, table, start, lens = inputs([1] * len(kvs), kvs, Hq, Hkv, D, 16, seed=D)
    wide = torch.full((len(kvs), 8192), -1, dtype=torch.int32)
    wide[:, : table.shape[1]] = table
    for window, sinks in ((0, 0), (200, 4)):
        want, bound = ref.attention(q, k, v, table, start, lens, window, sinks, D ** -0.5)
        check(run((q, k, v, table, start, lens), 1, window, sinks, D ** -0.5), want, bound)
        got = run((q, k, v, wide, start, lens), 1, window, sinks, D ** -0.5)
        check(got, want, bound)
        assert torch.equal(got, run((q, k, v, wide, start, lens), 1, window, sinks, D ** -0.5))


def test_attention_of_no_tokens():
    x = inputs([1], [8], 2, 1, 64, 16)
    none = (x[0][:0], x[1], x[2], x[3], torch.zeros(2, dtype=torch.int32), x[5])
    assert run(none, 1, 0, 0, 0.1).shape == (0, 2, 64)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_cut_over_a_cluster_keeps_what_a_row_sees(D):
    """Few queries at a long context: NaN values reach the rows that see them, freed pages are left out, results repeat."""
    nq, n, window, sinks = 70, 2000, 1200, 3
    x = list(inputs([nq], [n], 4, 2, D, 16, seed=6))
    want, bound = ref.attention(*x, window, sinks, D ** -0.5)
    got = run(x, nq, window, sinks, D ** -0.5)
    check(got, want, bound)
    assert torch.equal(got, run(x, nq, window, sinks, D ** -0.5))
    for at in (n - nq - window + 20, n - 30, 1):
        y = list(x)
        y[2] = x[2].clone()
        y[2][x[3][0, at // 16].long(), 1, at % 16, 5] = float("nan")
        bad = run(y, nq, window, sinks, D ** -0.5).double().cpu()
        sees = torch.tensor([at <= p and (at > p - window or at < sinks) for p in range(n - nq, n)])
        assert torch.isnan(bad[sees][:, 2:, 5]).all()
        rest = [d for d in range(D) if d != 5]
        check(bad[..., rest], want[..., rest], bound[..., rest])
        if not sees.all():
            check(bad[~sees], want[~sees], bound[~sees])
    y = list(x)
    y[3] = x[3].clone()
    y[3][0, [70, 90, 110]] = -1
    want, bound = ref.attention(*y, window, sinks, D ** -0.5)
    check(run(y, nq, window, sinks, D ** -0.5), want, bound)


@pytest.mark.parametrize("qs,kvs,page", [([1, 1], [700, 40], 256), ([200], [700], 256), ([200], [1400], 1024), ([130, 20], [300, 900], 128)])
def test_attention_pages_longer_than_a_tile(qs, kvs, page):
    for D in (64, 128):
        x = inputs(qs, kvs, 4, 2, D, page, seed=page + D)
        want, bound = ref.attention(*x, 150, 3, D ** -0.5)
        check(run(x, max(qs), 150, 3, D ** -0.5), want, bound)


@pytest.mark.parametrize("nq", [1, 40])
def test_attention_cache_offsets_beyond_32_bits(nq):
    """A cache of more than 2^32 bytes, and 2^31 elements, whose tokens lie at its end."""
    Hkv, page, D, n = 4, 16, 128, 90
    pages = (1 << 31) // (Hkv * page * D) + 64
    caches = [torch.empty((pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    g = torch.Generator().manual_seed(8)
    table = torch.arange(pages - 1, pages - 1 - (n + page - 1) // page, -1, dtype=torch.int32)[None]
    small = [torch.randn((table.shape[1], Hkv, page, D), generator=g).bfloat16() for _ in range(2)]
    for c, s in zip(caches, small):
        c[table[0].long().cuda()] = s.cuda()
    q = torch.randn((nq, 8, D), generator=g).bfloat16()
    start, lens = torch.tensor([0, nq], dtype=torch.int32), torch.tensor([n], dtype=torch.int32)
    want, bound = ref.attention(q, *small, torch.arange(table.shape[1], dtype=torch.int32)[None], start, lens, 50, 2, 0.1)
    got = ap.approxifer_attention(q.cuda(), *caches, table.cuda(), start.cuda(), lens.cuda(), nq, window=50, sinks=2, scale=0.1)
    check(got, want, bound)
    # and the same slots written by the norm and rotation
    cs = torch.cat([torch.ones(4, D // 2), torch.zeros(4, D // 2)], 1).cuda()
    slots = (table[0].long() * page + 3).cuda()
    T = len(slots)
    new = torch.randn((T, Hkv, D), generator=g).bfloat16().cuda()
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    ap.approxifer_qk_norm_rope(q[:1].expand(T, -1, -1).contiguous().cuda(), new, new, None, None, cs, pos, *caches, slots)
    for c in caches:
        assert torch.equal(c[table[0].long().cuda(), :, 3], new)


def test_attention_large_finite_values_behind_the_mask_do_not_reach_a_row():
    """Values of the type's largest magnitude in positions that a row does not see: their weight is zero exactly."""
    n, window = 260, 70
    x = list(inputs([n], [n], 4, 2, 64, 16, seed=4))
    want, bound = ref.attention(*x, window, 0, 0.125)
    for at in (0, 129, 259):
        y = list(x)
        y[2] = x[2].clone()
        y[2][x[3][0, at // 16].long(), :, at % 16] = 3.3e38
        got = run(y, n, window, 0, 0.125).double().cpu()
        sees = torch.tensor([at <= p < at + window for p in range(n)])
        check(got[~sees], want[~sees], bound[~sees])


def widened(x, columns):
    """The same inputs with a table that has room for far longer sequences: the library then expects long ones."""
    q, k, v, table, start, lens = x
    wide = torch.full((table.shape[0], columns), -1, dtype=torch.int32)
    wide[:, : table.shape[1]] = table
    return q, k, v, wide, start, lens


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("columns", [0, 1024])
def test_attention_of_queries_before_the_first_cached_token_is_zero(D, columns):
    """Blocks of queries that no key is there for, beside others: with 64 tokens to a query tile, 300 queries on nothing, 200 on 40
    (the first tiles see nothing) and on 100 (of a pair of tiles only the second does)."""
    qs, kvs = [300, 130, 200, 200], [0, 130, 40, 100]
    x = inputs(qs, kvs, 4, 2, D, 16, seed=D)
    want, bound = ref.attention(*x, 60, 3, D ** -0.5)
    none = (want == 0).flatten(1).all(dim=1)
    assert int(none.sum()) == 300 + 160 + 100
    y = widened(x, columns) if columns else x
    ap.reset_device_wait_timeouts()
    first = run(y, max(qs), 60, 3, D ** -0.5)
    for _ in range(5):
        got = run(y, max(qs), 60, 3, D ** -0.5)
        check(got, want, bound)
        assert not got.cpu()[none].any()
        assert torch.equal(got, first)
    assert ap.device_wait_timeouts() == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_attention_cut_over_a_cluster_keeps_a_bad_query_to_its_row(D, bad):
    """Short sequences under a wide table: CTAs of the cluster that have no key to walk.  One query is NaN or infinite."""
    qs, kvs = [70, 20, 5], [90, 20, 0]
    x = list(inputs(qs, kvs, 4, 2, D, 16, seed=D + 1))
    want, bound = ref.attention(*x, 0, 0, D ** -0.5)
    x[0][33, 1] = bad
    got = run(widened(x, 1024), max(qs), 0, 0, D ** -0.5).double().cpu()
    assert torch.isnan(got[33, 1]).all()
    got[33, 1], want[33, 1], bound[33, 1] = 0, 0, 1
    check(got, want, bound)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_attention_single_tokens_shorter_than_the_copies_ahead(D):
    """Pages that are no power of two, sequences of no token and of less than a chunk for every warp: the copies that run ahead
    find nothing.  The table names few pages and has room for many, so that a cluster shares a sequence."""
    kvs = [0, 1, 2, 15, 16, 33, 70]
    x = inputs([1] * len(kvs), kvs, 4, 2, D, 24, seed=D + 2)
    want, bound = ref.attention(*x, 0, 0, D ** -0.5)
    check(run(x, 1, 0, 0, D ** -0.5), want, bound)
    check(run(widened(x, 40), 1, 0, 0, D ** -0.5), want, bound)


@pytest.mark.parametrize("page", [16, 24])
def test_attention_over_a_cache_of_no_pages_is_zero(page):
    """No page is valid: whatever the table says, nothing is there (the pointer still names memory, full of NaN)."""
    q, k, v, table, start, lens = [t.cuda() for t in inputs([1, 1], [40, 3], 4, 2, 64, page, seed=1)]
    k.fill_(float("nan"))
    out = torch.full_like(q, 7.0)
    T, Hq, D = q.shape
    args = ATTENTION.pack(T, 2, 1, Hq, 2, D, page, 0, 0, 0.125, 0, q.data_ptr(), *q.stride()[:2], k.data_ptr(), *k.stride()[:3], k.data_ptr(), *k.stride()[:3], 0,
                          table.data_ptr(), table.stride(0), table.shape[1], start.data_ptr(), lens.data_ptr(), out.data_ptr(), *out.stride()[:2], 0, 0)
    assert ap.load().approxifer_attention(args, torch.cuda.current_stream().cuda_stream) == 0
    assert not out.any()


@pytest.mark.parametrize("nq", [1, 2, 40])
@pytest.mark.parametrize("D,page", [(64, 16), (64, 24), (128, 16), (200, 16), (33, 16)])
def test_attention_first_tokens_are_seen_where_the_window_lies_beyond_the_table(D, page, nq):
    """A table of two pages under a sequence of 200 tokens: of the window nothing is there, or only its start; the sinks are."""
    x = list(inputs([nq], [200], 4, 2, D, page, seed=D))
    x[3] = x[3][:, :2].contiguous()
    for window, sinks in ((5, 3), (200 - nq - 20, 4), (0, 0), (30, 40)):
        want, bound = ref.attention(*x, window, sinks, D ** -0.5)
        assert want.abs().amax(dim=-1).min() > 0  # every row sees something
        check(run(x, nq, window, sinks, D ** -0.5), want, bound)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_takes_any_upper_bound_on_the_queries(D):
    """The bound may be as loose as the type allows: the call costs what its tokens cost."""
    Hkv, batch = 16, 12
    x = inputs([3] + [1] * (batch - 1), [20 + b for b in range(batch)], Hkv, Hkv, D, 16, seed=D + 3)
    want, bound = ref.attention(*x, 0, 0, D ** -0.5)
    for max_q in (3, 1000, 2 ** 31 - 1):
        check(run(x, max_q, 0, 0, D ** -0.5), want, bound)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_one_query_for_all_tokens(D):
    """Queries broadcast over the tokens: a token stride of zero."""
    q, k, v, table, start, lens = inputs([20, 1], [50, 9], 4, 2, D, 16, seed=D + 5)
    q = q[:1].expand(21, -1, -1)
    want, bound = ref.attention(q, k, v, table, start, lens, 30, 2, D ** -0.5)
    wide = q[:1].cuda().expand(21, -1, -1)
    assert wide.stride(0) == 0
    check(run((wide, k, v, table, start, lens), 20, 30, 2, D ** -0.5), want, bound)
    one = (wide[19:], k, v, table, torch.tensor([0, 1, 2], dtype=torch.int32), lens)
    check(run(one, 1, 30, 2, D ** -0.5), want[19:], bound[19:])


def test_attention_refuses_what_the_library_cannot_take():
    q, k, v, table, start, lens = [t.cuda() for t in inputs([1], [20], 4, 2, 64, 16)]
    for bad in (dict(q=q.float()), dict(k=k.float()), dict(v=v[:-1]), dict(table=table.long()), dict(start=start[:1]), dict(lens=lens.float()), dict(q=q.cpu()),
                dict(k=k[..., :32]), dict(q=q.transpose(1, 2))):
        args = dict(dict(q=q, k=k, v=v, table=table, start=start, lens=lens), **bad)
        with pytest.raises(ValueError):
            ap.approxifer_attention(*args.values(), 1)
    for bad in (dict(window=-1), dict(sinks=-2), dict(scale=float("nan"))):
        with pytest.raises(ap.ApproxiferError):
            ap.approxifer_attention(q, k, v, table, start, lens, 1, **bad)
    with pytest.raises(ap.ApproxiferError):
        ap.approxifer_attention(q[:, :3], k, v, table, start, lens, 1)  # 3 query heads on 2 key heads
