"""approxifer_qk_norm_rope against its 64-bit plain form, and what it leaves untouched in the cache."""
import pytest
import torch

import hosted_reference as ref
import paper_2109_09868_b200 as ap

pytestmark = pytest.mark.gpu

EPS = 1e-5


def table(positions, rot):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def inputs(T, Hq, Hkv, D, rot, page, dtype, seed=0, weights=True):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g).to(dtype)  # noqa: E731
    pages = (T + page - 1) // page + 2
    return dict(qkv=rnd(T, (Hq + 2 * Hkv) * D), qw=1 + 0.1 * rnd(D) if weights else None, kw=1 + 0.1 * rnd(D) if weights else None,
                cs=table(5000, rot), pos=torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32),
                slots=torch.randperm(pages * page, generator=g)[:T], kc=rnd(pages, Hkv, page, D), vc=rnd(pages, Hkv, page, D))


def split(qkv, Hq, Hkv, D):
    q, k, v = qkv.split([Hq * D, Hkv * D, Hkv * D], 1)
    return q.unflatten(1, (Hq, D)), k.unflatten(1, (Hkv, D)), v.unflatten(1, (Hkv, D))


def check(got, want, bound):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    over = ((got - want).abs() - bound).max()
    assert over <= 0, float(over)


CASES = [  # T, Hq, Hkv, D, rot, interleaved, page, dtype, weights
    (1, 32, 8, 128, 128, False, 16, torch.bfloat16, True),
    (1, 1, 1, 2, 2, True, 1, torch.float32, True),
    (37, 8, 2, 64, 64, False, 16, torch.bfloat16, True),
    (37, 8, 2, 64, 32, True, 16, torch.bfloat16, True),
    (37, 15, 5, 80, 48, True, 16, torch.float32, True),
    (37, 6, 3, 80, 40, False, 8, torch.bfloat16, True),
    (50, 4, 4, 96, 96, False, 32, torch.float32, True),
    (50, 4, 1, 96, 24, False, 32, torch.bfloat16, True),   # halves of 12: not whole columns of 8
    (300, 3, 1, 128, 64, False, 64, torch.float32, False),
    (33, 2, 2, 256, 256, False, 16, torch.bfloat16, True),
    (33, 2, 2, 256, 128, False, 16, torch.float32, True),
    (33, 2, 1, 33, 10, False, 16, torch.float32, True),
    (33, 2, 1, 33, 0, False, 16, torch.bfloat16, True),
    (700, 16, 2, 128, 128, False, 16, torch.bfloat16, True),
    (5, 40, 40, 72, 72, True, 16, torch.bfloat16, False),
]


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,inter,page,dtype,weights", CASES)
def test_norm_rope_matches_the_plain_form(T, Hq, Hkv, D, rot, inter, page, dtype, weights):
    x = inputs(T, Hq, Hkv, D, rot, page, dtype, weights=weights)
    d = {n: None if t is None else t.cuda() for n, t in x.items()}
    q, k, v = split(d["qkv"], Hq, Hkv, D)
    status = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    got = ap.approxifer_qk_norm_rope(q, k, v, d["qw"], d["kw"], d["cs"], d["pos"], d["kc"], d["vc"], d["slots"], eps=EPS, interleaved=inter,
                                     status=status)
    q, k, v = split(x["qkv"], Hq, Hkv, D)
    check(got, *ref.norm_rope_rows(q, x["qw"], x["cs"], x["pos"], EPS, inter))
    page_at, row = x["slots"] // page, x["slots"] % page
    check(d["kc"].cpu()[page_at, :, row], *ref.norm_rope_rows(k, x["kw"], x["cs"], x["pos"], EPS, inter))
    assert torch.equal(d["vc"].cpu()[page_at, :, row], v)
    for name in ("kc", "vc"):  # all other slots hold what they held
        was, now = x[name].clone(), d[name].cpu()
        was[page_at, :, row] = 0
        now[page_at, :, row] = 0
        assert torch.equal(was, now)
    assert not status.any()


def test_norm_rope_padding_slots_and_positions_out_of_range():
    T, Hq, Hkv, D, page = 40, 4, 2, 64, 16
    for dtype in (torch.bfloat16, torch.float32):
        x = inputs(T, Hq, Hkv, D, D, page, dtype, seed=1)
        x["slots"][3], x["slots"][4] = -1, x["kc"].shape[0] * page
        x["pos"][7], x["pos"][8] = -1, 5000
        d = {n: t.cuda() for n, t in x.items()}
        q, k, v = split(d["qkv"], Hq, Hkv, D)
        status = torch.zeros(T, dtype=torch.int32, device="cuda")
        got = ap.approxifer_qk_norm_rope(q, k, v, d["qw"], d["kw"], d["cs"], d["pos"], d["kc"], d["vc"], d["slots"], eps=EPS, status=status)
        want_status = torch.zeros(T, dtype=torch.int32)
        want_status[4], want_status[7], want_status[8] = 64, 32, 32
        assert torch.equal(status.cpu(), want_status)
        assert not got[7:9].any()
        keep = [i for i in range(T) if i not in (7, 8)]
        q, k, v = split(x["qkv"], Hq, Hkv, D)
        check(got[keep], *(t for t in ref.norm_rope_rows(q[keep], x["qw"], x["cs"], x["pos"][keep], EPS, False)))
        written = [i for i in range(T) if i not in (3, 4, 7, 8)]
        page_at, row = x["slots"][written] // page, x["slots"][written] % page
        check(d["kc"].cpu()[page_at, :, row], *ref.norm_rope_rows(k[written], x["kw"], x["cs"], x["pos"][written], EPS, False))
        for name in ("kc", "vc"):
            was, now = x[name].clone(), d[name].cpu()
            was[page_at, :, row] = 0
            now[page_at, :, row] = 0
            assert torch.equal(was, now)


def test_norm_rope_in_place_queries_only_strided_and_unaligned():
    T, Hq, D = 19, 6, 128
    for dtype in (torch.bfloat16, torch.float32):
        x = inputs(T, Hq, 1, D, D, 16, dtype, seed=2)
        q, k, v = split(x["qkv"], Hq, 1, D)
        want, bound = ref.norm_rope_rows(q, x["qw"], x["cs"], x["pos"], EPS, False)
        wide = torch.full((T, Hq, D + 16), 3.0, dtype=dtype, device="cuda")
        wide[:, :, 8:8 + D] = q.cuda()
        view = wide[:, :, 8:8 + D]
        ap.approxifer_qk_norm_rope(view, None, None, x["qw"].cuda(), None, x["cs"].cuda(), x["pos"].cuda(), None, None, None, q_out=view, eps=EPS)
        check(view, want, bound)
        assert bool((wide[:, :, :8] == 3.0).all()) and bool((wide[:, :, 8 + D:] == 3.0).all())
        odd = torch.full((T, Hq, D + 5), 3.0, dtype=dtype, device="cuda")
        odd[:, :, 3:3 + D] = q.cuda()
        out = torch.full((T, Hq, D + 1), 3.0, dtype=dtype, device="cuda")
        ap.approxifer_qk_norm_rope(odd[:, :, 3:3 + D], None, None, x["qw"].cuda(), None, x["cs"].cuda(), x["pos"].cuda(), None, None, None,
                                   q_out=out[:, :, 1:], eps=EPS)
        check(out[:, :, 1:], want, bound)
        assert bool((out[:, :, 0] == 3.0).all())


def test_norm_rope_of_zero_rows_and_of_no_tokens():
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    cs = table(4, 64).cuda()
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    assert not ap.approxifer_qk_norm_rope(x, None, None, w, None, cs, pos, None, None, None, eps=EPS).any()
    assert ap.approxifer_qk_norm_rope(x[:0], None, None, w, None, cs, pos[:0], None, None, None).shape == (0, 2, 64)


def test_norm_rope_refuses_what_the_library_cannot_take():
    x = inputs(5, 4, 2, 64, 64, 16, torch.bfloat16)
    d = {n: t.cuda() for n, t in x.items()}
    q, k, v = split(d["qkv"], 4, 2, 64)
    good = dict(q=q, k=k, v=v, q_weight=d["qw"], k_weight=d["kw"], cos_sin=d["cs"], positions=d["pos"], k_cache=d["kc"], v_cache=d["vc"], slots=d["slots"])
    for bad in (dict(q=q.float()), dict(k=k.float()), dict(q_weight=d["qw"][:32]), dict(cos_sin=d["cs"].bfloat16()), dict(positions=d["pos"].long()),
                dict(slots=d["slots"].int()), dict(k=None), dict(v_cache=None), dict(slots=None), dict(k_cache=d["kc"][:, :1]), dict(q=q.cpu())):
        with pytest.raises(ValueError):
            ap.approxifer_qk_norm_rope(**dict(good, **bad))
    with pytest.raises(ap.ApproxiferError):
        ap.approxifer_qk_norm_rope(**dict(good, cos_sin=d["cs"][:, :33].contiguous()))  # an odd rotation
    with pytest.raises(ap.ApproxiferError):
        ap.approxifer_qk_norm_rope(**good, eps=-1.0)


def test_norm_rope_passes_on_the_error_of_an_argument_without_a_truth_value():
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(RuntimeError, match="ambiguous"):
        ap.approxifer_qk_norm_rope(x, None, None, None, None, table(4, 64).cuda(), torch.arange(3, dtype=torch.int32, device="cuda"), None, None, None,
                                   interleaved=torch.ones(2))
