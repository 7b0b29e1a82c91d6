"""approxifer_block_norm against its 64-bit plain form: widths and token counts of every path, types, norms, gates, strides."""
import pytest
import torch

import hosted_more_reference as ref
import paper_2109_09868_b200 as ap

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def normal(shape, seed, dtype=BF, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std + mean).to(dtype)


def check(got, want, name):
    value, bound = want
    got = got.double().cpu()
    assert torch.isfinite(got).all(), name
    over = ((got - value).abs() - bound).max()
    assert over <= 0, (name, float(over))


def case(T, N, stream, dtype, after, before, gate, act, bias, mean=0.0):
    v = dict(residual=normal((T, N), 1, stream, 3.0, mean), block=normal((T, N), 2, dtype, 5.0, mean), gate=None, block_weight=None, block_bias=None,
             next_weight=None, next_bias=None)
    if gate:
        v["gate"] = normal({"column": (N,), "token": (T, 1), "element": (T, N)}[gate], 3, dtype)
    if after:
        v["block_weight"] = normal(N, 4, dtype, 0.2, 1.0)
        v["block_bias"] = normal(N, 5, dtype) if bias else None
    if before:
        v["next_weight"] = normal(N, 6, dtype, 0.2, 1.0)
        v["next_bias"] = normal(N, 7, dtype) if bias else None
    return v, dict(after=after, before=before, gate_activation=act)


def run(v, k, scales=(1.0, 1.0), eps=1e-6, **more):
    dev = {n: None if t is None else t.cuda() for n, t in v.items()}
    return ap.approxifer_block_norm(**dev, **k, residual_scale=scales[0], block_scale=scales[1], eps=eps, **more)


CASES = [  # T, N, stream, type, after, before, gate, activation, biases, mean
    (1, 1, BF, BF, "rms", "rms", None, "none", False, 0.0),
    (1, 7, F32, F32, "layer", "layer", "element", "sigmoid", True, 1.0),
    (5, 8, BF, BF, "layer", "rms", "column", "none", False, 0.0),
    (3, 100, F32, BF, "rms", "layer", "token", "tanh", True, 0.0),
    (130, 256, BF, BF, "rms", "rms", "column", "tanh", False, 0.0),
    (1, 264, BF, BF, "rms", "rms", "element", "sigmoid", True, 0.0),
    (1, 4096, BF, BF, "rms", "rms", "column", "none", False, 0.0),
    (3, 4097, BF, BF, "layer", "layer", None, "none", True, 2.0),
    (2, 8192, F32, F32, "layer", "layer", "token", "none", True, 3.0),
    (2, 8200, BF, BF, "rms", "rms", "element", "tanh", False, 0.0),
    (2, 16384, F32, BF, "layer", "rms", "column", "sigmoid", True, 0.0),
    (2, 16381, F32, F32, "layer", "layer", "element", "none", True, 5.0),
    (700, 8192, BF, BF, "layer", "layer", "column", "tanh", True, 0.0),     # many rows: turns over the ring
    (701, 4096, F32, F32, "layer", "rms", "element", "sigmoid", True, 0.0),
    (1500, 1000, F32, BF, "rms", "rms", "token", "tanh", False, 0.0),
    (5000, 520, BF, F32, "rms", "layer", "column", "sigmoid", True, 1.0),
    (9001, 264, BF, BF, "rms", "rms", "element", "none", False, 0.0),
    (9001, 288, BF, BF, None, "rms", None, "none", False, 0.0),
    (1237, 1003, F32, F32, "layer", "layer", "element", "sigmoid", True, 0.0),
    (900, 2048, BF, BF, "rms", None, "column", "none", True, 0.0),
    (30000, 264, BF, BF, "rms", "layer", "column", "tanh", True, 0.0),      # many narrow rows: turns over the ring
    (12000, 1000, F32, BF, "layer", "rms", None, "none", True, 1.0),
    (12000, 520, F32, F32, "rms", "rms", "token", "sigmoid", False, 0.0),
    (900, 2056, F32, BF, None, None, "element", "tanh", False, 0.0),
]


@pytest.mark.parametrize("T,N,stream,dtype,after,before,gate,act,bias,mean", CASES)
def test_block_norm_matches_the_plain_form(T, N, stream, dtype, after, before, gate, act, bias, mean):
    v, k = case(T, N, stream, dtype, after, before, gate, act, bias, mean)
    scales = (0.5, 1.0) if N % 3 == 0 else (1.0, 0.7)
    first, second = ref.block_norm(**v, **k, residual_scale=scales[0], block_scale=scales[1], eps=1e-6)
    r, x = run(v, k, scales)
    assert r.dtype == stream and r.shape == (T, N)
    check(r, first, "residual")
    if before is None:
        assert x is None
    else:
        assert x.dtype == dtype
        check(x, second, "next")


@pytest.mark.parametrize("T,N", [(3, 64), (40, 4096), (2000, 1024), (3, 77)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_block_norm_without_a_block(T, N, dtype):
    r, w, b = normal((T, N), 1, dtype, 3.0), normal(N, 2, BF, 0.2, 1.0), normal(N, 3)
    for before, weight, bias in (("rms", w, None), ("layer", w, b), ("layer", None, None)):
        _, want = ref.block_norm(r, None, None, None, None, weight, bias, None, before, "none", 1.0, 1.0, 1e-5)
        rd = r.cuda()
        same, x = ap.approxifer_block_norm(rd, next_weight=None if weight is None else weight.cuda(), next_bias=None if bias is None else bias.cuda(), before=before, eps=1e-5)
        assert same is rd
        check(x, want, before)


@pytest.mark.parametrize("T,N", [(2, 512), (1700, 1024), (9, 515)])
def test_block_norm_strides_and_in_place(T, N):
    v, k = case(T, N, F32, BF, "rms", "layer", "element", "sigmoid", True)
    first, second = ref.block_norm(**v, **k, residual_scale=1.0, block_scale=1.0, eps=1e-6)
    wide = {}
    for n in ("residual", "block", "gate"):
        wide[n] = torch.full((T + 1, N + 24), float("nan"), dtype=v[n].dtype, device="cuda")
        wide[n][1:, 8: 8 + N] = v[n].cuda()
    views = {n: w[1:, 8: 8 + N] for n, w in wide.items()}
    rest = {n: t.cuda() for n, t in v.items() if n not in views and t is not None}
    r, x = ap.approxifer_block_norm(**views, **rest, **k, residual_out=views["residual"], next_out=views["block"])
    assert r is views["residual"] and x is views["block"]
    check(r, first, "residual")
    check(x, second, "next")
    for n in ("residual", "block"):  # what lies around the rows is as it was
        views[n].fill_(float("nan"))
        assert bool(torch.isnan(wide[n]).all())


def test_block_norm_of_broadcast_rows_and_of_no_rows():
    T, N = 600, 2048
    v, k = case(T, N, BF, BF, "rms", "rms", "element", "none", False)
    for n in ("residual", "block", "gate"):
        v[n] = v[n][:1].expand(T, N)
    first, second = ref.block_norm(**{n: t if t is None or t.dim() == 1 else t[:1] for n, t in v.items()}, **k, residual_scale=1.0, block_scale=1.0, eps=1e-6)
    dev = {n: None if t is None else t[:1].cuda().expand(T, N) if t.dim() == 2 else t.cuda() for n, t in v.items()}
    r, x = ap.approxifer_block_norm(**dev, **k)
    check(r, (first[0].expand(T, N), first[1].expand(T, N)), "residual")
    check(x, (second[0].expand(T, N), second[1].expand(T, N)), "next")
    r, x = ap.approxifer_block_norm(torch.empty((0, 64), device="cuda"), torch.empty((0, 64), device="cuda"))
    assert r.shape == x.shape == (0, 64)


def test_block_norm_infinities_and_nan_stay_in_their_rows():
    for T, N in ((7, 256), (7, 333), (1300, 2048)):
        v, k = case(T, N, BF, BF, "layer", "rms", "column", "sigmoid", False)
        first, second = ref.block_norm(**v, **k, residual_scale=1.0, block_scale=1.0, eps=1e-6)
        v["block"][2, 5], v["residual"][4, 3] = float("nan"), float("inf")
        r, x = (t.double().cpu() for t in run(v, k))
        assert torch.isnan(r[2]).all() and torch.isnan(x[2]).all() and torch.isinf(r[4, 3]) and torch.isnan(x[4, 3])
        keep = [i for i in range(T) if i not in (2, 4)]
        check(r[keep], (first[0][keep], first[1][keep]), "residual")
        check(x[keep], (second[0][keep], second[1][keep]), "next")


@pytest.mark.parametrize("T,N", [(3, 128), (900, 1024)])
def test_block_norm_of_zeros_and_of_large_rows(T, N):
    zero = torch.zeros((T, N), dtype=F32)
    r, x = run(dict(residual=zero, block=zero, gate=None, block_weight=None, block_bias=None, next_weight=None, next_bias=None), dict(after="rms", before="layer"))
    assert bool((r == 0).all()) and bool((x == 0).all())
    # squares up to 1e36 times the row's length still fit 32 bits
    v, k = case(T, N, F32, F32, "rms", "rms", None, "none", False)
    v["block"] = v["block"] * 1e17
    first, second = ref.block_norm(**v, **k, residual_scale=1.0, block_scale=1.0, eps=0.0)
    r, x = run(v, k, eps=0.0)
    check(r, first, "residual")
    check(x, second, "next")


def test_block_norm_is_repeatable_and_runs_on_a_stream_and_in_a_graph():
    v, k = case(1500, 1024, F32, BF, "layer", "rms", "column", "tanh", True)
    dev = {n: t.cuda() for n, t in v.items()}
    r0, x0 = ap.approxifer_block_norm(**dev, **k)
    for _ in range(3):
        r, x = ap.approxifer_block_norm(**dev, **k)
        assert torch.equal(r, r0) and torch.equal(x, x0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r, x = ap.approxifer_block_norm(**dev, **k, stream=s)
    s.synchronize()
    assert torch.equal(r, r0) and torch.equal(x, x0)
    r, x = torch.zeros_like(r0), torch.zeros_like(x0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ap.approxifer_block_norm(**dev, **k, residual_out=r, next_out=x)
    r.zero_(), x.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(r, r0) and torch.equal(x, x0)
    assert ap.device_wait_timeouts() == 0


def test_block_norm_offsets_beyond_32_bits():
    T, N = 300000, 8192  # 2.5e9 elements
    r = torch.zeros((T, N), dtype=BF, device="cuda")
    rows = [0, 1, 262143, 262144, T - 1]
    some = normal((len(rows), N), 1)
    r[rows] = some.cuda()
    x = ap.approxifer_block_norm(r)[1]
    _, want = ref.block_norm(some, None, None, None, None, None, None, None, "rms", "none", 1.0, 1.0, 1e-6)
    check(x[rows], want, "next")
    assert bool((x[2:262143:997] == 0).all())


def test_block_norm_refuses_what_the_library_cannot_take():
    r, y = normal((4, 64), 1).cuda(), normal((4, 64), 2).cuda()
    w = normal(64, 3).cuda()
    good = dict(residual=r, block=y)
    for bad in (dict(residual=r.cpu()), dict(residual=r[0]), dict(block=y[:3]), dict(block=y.half()), dict(gate=w[:10]), dict(gate=r.float()), dict(after="max"),
                dict(before="max"), dict(gate_activation="relu"), dict(next_weight=w.float()), dict(block_weight=w), dict(residual_out=r.float()),
                dict(before=None, next_weight=w), dict(block=None, residual_out=r), dict(residual=r.t().contiguous().t())):
        with pytest.raises(ValueError):
            ap.approxifer_block_norm(**dict(good, **bad))
    for bad in (dict(block=None, before=None), dict(block=None, gate=w), dict(block=None, residual_scale=0.5), dict(eps=-1.0), dict(residual_scale=float("nan")),
                dict(residual_out=r.expand(4, 64)[:1].expand(4, 64))):
        with pytest.raises(ap.ApproxiferError):
            ap.approxifer_block_norm(**dict(good, **bad))


@pytest.mark.parametrize("T,N", [(1, 5), (9, 77), (300, 515), (40, 1004), (7, 4100), (3, 8189), (3, 8192), (2, 16381), (2, 16382), (2, 16384), (160, 2051), (150, 8189)])
@pytest.mark.parametrize("stream,dtype", [(F32, F32), (F32, BF), (BF, BF)])
def test_block_norm_rows_that_begin_anywhere(T, N, stream, dtype):
    """Rows that lie alike in all arrays, at each distance from a whole address, and rows that do not."""
    gates = ("element", "column", "token", None)
    for i, offsets in enumerate(((1, 1, 1, 1, 1), (2, 2, 2, 2, 2), (3, 7, 3, 3, 11), (0, 0, 0, 0, 0), (1, 2, 3, 4, 5), (0, 0, 1, 0, 0))):
        for pads in ((5, 5, 5, 5, 5), (12, 12, 12, 12, 12), (12, 13, 14, 12, 15)):
            v, k = case(T, N, stream, dtype, "layer" if i % 2 else "rms", "rms" if i % 2 else "layer", gates[i % 4], "sigmoid", i % 3 == 0, 1.0)
            first, second = ref.block_norm(**v, **k, residual_scale=0.5, block_scale=1.0, eps=1e-6)
            dev = {n: None if t is None else t.cuda() for n, t in v.items()}
            types = (stream, dtype, dtype, stream, dtype)
            wide = [torch.full((T + 2, N + 11 + p), 7.0, dtype=t, device="cuda") for p, t in zip(pads, types)]
            views = [w[1: 1 + T, o: o + N] for w, o in zip(wide, offsets)]
            for n, view in zip(("residual", "block", "gate"), views):
                if dev[n] is not None and dev[n].shape == view.shape:
                    view.copy_(dev[n])
                    dev[n] = view
            r, x = ap.approxifer_block_norm(**dev, **k, residual_scale=0.5, block_scale=1.0, eps=1e-6, residual_out=views[3], next_out=views[4])
            check(r, first, "residual")
            check(x, second, "next")
            for w, view in zip(wide[3:], views[3:]):
                view.fill_(7.0)
                assert bool((w == 7.0).all())
