"""approxifer_linear against its 64-bit plain form: shapes from one row to several tiles, odd sizes, strides, unaligned
bases, every activation, bias and residual present or not, both output types."""
import math

import pytest
import torch

import hosted_reference as ref
import paper_2109_09868_b200 as ap

pytestmark = pytest.mark.gpu


def normal(shape, seed, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def check(got, want, bound):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    over = ((got - want).abs() - bound).max()
    assert over <= 0, float(over)


CASES = [  # M, N, K, bias, activation, residual, out
    (1, 1, 1, True, "none", True, torch.bfloat16),
    (1, 10, 8, False, "none", False, torch.float32),
    (1, 4096, 512, False, "none", True, torch.bfloat16),
    (2, 1000, 784, True, "gelu", False, torch.bfloat16),
    (7, 129, 72, True, "relu", True, torch.float32),
    (16, 256, 1024, True, "silu", False, torch.bfloat16),
    (17, 520, 2048, False, "gelu_tanh", True, torch.bfloat16),
    (33, 128, 64, True, "none", True, torch.bfloat16),
    (65, 300, 200, True, "silu", True, torch.float32),
    (100, 1000, 96, False, "gelu", False, torch.bfloat16),
    (128, 256, 64, False, "none", False, torch.bfloat16),
    (129, 257, 136, True, "gelu_tanh", True, torch.bfloat16),
    (320, 10, 784, True, "none", False, torch.float32),
    (513, 384, 1000, True, "relu", True, torch.bfloat16),
    (1000, 1000, 160, False, "none", True, torch.float32),
    (2300, 1100, 320, True, "gelu", True, torch.bfloat16),
    (3000, 24, 64, False, "silu", False, torch.bfloat16),
    (3, 1003, 2056, True, "gelu", True, torch.float32),      # few rows: K in turns of 1,024, odd N
    (8, 4700, 136, False, "silu", True, torch.bfloat16),
    (5, 40, 8192, True, "relu", False, torch.bfloat16),
    (8, 50, 8200, True, "none", True, torch.float32),
    (4000, 1100, 320, True, "gelu", True, torch.bfloat16),   # many tiles: pairs of CTAs
    (4000, 1100, 72, True, "gelu_tanh", False, torch.float32),
    (2049, 2305, 520, True, "silu", True, torch.float32),
    (6500, 1029, 136, True, "relu", True, torch.bfloat16),
    (1800, 3000, 64, False, "none", False, torch.bfloat16),
    (40, 33, 77, True, "gelu", True, torch.bfloat16),      # odd K: rows are not whole 16 bytes
    (300, 65, 13, False, "relu", False, torch.float32),
]


@pytest.mark.parametrize("M,N,K,bias,act,residual,out", CASES)
def test_linear_matches_the_plain_form(M, N, K, bias, act, residual, out):
    x, w = normal((M, K), 1), normal((N, K), 2, std=K ** -0.5)
    b = normal((N,), 3) if bias else None
    r = normal((M, N), 4, out) if residual else None
    want, bound = ref.linear(x, w, b, act, r, out)
    dev = [None if t is None else t.cuda() for t in (x, w, b, r)]
    got = ap.approxifer_linear(dev[0], dev[1], bias=dev[2], activation=act, residual=dev[3], out_dtype=out)
    assert got.dtype == out and got.shape == (M, N)
    check(got, want, bound)


@pytest.mark.parametrize("M,N,K", [(3, 200, 256), (150, 328, 200), (700, 512, 512), (2100, 1800, 200)])
def test_linear_strides_guards_and_the_residual_in_place(M, N, K):
    x, w, r = normal((M, K), 1), normal((N, K), 2, std=K ** -0.5), normal((M, N), 3)
    want, bound = ref.linear(x, w, None, "none", r, torch.bfloat16)
    xp = torch.full((M, K + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wp = torch.full((N, K + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    y = torch.full((M + 2, N + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    xp[:, 16:16 + K], wp[:, :K] = x.cuda(), w.cuda()
    y[1:-1, 8:8 + N] = r.cuda()
    view = y[1:-1, 8:8 + N]
    got = ap.approxifer_linear(xp[:, 16:16 + K], wp[:, :K], residual=view, Y=view)
    check(got, want, bound)
    view.fill_(7.0)
    assert bool((y == 7.0).all())
    # the same numbers from bases that are not whole 16 bytes
    odd = torch.full((M, K + 3), float("nan"), dtype=torch.bfloat16, device="cuda")
    odd[:, 3:] = x.cuda()
    yo = torch.empty((M, N + 1), dtype=torch.bfloat16, device="cuda")
    check(ap.approxifer_linear(odd[:, 3:], wp[:, :K], residual=r.cuda(), Y=yo[:, 1:]), want, bound)
    # an aligned product into an output whose rows are not whole 16 bytes
    check(ap.approxifer_linear(xp[:, 16:16 + K], wp[:, :K], residual=r.cuda(), Y=yo[:, 1:]), want, bound)


def test_linear_infinities_and_nan_stay_in_their_rows():
    for M, N, K in ((5, 140, 128), (300, 200, 128), (2500, 1300, 128)):
        x, w = normal((M, K), 1), normal((N, K), 2, std=K ** -0.5)
        want, bound = ref.linear(x, w, None, "relu", None, torch.bfloat16)
        x[2, 5], x[4, 7] = float("nan"), float("inf")
        got = ap.approxifer_linear(x.cuda(), w.cuda(), activation="relu").double().cpu()
        assert torch.isnan(got[2]).all() and torch.equal(torch.isinf(got[4]), w[:, 7].double() > 0)
        keep = [i for i in range(M) if i not in (2, 4)]
        check(got[keep], want[keep], bound[keep])


def test_linear_is_repeatable_and_runs_on_a_stream_and_in_a_graph():
    x, w, b = normal((24, 2048), 1).cuda(), normal((1024, 2048), 2, std=0.02).cuda(), normal((1024,), 3).cuda()
    first = ap.approxifer_linear(x, w, bias=b, activation="gelu")
    for _ in range(5):
        assert torch.equal(ap.approxifer_linear(x, w, bias=b, activation="gelu"), first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = ap.approxifer_linear(x, w, bias=b, activation="gelu", stream=s)
    s.synchronize()
    assert torch.equal(y, first)
    out = torch.zeros_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ap.approxifer_linear(x, w, bias=b, activation="gelu", Y=out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first)


def test_linear_on_another_stream_leaves_memory_alone_that_the_current_one_still_reads():
    x, w = normal((512, 512), 1).cuda(), normal((1024, 512), 2, std=0.05).cuda()
    s = torch.cuda.Stream()
    want = ap.approxifer_linear(x, w)
    torch.cuda.synchronize()
    for _ in range(5):
        held = torch.full((512, 1024), 3.0, dtype=torch.bfloat16, device="cuda")
        copy = torch.empty_like(held)
        s.wait_stream(torch.cuda.current_stream())
        torch.cuda._sleep(20_000_000)  # (some 10 ms)
        copy.copy_(held)               # still to come when the block is given back ...
        del held
        y = ap.approxifer_linear(x, w, stream=s)  # ... and an output of the same size is asked for
        s.synchronize()
        torch.cuda.synchronize()
        assert bool((copy == 3.0).all()) and torch.equal(y, want)


@pytest.mark.parametrize("M,K", [(2, 64), (40, 64), (300, 64), (2600, 64), (20, 13)])
def test_linear_activations_keep_their_relative_accuracy_in_fp32(M, K):
    """Sums that are exact (one element of each row of X is 1), so that only the activation errs: x / (1 + e^-x) by at most 2^-23 for
    each of the exponential (twice that), the sum and the quotient, relative to the result, also where that is small."""
    N = 1200 if M == 2600 else 200
    x = torch.zeros((M, K))
    x[:, 3] = 1
    w = torch.zeros((N, K))
    w[:, 3] = torch.linspace(-80, 12, N)
    x, w = x.bfloat16(), w.bfloat16()
    z = w[:, 3].double()
    want = (z / (1 + torch.exp(-z))).expand(M, N)
    got = ap.approxifer_linear(x.cuda(), w.cuda(), activation="silu", out_dtype=torch.float32).double().cpu()
    assert ((got - want).abs() <= 4 * 2.0 ** -23 * want.abs() + 2.0 ** -130).all()
    # gelu by tanh: x / (1 + e^u) with u = -2 sqrt(2/pi) (x + 0.044715 x^3) in some six operations, each an error of e^u that grows with |u|
    u = -2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    want = (z / (1 + torch.exp(u))).expand(M, N)
    got = ap.approxifer_linear(x.cuda(), w.cuda(), activation="gelu_tanh", out_dtype=torch.float32).double().cpu()
    near = u.expand(M, N) < 80
    over = (got - want).abs() - ((6 * u.abs() + 4) * 2.0 ** -23 * want.abs() + 2.0 ** -100)
    assert (over[near] <= 0).all()


@pytest.mark.parametrize("M,N", [(3, 70), (40, 70), (300, 200), (2500, 1300)])
@pytest.mark.parametrize("K", [1, 13, 77, 201])
def test_linear_rows_of_odd_length_in_whole_columns(M, N, K):
    """Rows of any length K at strides of whole 16 bytes run on the tensor cores; what lies behind a row is NaN."""
    x, w = normal((M, K), 1), normal((N, K), 2, std=K ** -0.5)
    want, bound = ref.linear(x, w, None, "silu", None, torch.float32)
    wide = (K + 15) // 8 * 8
    xp = torch.full((M, wide), float("nan"), dtype=torch.bfloat16, device="cuda")
    wp = torch.full((N, wide), float("nan"), dtype=torch.bfloat16, device="cuda")
    xp[:, :K], wp[:, :K] = x.cuda(), w.cuda()
    check(ap.approxifer_linear(xp[:, :K], wp[:, :K], activation="silu", out_dtype=torch.float32), want, bound)


def test_linear_of_no_rows():
    assert ap.approxifer_linear(torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((5, 64), dtype=torch.bfloat16, device="cuda")).shape == (0, 5)


def test_linear_output_offsets_beyond_32_bits():
    M, N, K = 66000, 33000, 64  # 2.18e9 elements
    x, w = normal((M, K), 1), normal((N, K), 2, std=K ** -0.5)
    y = ap.approxifer_linear(x.cuda(), w.cuda())
    rows = [0, 1, 40000, 65071, 65072, M - 1]
    want, bound = ref.linear(x[rows], w, None, "none", None, torch.bfloat16)
    check(y[rows], want, bound)


def test_linear_refuses_what_the_library_cannot_take():
    x, w = normal((4, 64), 1).cuda(), normal((8, 64), 2).cuda()
    for bad in (dict(X=x.float()), dict(weight=w[:, :32]), dict(bias=x[0]), dict(residual=x), dict(activation="tanh"), dict(out_dtype=torch.float16), dict(X=x.cpu()),
                dict(X=x[0]), dict(Y=torch.empty((4, 8), device="cuda").bfloat16(), out_dtype=torch.float32), dict(X=x.t().contiguous().t())):
        with pytest.raises(ValueError):
            ap.approxifer_linear(**dict(dict(X=x, weight=w), **bad))
