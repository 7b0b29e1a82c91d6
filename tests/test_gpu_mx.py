"""The 4-bit microscaled arrays bit for bit, and approxifer_mx_linear against its 64-bit plain form."""
import pytest
import torch

import hosted_more_reference as ref
import paper_2109_09868_b200 as ap

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def normal(shape, seed, dtype=BF, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def spread(shape, seed, dtype=BF):
    """Magnitudes over a wide range, ties among them, some zeros."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(3 * torch.randn((shape[0], 1), generator=g))
    ties = torch.randint(-16, 17, shape, generator=g) * 0.25
    x = torch.where(torch.rand(shape, generator=g) < 0.3, ties, x)
    return torch.where(torch.rand(shape, generator=g) < 0.05, torch.zeros(()), x).to(dtype)


def special(dtype):
    """Rows of ties at every scale, zeros, the smallest and the largest numbers, infinities and NaN."""
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.9, 0.2, 0.3, 0.0, -0.0, 4.0, 1.0])
    ties = torch.cat([ties, -ties]).to(dtype)
    rows = [ties * 2.0 ** e for e in (0, 1, -1, 20, -20, 100, -100)]
    tiny = torch.finfo(dtype).smallest_normal
    rows += [torch.zeros(32), torch.full((32,), -0.0), torch.full((32,), tiny), ties * tiny, torch.full((32,), torch.finfo(dtype).max), ties / 8 * torch.finfo(dtype).max]
    for bad in (float("inf"), float("-inf"), float("nan")):
        row = ties.clone()
        row[3] = bad
        rows.append(row)
    rows.append(torch.full((32,), 2.0 ** -133))  # below the normal numbers
    return torch.stack([r.to(dtype) for r in rows])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,K", [(1, 32), (3, 64), (31, 96), (33, 128), (128, 160), (129, 2080), (300, 512)])
def test_quantize_bit_for_bit_and_back(M, K, dtype):
    x = spread((M, K), M + K, dtype)
    codes, scales = ap.approxifer_mx_quantize(x.cuda())
    want_codes, want_scales = ref.mx_quantize(x)
    assert torch.equal(scales.cpu(), want_scales)
    assert torch.equal(codes.cpu(), want_codes)
    values = ref.mx_values(want_codes, want_scales)
    for out in (BF, F32):
        assert torch.equal(ap.approxifer_mx_dequantize(codes, scales, out_dtype=out).double().cpu(), values)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantize_special_values(dtype):
    x = special(dtype)
    x = torch.cat([x, x.flip(0), spread(x.shape, 1, dtype)], dim=1)
    codes, scales = ap.approxifer_mx_quantize(x.cuda())
    want_codes, want_scales = ref.mx_quantize(x)
    assert torch.equal(scales.cpu(), want_scales) and torch.equal(codes.cpu(), want_codes)
    back, want = ap.approxifer_mx_dequantize(codes, scales, out_dtype=F32).double().cpu(), ref.mx_values(want_codes, want_scales)
    assert torch.equal(torch.isnan(back), torch.isnan(want)) and torch.equal(back.nan_to_num(), want.nan_to_num())
    # every code at every scale
    codes = torch.arange(256, dtype=torch.uint8)[None, :].expand(256, 256).contiguous()
    byte = torch.arange(256, dtype=torch.int64)
    scales = torch.zeros((2, 4, 512), dtype=torch.uint8)
    for g in range(16):
        scales[byte // 128, g // 4, (byte % 32) * 16 + (byte // 32) % 4 * 4 + g % 4] = byte.to(torch.uint8)
    want = ref.mx_values(codes, scales)
    for out in (BF, F32):
        got = ap.approxifer_mx_dequantize(codes.cuda(), scales.cuda(), out_dtype=out).cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.to(out).nan_to_num())


def test_quantize_strides_and_what_lies_around():
    M, K = 200, 160
    x = spread((M, K), 3)
    want_codes, want_scales = ref.mx_quantize(x)
    for at in (8, 3):  # bases of whole 16 bytes, and others
        wide = torch.full((M, K + 24), float("nan"), dtype=BF, device="cuda")
        wide[:, at: at + K] = x.cuda()
        codes = torch.full((M + 2, K // 2 + 16), 171, dtype=torch.uint8, device="cuda")
        scales = torch.full((2, 2, 512), 99, dtype=torch.uint8, device="cuda")
        room = codes[1:-1, : K // 2]
        a, b = ap.approxifer_mx_quantize(wide[:, at: at + K], codes=room, scales=scales)
        assert a is room and b is scales and torch.equal(room.cpu(), want_codes) and torch.equal(scales.cpu(), want_scales)
        back = torch.full((M + 2, K + 24), 7.0, dtype=BF, device="cuda")
        assert torch.equal(ap.approxifer_mx_dequantize(room, scales, X=back[1:-1, at: at + K]).double().cpu(), ref.mx_values(want_codes, want_scales))
        back[1:-1, at: at + K] = 7.0
        room.fill_(171)
        assert bool((back == 7.0).all()) and bool((codes == 171).all())


def test_quantize_no_rows_and_offsets_beyond_32_bits():
    codes, scales = ap.approxifer_mx_quantize(torch.empty((0, 64), dtype=BF, device="cuda"))
    assert codes.shape == (0, 32) and scales.shape == (0, 1, 512)
    assert ap.approxifer_mx_dequantize(codes, scales).shape == (0, 64)
    M, K = 70000, 65536  # 4.6e9 elements
    x = torch.zeros((M, K), dtype=BF, device="cuda")
    rows = [0, 1, 32768, 65535, 65536, M - 1]
    some = spread((len(rows), K), 5)
    x[rows] = some.cuda()
    codes, scales = ap.approxifer_mx_quantize(x)
    del x
    want_codes, want_scales = ref.mx_quantize(some)
    assert torch.equal(codes[rows].cpu(), want_codes)
    back = ap.approxifer_mx_dequantize(codes, scales)
    assert torch.equal(back[rows].double().cpu(), ref.mx_values(want_codes, want_scales))
    assert bool((back[2:32768:997] == 0).all())


def check(got, want, bound):
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    over = ((got - want).abs() - bound).max()
    assert over <= 0, float(over)


CASES = [  # M, N, K, coded, bias, activation, residual, out
    (1, 1, 32, False, True, "none", True, BF),
    (1, 10, 64, True, False, "none", False, F32),
    (1, 4096, 512, False, False, "none", True, BF),
    (1, 130, 4096, False, True, "silu", False, F32),
    (2, 1000, 800, False, True, "gelu", False, BF),
    (7, 129, 96, True, True, "relu", True, F32),
    (8, 127, 2080, False, False, "none", False, F32),
    (9, 300, 1024, False, True, "gelu", True, BF),
    (16, 256, 1024, True, True, "silu", False, BF),
    (17, 520, 2048, False, False, "gelu_tanh", True, BF),
    (33, 128, 64, False, True, "none", True, BF),
    (64, 257, 288, True, False, "none", True, F32),
    (65, 300, 192, False, True, "silu", True, F32),
    (100, 1000, 96, True, False, "gelu", False, BF),
    (128, 256, 64, False, False, "none", False, BF),
    (129, 257, 160, False, True, "gelu_tanh", True, BF),
    (256, 4224, 544, True, True, "none", False, BF),
    (320, 10, 800, False, True, "none", False, F32),
    (333, 1003, 2080, True, True, "none", False, F32),
    (513, 384, 992, False, True, "relu", True, BF),
    (1000, 1000, 160, True, False, "none", True, F32),
    (2300, 1100, 320, False, True, "gelu", True, BF),
    (3000, 24, 64, True, False, "silu", False, BF),
    (8, 4700, 128, False, False, "silu", True, BF),
    (5, 40, 8192, True, True, "relu", False, BF),
    (4000, 1100, 320, False, True, "gelu", True, BF),
    (4000, 1100, 96, True, True, "gelu_tanh", False, F32),
    (2049, 2305, 544, True, True, "silu", True, F32),
    (6500, 1029, 160, False, True, "relu", True, BF),
    (1800, 3000, 64, True, False, "none", False, BF),
    (40, 33, 32, False, True, "gelu", True, BF),
]


@pytest.mark.parametrize("M,N,K,coded,bias,act,residual,out", CASES)
def test_mx_linear_matches_the_plain_form(M, N, K, coded, bias, act, residual, out):
    x, (w, ws) = spread((M, K), 1), ref.mx_quantize(normal((N, K), 2, std=K ** -0.5))
    xq = ref.mx_quantize(x)
    b = normal((N,), 3) if bias else None
    r = normal((M, N), 4, out) if residual else None
    want, bound = ref.linear(ref.mx_values(*xq), ref.mx_values(w, ws), b, act, r, out)
    dev = [None if t is None else t.cuda() for t in (w, ws, b, r)]
    X, xs = (xq[0].cuda(), xq[1].cuda()) if coded else (x.cuda(), None)
    got = ap.approxifer_mx_linear(X, dev[0], dev[1], x_scales=xs, bias=dev[2], activation=act, residual=dev[3], out_dtype=out)
    assert got.dtype == out and got.shape == (M, N)
    check(got, want, bound)
    assert ap.device_wait_timeouts() == 0


@pytest.mark.parametrize("M", [1, 5, 20, 40, 100, 300, 2600])
def test_mx_linear_takes_the_same_form_of_x_within_the_call(M):
    """bfloat16 X gives what its codes give, bit for bit, also with scales and zeros of every kind."""
    K, N = 1088, 1500
    x = spread((M, K), 5)
    rows = special(BF)[[0, 1, 2, 3, 4, 7, 8, 16]]  # (finite, and no sum overflows)
    x[: len(rows[:M]), :32] = rows[:M]
    x = x.cuda()
    w, ws = ap.approxifer_mx_quantize(normal((N, K), 2, std=0.02).cuda())
    codes, scales = ap.approxifer_mx_quantize(x)
    for out in (BF, F32):
        assert torch.equal(ap.approxifer_mx_linear(x, w, ws, out_dtype=out), ap.approxifer_mx_linear(codes, w, ws, x_scales=scales, out_dtype=out))


@pytest.mark.parametrize("M,N,K", [(1, 200, 256), (3, 200, 256), (150, 328, 224), (700, 512, 512), (2100, 1800, 224)])
def test_mx_linear_strides_guards_and_the_residual_in_place(M, N, K):
    x, r = spread((M, K), 1), normal((M, N), 3)
    w, ws = ref.mx_quantize(normal((N, K), 2, std=K ** -0.5))
    xq = ref.mx_quantize(x)
    want, bound = ref.linear(ref.mx_values(*xq), ref.mx_values(w, ws), None, "none", r, BF)
    wp = torch.full((N + 1, K // 2 + 32), 0x77, dtype=torch.uint8, device="cuda")
    wp[1:, 16: 16 + K // 2] = w.cuda()
    wv, wsd = wp[1:, 16: 16 + K // 2], ws.cuda()
    y = torch.full((M + 2, N + 16), 7.0, dtype=BF, device="cuda")
    view = y[1:-1, 8: 8 + N]
    for at in (8, 3):
        view.copy_(r.cuda())
        xp = torch.full((M, K + 24), float("nan"), dtype=BF, device="cuda")
        xp[:, at: at + K] = x.cuda()
        assert ap.approxifer_mx_linear(xp[:, at: at + K], wv, wsd, residual=view, Y=view) is view
        check(view, want, bound)
    cp = torch.full((M + 1, K // 2 + 16), 0x77, dtype=torch.uint8, device="cuda")
    cp[1:, : K // 2] = xq[0].cuda()
    yo = torch.full((M, N + 3), 7.0, dtype=BF, device="cuda")
    check(ap.approxifer_mx_linear(cp[1:, : K // 2], wv, wsd, x_scales=xq[1].cuda(), residual=r.cuda(), Y=yo[:, 1: 1 + N]), want, bound)
    view.fill_(7.0)
    yo[:, 1: 1 + N] = 7.0
    assert bool((y == 7.0).all()) and bool((yo == 7.0).all())


@pytest.mark.parametrize("M,N,K", [(5, 140, 128), (40, 140, 128), (300, 200, 160), (2500, 1300, 128)])
def test_mx_linear_nan_stays_in_its_rows_and_columns(M, N, K):
    x, w = spread((M, K), 1), normal((N, K), 2, std=K ** -0.5)
    x[2, 5], x[4, 7] = float("nan"), float("inf")
    w[7, 3] = float("inf")
    wq = ref.mx_quantize(w)
    xq = ref.mx_quantize(x)
    want, bound = ref.linear(ref.mx_values(*xq).nan_to_num(), ref.mx_values(*wq).nan_to_num(), None, "none", None, BF)
    got = ap.approxifer_mx_linear(x.cuda(), wq[0].cuda(), wq[1].cuda()).double().cpu()
    assert torch.isnan(got[[2, 4]]).all() and torch.isnan(got[:, 7]).all()
    rows, cols = [i for i in range(M) if i not in (2, 4)], [i for i in range(N) if i != 7]
    check(got[rows][:, cols], want[rows][:, cols], bound[rows][:, cols])


@pytest.mark.parametrize("M,N", [(1, 40), (20, 300), (300, 1003), (3000, 1400), (3000, 1003)])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("out", [BF, F32])
def test_mx_linear_activations_at_their_ends(M, N, act, out):
    """Infinities, NaN, the largest and very negative numbers before the activation: what the formula makes of them in 64 bits."""
    x, w = spread((M, 64), 1), ref.mx_quantize(normal((N, 64), 2, std=0.1))
    ends = torch.tensor([float("inf"), float("-inf"), float("nan"), 3e38, -3e38, 1e5, -1e5, 95.0, -95.0, 0.0], dtype=BF)
    b = ends.repeat(N // len(ends) + 1)[:N].contiguous()
    z = ref.mx_values(*ref.mx_quantize(x)) @ ref.mx_values(*w).T + b.double()
    f = torch.nn.functional
    want = {"none": lambda t: t, "relu": f.relu, "gelu": f.gelu, "gelu_tanh": lambda t: f.gelu(t, approximate="tanh"), "silu": f.silu}[act](z)
    _, bound = ref.linear(ref.mx_values(*ref.mx_quantize(x)), ref.mx_values(*w), torch.where(torch.isfinite(b), b, torch.zeros_like(b)), act, None, out)
    got = ap.approxifer_mx_linear(x.cuda(), w[0].cuda(), w[1].cuda(), bias=b.cuda(), activation=act, out_dtype=out).double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got == float("inf"), want == float("inf")) and torch.equal(got == float("-inf"), want == float("-inf"))
    finite = torch.isfinite(want)
    assert ((got - want).abs() <= bound)[finite].all()


@pytest.mark.parametrize("M", [1, 24, 300, 3000])
def test_mx_linear_is_repeatable_and_runs_on_a_stream_and_in_a_graph(M):
    x, b = spread((M, 2048), 1).cuda(), normal((1024,), 3).cuda()
    w, ws = ap.approxifer_mx_quantize(normal((1024, 2048), 2, std=0.02).cuda())
    first = ap.approxifer_mx_linear(x, w, ws, bias=b, activation="gelu")
    for _ in range(3):
        assert torch.equal(ap.approxifer_mx_linear(x, w, ws, bias=b, activation="gelu"), first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = ap.approxifer_mx_linear(x, w, ws, bias=b, activation="gelu", stream=s)
    s.synchronize()
    assert torch.equal(y, first)
    out = torch.zeros_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ap.approxifer_mx_linear(x, w, ws, bias=b, activation="gelu", Y=out)
        ap.approxifer_mx_linear(x, w, ws, bias=b, activation="gelu", Y=out)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)


def test_mx_linear_of_no_rows_and_offsets_beyond_32_bits():
    w, ws = ap.approxifer_mx_quantize(normal((33000, 64), 2, std=0.1).cuda())
    assert ap.approxifer_mx_linear(torch.empty((0, 64), dtype=BF, device="cuda"), w, ws).shape == (0, 33000)
    codes, scales = ap.approxifer_mx_quantize(torch.empty((0, 64), dtype=BF, device="cuda"))
    assert ap.approxifer_mx_linear(codes, w, ws, x_scales=scales).shape == (0, 33000)
    M = 66000  # 2.18e9 outputs
    x = normal((M, 64), 1)
    y = ap.approxifer_mx_linear(x.cuda(), w, ws)
    rows = [0, 1, 40000, 65071, 65072, M - 1]
    want, bound = ref.linear(ref.mx_values(*ref.mx_quantize(x[rows])), ref.mx_values(w.cpu(), ws.cpu()), None, "none", None, BF)
    check(y[rows], want, bound)


def test_mx_refuses_what_the_library_cannot_take():
    x = normal((4, 64), 1).cuda()
    w, ws = ap.approxifer_mx_quantize(normal((8, 64), 2).cuda())
    xq, xs = ap.approxifer_mx_quantize(x)
    for bad in (dict(X=x.float()), dict(X=x[:, :32]), dict(X=xq), dict(weight=w[:, :16]), dict(weight_scales=ws[:, :, :256]), dict(weight_scales=xs.cpu()), dict(x_scales=xs),
                dict(X=xq[:, :16], x_scales=xs), dict(bias=x[0]), dict(residual=x), dict(activation="tanh"), dict(out_dtype=torch.float16), dict(X=x.cpu()), dict(X=x[0]),
                dict(Y=torch.empty((4, 8), device="cuda").bfloat16(), out_dtype=F32), dict(X=x.t().contiguous().t())):
        with pytest.raises(ValueError):
            ap.approxifer_mx_linear(**dict(dict(X=x, weight=w, weight_scales=ws), **bad))
    odd = torch.zeros((8, 40), dtype=torch.uint8, device="cuda")[:, :32]  # rows 40 bytes apart
    for bad in (dict(weight=odd), dict(X=odd[:4], x_scales=xs)):
        with pytest.raises(ap.ApproxiferError):
            ap.approxifer_mx_linear(**dict(dict(X=x, weight=w, weight_scales=ws), **bad))
    for bad in (dict(X=x[:, :40]), dict(X=x.half()), dict(X=x.cpu()), dict(X=x, codes=xq[:3]), dict(X=x, codes=xq, scales=ws[:, :, :1])):
        with pytest.raises(ValueError):
            ap.approxifer_mx_quantize(**bad)
    for bad in (dict(codes=xq, scales=xs[0]), dict(codes=xq.int(), scales=xs), dict(codes=xq, scales=xs, out_dtype=torch.float16), dict(codes=xq, scales=xs, X=x[:3])):
        with pytest.raises(ValueError):
            ap.approxifer_mx_dequantize(**bad)
