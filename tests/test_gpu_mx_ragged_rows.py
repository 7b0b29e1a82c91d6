"""approxifer_mx_linear into rows that end within 16 bytes while their stride is of whole 16 bytes: a column slice of a wider array.  What
lies behind the rows stays as it is, between them and behind the last one."""
import pytest
import torch

import hosted_more_reference as ref
import paper_2109_09868_b200 as ap

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def normal(shape, seed, dtype=BF, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("M,N", [(1, 130), (20, 77), (300, 133), (300, 1003), (2500, 1537), (2500, 1538), (2500, 1539), (2311, 1543), (2500, 1540), (2500, 1599), (2049, 1345),
                                 (1800, 1921), (2500, 1536)])
def test_what_lies_behind_the_rows_stays(M, N, out):
    K = 96
    x, w, b, r = normal((M, K), 1), normal((N, K), 2, std=K ** -0.5), normal((N,), 3), normal((M, N), 4, out)
    xq, (wc, ws) = ref.mx_values(*(t.cpu() for t in ap.approxifer_mx_quantize(x.cuda()))), ap.approxifer_mx_quantize(w.cuda())
    wq = ref.mx_values(wc.cpu(), ws.cpu())
    whole = 16 // r.element_size()
    for act, residual, in_place in (("none", False, False), ("silu", True, False), ("relu", True, True)):
        want, bound = ref.linear(xq, wq, b, act, r if residual else None, out)
        stride = (N + whole - 1) // whole * whole + whole * (1 if in_place else 0)
        room = torch.full((M * stride + whole,), 7.0, dtype=out, device="cuda")
        view = room[whole:].view(M, stride)[:, :N]
        res = r.cuda() if residual else None
        if in_place:
            view.copy_(res)
            res = view
        assert ap.approxifer_mx_linear(x.cuda(), wc, ws, bias=b.cuda(), activation=act, residual=res, Y=view) is view
        got = view.double().cpu()
        assert torch.isfinite(got).all() and ((got - want).abs() <= bound).all()
        view.fill_(7.0)
        assert bool((room == 7.0).all())
    assert ap.device_wait_timeouts() == 0


@pytest.mark.parametrize("out", [BF, F32])
def test_two_products_side_by_side(out):
    """Columns of one array, the second product's first."""
    M, K, first, second = 2400, 64, 1539, 1501
    x = normal((M, K), 1).cuda()
    y = torch.empty((M, first + second), dtype=out, device="cuda")
    parts = y[:, :first], y[:, first:]
    want = []
    for i, (n, part) in reversed(list(enumerate(((first, parts[0]), (second, parts[1]))))):
        w, ws = ap.approxifer_mx_quantize(normal((n, K), 5 + i).cuda())
        ap.approxifer_mx_linear(x, w, ws, Y=part)
        want.insert(0, ap.approxifer_mx_linear(x, w, ws, out_dtype=out))
    assert torch.equal(parts[0], want[0]) and torch.equal(parts[1], want[1])
