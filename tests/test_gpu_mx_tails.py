"""approxifer_mx_linear's activations far below zero, where their results are small and keep their relative accuracy.

The sum before the activation is the bias alone (all codes are zero), exact in fp32.  Bounds: a bfloat16 output is rounded by at most
2^-8 of it; the function itself errs by at most 8e-4 (gelu, bfloat16: the fit behind it), 1e-4 (silu, gelu_tanh: an exponential whose
argument of up to 126 is rounded twice or three times by 2^-24: 3 126 2^-24 ln 2 = 1.6e-5, and a few units), with an fp32 output as much.
The quotient may be taken as zero where it is below 2^-126: |x| 2^-126 more, and as much for results below the normal numbers."""
import pytest
import torch

import paper_2109_09868_b200 as ap

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def exact(act, x):
    if act == "gelu":
        return 0.5 * x * torch.special.erfc(-x * 0.5 ** 0.5)
    u = x if act == "silu" else 2 * (2 / torch.pi) ** 0.5 * (x + 0.044715 * x ** 3)
    return torch.where(u < -700, torch.zeros_like(x), x * torch.sigmoid(u))


@pytest.mark.parametrize("M,N", [(1, 600), (20, 600), (300, 600), (2600, 1500)])  # each kernel
@pytest.mark.parametrize("act,out", [("gelu", BF), ("gelu_tanh", BF), ("silu", BF), ("gelu_tanh", F32), ("silu", F32)])
def test_small_results_keep_their_accuracy(M, N, act, out):
    w, ws = ap.approxifer_mx_quantize(torch.zeros((N, 32), dtype=BF, device="cuda"))
    lowest = -100.0 if act == "silu" else -14.0
    x = torch.cat([torch.linspace(lowest, 0, N - 200), torch.linspace(-6, 6, 150), -torch.logspace(-20, 0, 50)]).to(BF)
    got = ap.approxifer_mx_linear(torch.zeros((M, 32), dtype=BF, device="cuda"), w, ws, bias=x.cuda(), activation=act, out_dtype=out).double().cpu()
    x = x.double()
    want = exact(act, x)
    bound = ((2.0 ** -8 if out == BF else 2.0 ** -23) + (8e-4 if act == "gelu" else 1e-4)) * want.abs() + (x.abs() + 1) * 2.0 ** -126
    over = ((got - want).abs() - bound).amax(0)
    assert over.max() <= 0, [(float(x[i]), float(got[0, i]), float(want[i])) for i in over.topk(3).indices]
