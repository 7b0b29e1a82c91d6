"""The hosted-model operators together, as the example runs them: against the same decoder in plain 64-bit operations, and the
same tokens taken at once, in chunks and one by one."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2109_09868_b200 as ap

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


def example():
    spec = importlib.util.spec_from_file_location("hosted_decoder", os.path.join(os.path.dirname(HERE), "examples", "hosted_decoder.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain(decoder, x):
    """All tokens of x [sequences][tokens][width] in 64 bits -> predictions after each of them."""
    h = x.double()
    B, T, _ = h.shape
    H, Hk, D = decoder.heads, decoder.kv_heads, decoder.head
    cs = decoder.cos_sin.double()[:T]
    c, s = cs[:, None, : D // 2], cs[:, None, D // 2:]
    at = torch.arange(T, device=x.device)
    seen = at[None, :] <= at[:, None]
    if decoder.window:
        seen &= (at[None, :] > at[:, None] - decoder.window) | (at[None, :] < decoder.sinks)

    def turn(y, w):
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w.double()
        a, b = y[..., : D // 2], y[..., D // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    for w in decoder.layers:
        q, k, v = (h @ w["qkv"].double().T + w["qkv_bias"].double()).split([H * D, Hk * D, Hk * D], -1)
        q, k = turn(q.unflatten(-1, (H, D)), w["q_norm"]), turn(k.unflatten(-1, (Hk, D)), w["k_norm"])
        k, v = (t.repeat_interleave(H // Hk, dim=2) for t in (k, v.unflatten(-1, (Hk, D))))
        p = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(D)
        p = torch.softmax(p.masked_fill(~seen, -math.inf), -1)
        h = h + torch.einsum("bhij,bjhd->bihd", p, v).flatten(2) @ w["out"].double().T
        u = h @ w["up"].double().T + w["up_bias"].double()
        h = h + (u * 0.5 * (1 + torch.erf(u / math.sqrt(2)))) @ w["down"].double().T
    return h @ decoder.classes.double().T


# Two layers of five bfloat16 roundings each on a residual stream: every rounding is at most 2^-8 of its value, they add up
# like independent errors (the square root of ten of them) to some 1.2 % of the stream, and the head mixes 256 such elements
# into predictions of the stream's own size.  4 % of the predictions' root mean square leaves a factor of three.
TOLERANCE = 0.04


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_the_decoder_agrees_with_plain_operations_however_the_tokens_come(window, sinks):
    E = example()
    B, T = 3, 61
    x = torch.randn((B, T, 256), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    make = lambda: E.HostedDecoder(B, T, window=window, sinks=sinks, seed=5)  # noqa: E731
    want = plain(make(), x)
    size = want.square().mean().sqrt()
    for chunks in ([T], [40, 21], [33] + [1] * (T - 33), [1] * T):
        decoder, at = make(), 0
        for n in chunks:
            got = decoder(x[:, at: at + n])
            at += n
            error = (got.double() - want[:, at - 1]).square().mean().sqrt() / size
            assert error <= TOLERANCE, (chunks[:3], at, float(error))
        if window and len(chunks) > 2:
            assert len(decoder.free) > 0  # pages that left the window were freed


def test_the_example_runs(capsys):
    before = ap.launch_count()
    example().main()
    out = capsys.readouterr().out
    assert out.count("step") == 3 and "nan" not in out
    assert ap.launch_count() - before > 41 * 2 * 6
    assert ap.device_wait_timeouts() == 0
