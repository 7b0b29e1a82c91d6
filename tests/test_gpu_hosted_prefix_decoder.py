"""The operators of examples/hosted_prefix_decoder.py in the run in which they are used: every call's output against the 64-bit plain
form of what that call was given, prompt and single tokens, and the whole captured into a graph."""
import importlib.util
import os
import subprocess
import sys

import pytest
import torch

import hosted_more_reference as ref
import hosted_reference
import paper_2109_09868_b200 as ap

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PATH = os.path.join(ROOT, "examples", "hosted_prefix_decoder.py")


def example():
    spec = importlib.util.spec_from_file_location("hosted_prefix_decoder", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def within(got, want, name):
    value, bound = want
    got = got.double().cpu()
    assert torch.isfinite(got).all(), name
    over = ((got - value).abs() - bound).max()
    assert over <= 0, (name, float(over))


class Checked:
    """The package's operators, each call compared with its plain form."""

    def __init__(self):
        self.calls = []

    def approxifer_mx_quantize(self, x):
        codes, scales = ap.approxifer_mx_quantize(x)
        want = ref.mx_quantize(x.cpu())
        assert torch.equal(codes.cpu(), want[0]) and torch.equal(scales.cpu(), want[1])
        return codes, scales

    def approxifer_mx_linear(self, x, weight, scales, bias=None, activation="none"):
        y = ap.approxifer_mx_linear(x, weight, scales, bias=bias, activation=activation)
        xq = ref.mx_values(*ref.mx_quantize(x.cpu()))
        within(y, hosted_reference.linear(xq, ref.mx_values(weight.cpu(), scales.cpu()), None if bias is None else bias.cpu(), activation, None, y.dtype), "mx_linear")
        self.calls.append("mx_linear")
        return y

    def approxifer_block_norm(self, residual, block=None, gate=None, block_weight=None, next_weight=None, after=None, gate_activation="none", residual_out=None):
        args = [None if t is None else t.cpu() for t in (residual, block, gate, block_weight, None, next_weight, None)]  # (before it is written over)
        first, second = ref.block_norm(*args, after, "rms", gate_activation, 1.0, 1.0, 1e-6)
        r, x = ap.approxifer_block_norm(residual, block, gate=gate, block_weight=block_weight, next_weight=next_weight, after=after, gate_activation=gate_activation,
                                        residual_out=residual_out)
        within(r, first, "residual")
        within(x, second, "next")
        self.calls.append("block_norm")
        return r, x

    def approxifer_qk_norm_rope(self, *args):
        return ap.approxifer_qk_norm_rope(*args)

    def approxifer_prefix_attention(self, q, k_cache, v_cache, prefix_table, prefix, table, start, length, max_q):
        out = ap.approxifer_prefix_attention(q, k_cache, v_cache, prefix_table, prefix, table, start, length, max_q)
        within(out, ref.prefix_attention(*[t.cpu() for t in (q, k_cache, v_cache, prefix_table)], prefix, table.cpu(), start.cpu(), length.cpu(), q.shape[2] ** -0.5), "attention")
        self.calls.append("attention")
        return out

    def approxifer_linear(self, x, weight, out_dtype):
        return ap.approxifer_linear(x, weight, out_dtype=out_dtype)


@pytest.mark.parametrize("heads,kv_heads,head,page", [(8, 2, 32, 16), (4, 4, 64, 8), (2, 1, 128, 32)])
def test_every_call_of_a_run_matches_its_plain_form(heads, kv_heads, head, page):
    sequences, prefix, width = 5, 75, 256
    ops = Checked()
    decoder = example().PrefixDecoder(sequences, prefix, 24, width=width, heads=heads, kv_heads=kv_heads, head=head, page=page, ops=ops)
    g = torch.Generator().manual_seed(1)
    decoder.prompt(torch.randn((prefix, width), generator=g).bfloat16().cuda())
    for n in (9, 1, 1, 3):
        y = decoder(torch.randn((sequences, n, width), generator=g).bfloat16().cuda())
        assert y.shape == (sequences, 10) and torch.isfinite(y).all()
    assert ops.calls.count("attention") == 5 * 2 and ops.calls.count("mx_linear") == 5 * 2 * 4 and ops.calls.count("block_norm") == 5 * 5
    assert ap.device_wait_timeouts() == 0


def test_a_step_in_a_graph_repeats_the_step():
    sequences, prefix, width = 6, 130, 256
    g = torch.Generator().manual_seed(2)
    prompt, x = torch.randn((prefix, width), generator=g).bfloat16().cuda(), torch.randn((sequences, 1, width), generator=g).bfloat16().cuda()
    decoder = example().PrefixDecoder(sequences, prefix, 8, width=width)
    decoder.prompt(prompt)
    want = decoder(x)
    decoder.length = 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = decoder(x)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_a_common_prompt_is_its_own_code():
    """K equal queries are encoded to themselves: the weights of a coded query sum to one, up to their own rounding (a sum of K
    weighted terms in fp32: (K + 2) 2^-23 of the sum of their magnitudes), and bfloat16 rounds it once more."""
    for K, W in ((4, 6), (8, 12)):
        p = ap.make_params(K, W)
        x = torch.randn((1, 1, 4096), generator=torch.Generator().manual_seed(3)).bfloat16().cuda().expand(1, K, 4096).contiguous()
        coded = ap.approxifer_encode_bf16(p, x)
        size = ap.approxifer_debug_weights(p).abs().sum(1).max().item()
        err = (coded.double() - x[:, :1].double()).abs()
        assert bool((err <= (2.0 ** -8 + 2 * (K + 2) * 2.0 ** -23 * size) * x[:, :1].double().abs()).all())


def test_the_example_runs():
    done = subprocess.run([sys.executable, PATH], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr
    assert done.stdout.count("step") == 3 and "nan" not in done.stdout
