"""What a captured call reads is what the kernels before it have just written: lengths, starts, tables, queries and caches that differ from
replay to replay, in each form of approxifer_prefix_attention, and through a whole step of the example's decoder.  (The kernels over the
sequences' own keys start before the kernel over the prefix ends; they may, because that kernel has waited for what came before the call.)"""
import importlib.util
import os

import pytest
import torch

import paper_2109_09868_b200 as ap
from test_gpu_prefix import problem
from test_gpu_prefix_forms import CASES

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def two_of_a_kind(prefix, kv, qs, Hq, Hkv, D, page):
    """Two problems whose arrays have the same shapes and whose lengths, starts, tables and values differ."""
    def pages(lengths):
        return sum((n + page - 1) // page for n in [prefix] + lengths)

    shorter = [kv[0]] + [max(1, n - 7 * i) for i, n in enumerate(kv)][1:]
    if max(shorter) != max(kv):
        shorter[kv.index(max(kv))] = max(kv)
    a = problem(prefix, kv, qs, Hq, Hkv, D, page, seed=1)
    b = problem(prefix, shorter, qs[::-1], Hq, Hkv, D, page, seed=20, spare=3 + pages(kv) - pages(shorter))
    assert all(a[n].shape == b[n].shape for n in a if isinstance(a[n], torch.Tensor))
    return a, b


@pytest.mark.parametrize("case", [0, 1, 3, 5, 6, 7, 8, 9, 11, 12, 13, 15, 16, 17, 19])
def test_a_captured_call_reads_what_was_written_just_before(case):
    _, prefix, kv, qs, Hq, Hkv, D, page = CASES[case]
    both = [{n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in p.items()} for p in two_of_a_kind(prefix, kv, qs, Hq, Hkv, D, page)]
    want = []
    for p in both:
        want.append(ap.approxifer_prefix_attention(**p, max_q=max(qs), scale=0.1))
        torch.cuda.synchronize()
    arrays = [n for n, t in both[0].items() if isinstance(t, torch.Tensor)]
    source, live = ({n: torch.zeros_like(both[0][n]) for n in arrays} for _ in range(2))
    room = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(want[0]) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for out in outs:  # (the second time round they write over what the first call has read, and its workspace)
            for n in arrays:
                live[n].zero_()
            for n in ["k_cache", "v_cache", "q", "prefix_table", "block_table", "q_start", "kv_len"]:  # (kernels; the lengths come last)
                torch.mul(source[n], 1, out=live[n])
            ap.approxifer_prefix_attention(**live, prefix_len=prefix, max_q=max(qs), scale=0.1, workspace=room, out=out)
    for i in (0, 1, 1, 0, 1):
        for n in arrays:
            source[n].copy_(both[i][n])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[i]) and torch.equal(outs[1], want[i])


def test_a_captured_step_of_the_decoder_follows_its_inputs():
    spec = importlib.util.spec_from_file_location("hosted_prefix_decoder", os.path.join(ROOT, "examples", "hosted_prefix_decoder.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    g = torch.Generator().manual_seed(4)
    for sequences, prefix, tokens in ((6, 130, 1), (40, 2500, 1), (3, 700, 9)):
        steps = [torch.randn((sequences, tokens, 256), generator=g).bfloat16().cuda() for _ in range(3)]
        decoder = module.PrefixDecoder(sequences, prefix, 16)
        decoder.prompt(torch.randn((prefix, 256), generator=g).bfloat16().cuda())
        want = []
        for x in steps:
            decoder.length = 0
            want.append(decoder(x))
            torch.cuda.synchronize()
        x = torch.zeros_like(steps[0])
        decoder.length = 0
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = decoder(x)
        for i in (0, 1, 2, 1, 0):
            x.copy_(steps[i])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want[i])
