"""What the hosted-model operators refuse, found on the host before anything is launched."""
import ctypes
import os
import struct
import subprocess
import sys

import pytest
import torch

import paper_2109_09868_b200 as ap
from paper_2109_09868_b200 import binding

HERE = os.path.dirname(os.path.abspath(__file__))

# the argument structs of the header, field by field (native alignment)
LINEAR = struct.Struct("@qqqPqPqPPqPqii")
NORM_ROPE = struct.Struct("@qiiiiiiPqqPqqPqqPPPqPPqqPqqqPqqqqPifP")
ATTENTION = struct.Struct("@qiiiiiiiifiPqqPqqqPqqqqPqqPPPqqPq")


def linear_rc(M=4, N=8, K=16, X=16, xs=16, W=16, ws=16, bias=0, R=0, rs=0, Y=16, ys=8, act=0, kind=0):
    return ap.load().approxifer_linear(LINEAR.pack(M, N, K, X, xs, W, ws, bias, R, rs, Y, ys, act, kind), None)


def test_linear_refusals():
    assert linear_rc(M=0, X=0, W=0, Y=0) == binding.OK
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(M=2 ** 31), dict(N=2 ** 31), dict(K=2 ** 31), dict(xs=15), dict(ws=8), dict(ys=7), dict(R=16, rs=7)):
        assert linear_rc(**bad) == binding.E_RANGE, bad
    for bad in (dict(X=0), dict(W=0), dict(Y=0)):
        assert linear_rc(**bad) == binding.E_NULL, bad
    for bad in (dict(act=5), dict(act=-1), dict(kind=2), dict(X=17), dict(W=1), dict(bias=3), dict(Y=18, kind=1), dict(R=18, rs=8, kind=1)):
        assert linear_rc(**bad) == binding.E_PARAM, bad
    assert ap.load().approxifer_linear(None, None) == binding.E_NULL


def norm_rope_rc(T=3, Hq=4, Hkv=2, D=8, rot=8, inter=0, kind=0, q=16, qs=(32, 8), k=16, ks=(16, 8), v=16, vs=(16, 8), qw=0, kw=0, cs=16, npos=9,
                 pos=16, qo=16, qos=(32, 8), kc=16, kcs=(128, 64, 8), vc=16, vcs=(128, 64, 8), pages=5, slots=16, page=8, eps=1e-6, status=0):
    return ap.load().approxifer_qk_norm_rope(NORM_ROPE.pack(
        T, Hq, Hkv, D, rot, inter, kind, q, *qs, k, *ks, v, *vs, qw, kw, cs, npos, pos, qo, *qos, kc, *kcs, vc, *vcs, pages, slots, page, eps, status), None)


def test_norm_rope_refusals():
    assert norm_rope_rc(T=0, q=0, qo=0, cs=0, pos=0, slots=0) == binding.OK
    for bad in (dict(T=-1), dict(Hq=0), dict(Hkv=0), dict(D=0), dict(D=257, rot=0), dict(rot=10), dict(rot=-2), dict(page=0), dict(pages=-1), dict(qs=(32, 7)),
                dict(qos=(-1, 8)), dict(ks=(16, 4)), dict(vcs=(128, 64, 7)), dict(kcs=(7, 64, 8))):
        assert norm_rope_rc(**bad) == binding.E_RANGE, bad
    for bad in (dict(rot=7), dict(kind=2), dict(eps=-1.0), dict(eps=float("nan")), dict(q=17), dict(kc=17), dict(kind=1, q=18), dict(cs=18)):
        assert norm_rope_rc(**bad) == binding.E_PARAM, bad
    for bad in (dict(q=0), dict(qo=0), dict(cs=0), dict(pos=0), dict(slots=0), dict(k=0), dict(vc=0)):
        assert norm_rope_rc(**bad) == binding.E_NULL, bad
    assert ap.load().approxifer_qk_norm_rope(None, None) == binding.E_NULL


def attention_rc(T=3, batch=1, max_q=3, Hq=4, Hkv=2, D=8, page=8, window=0, sinks=0, scale=1.0, reserved=0, q=16, qs=(32, 8), kc=16, kcs=(128, 64, 8), vc=16,
                 vcs=(128, 64, 8), pages=5, table=16, ts=4, tp=4, start=16, lens=16, out=16, os=(32, 8),
                 ws=0, wb=0):
    return ap.load().approxifer_attention(ATTENTION.pack(
        T, batch, max_q, Hq, Hkv, D, page, window, sinks, scale, reserved, q, *qs, kc, *kcs, vc, *vcs, pages, table, ts, tp, start, lens, out, *os, ws, wb), None)


def test_attention_refusals():
    assert attention_rc(T=0, batch=0, q=0, kc=0, vc=0, out=0) == binding.OK
    for bad in (dict(T=-1), dict(batch=0), dict(max_q=0), dict(Hq=0), dict(Hkv=0), dict(D=0), dict(D=257), dict(page=0), dict(window=-1), dict(sinks=-1),
                dict(pages=-1), dict(tp=-1), dict(qs=(32, 7)), dict(os=(-32, 8)), dict(kcs=(128, 64, 7)), dict(vcs=(128, 7, 8)), dict(ts=-4), dict(wb=-1)):
        assert attention_rc(**bad) == binding.E_RANGE, bad
    for bad in (dict(Hq=5), dict(scale=float("nan")), dict(scale=float("inf")), dict(reserved=1), dict(q=17), dict(vc=17), dict(ws=8, wb=64)):
        assert attention_rc(**bad) == binding.E_PARAM, bad
    for bad in (dict(q=0), dict(kc=0), dict(vc=0), dict(table=0), dict(start=0), dict(lens=0), dict(out=0)):
        assert attention_rc(**bad) == binding.E_NULL, bad
    assert ap.load().approxifer_attention(None, None) == binding.E_NULL


def test_packed_structs_are_as_long_as_the_header_says():
    # eight bytes a pointer or 64-bit integer, four the others
    assert LINEAR.size == 12 * 8 + 2 * 4
    assert NORM_ROPE.size == 29 * 8 + 8 * 4
    assert ATTENTION.size == 23 * 8 + 10 * 4
    assert ctypes.sizeof(ctypes.c_void_p) == 8


def test_binding_refuses_what_the_library_cannot_take():
    x = torch.zeros(2, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ap.approxifer_linear(x, x)
    with pytest.raises(ValueError):
        ap.approxifer_qk_norm_rope(x.view(2, 1, 8), None, None, None, None, torch.zeros(4, 8), torch.zeros(2, dtype=torch.int32), None, None, None)
    with pytest.raises(ValueError):
        ap.approxifer_attention(x.view(2, 1, 8), x.view(1, 1, 2, 8), x.view(1, 1, 2, 8), torch.zeros(1, 1, dtype=torch.int32),
                                torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 2)


def test_outputs_for_another_stream_come_from_that_streams_memory(monkeypatch):
    """A block of the current stream's memory may be in use there by work that the other stream does not wait for."""
    from paper_2109_09868_b200 import hosted

    seen = []

    class Stream:
        cuda_stream = 77

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            seen.append(("on", self.stream))

        def __exit__(self, *a):
            seen.append("off")

    class Out:
        def record_stream(self, stream):
            seen.append(("kept for", stream))

    class Native:
        def __getattr__(self, name):
            return lambda *args: (seen.append((name, args[-1])), Out())[1]

    monkeypatch.setattr(hosted, "_native", Native())
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: "user")
    s = Stream()
    calls = {"linear": lambda **k: ap.approxifer_linear(1, 2, **k), "norm_rope": lambda **k: ap.approxifer_qk_norm_rope(*range(10), **k),
             "attention": lambda **k: ap.approxifer_attention(*range(7), **k)}
    for name, call in calls.items():
        del seen[:]
        call(stream=s)
        assert seen == [("on", s), (name, 77), "off", ("kept for", "user")]
        del seen[:]
        call(stream=s, **{{"linear": "Y", "norm_rope": "q_out", "attention": "out"}[name]: "given"})
        assert seen == [(name, 77)]
        del seen[:]
        call()
        assert seen == [(name, None)]


def test_attention_refuses_more_tokens_than_the_bound_on_the_queries_allows():
    # (such a call would leave rows unwritten)
    assert attention_rc(T=7, batch=2, max_q=3) == binding.E_RANGE
    assert attention_rc(T=7, batch=2, max_q=3, q=0) == binding.E_RANGE
    assert attention_rc(T=6, batch=2, max_q=3, q=0) == binding.E_NULL
    assert attention_rc(T=6, batch=2 ** 31 - 1, max_q=2 ** 31 - 1, q=0) == binding.E_NULL


def test_extents_whose_products_overflow_are_refused():
    assert attention_rc(tp=2 ** 31) == binding.E_RANGE
    assert attention_rc(tp=2 ** 40, page=2 ** 31 - 1) == binding.E_RANGE
    assert attention_rc(tp=2 ** 31 - 1, page=2 ** 31 - 1, q=0) == binding.E_NULL
    assert norm_rope_rc(pages=2 ** 31) == binding.E_RANGE
    assert norm_rope_rc(pages=2 ** 62) == binding.E_RANGE
    assert norm_rope_rc(pages=2 ** 31 - 1, q=0) == binding.E_NULL


@pytest.mark.parametrize("page", [2 ** 30 + 1, 2 ** 31 - 1])
@pytest.mark.parametrize("max_q,T", [(1, 1), (3, 3)])
def test_the_choice_of_kernel_ends_for_the_longest_pages(page, max_q, T):
    """In a process without a device, so that nothing can be launched: the call gets as far as that."""
    code = ("import sys; sys.path[:0] = [%r, %r]\nimport test_hosted_cpu as t\n"
            "assert t.attention_rc(T=%d, max_q=%d, tp=1, page=%d) == t.binding.E_CUDA" % (os.path.dirname(HERE), HERE, T, max_q, page))
    subprocess.run([sys.executable, "-c", code], check=True, timeout=120, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""))


def test_only_the_hosted_operators_need_their_binding(monkeypatch, tmp_path):
    """Without _hosted.so, and without what it takes to build it, the library loads; the hosted operators say what is missing."""
    from paper_2109_09868_b200 import build, hosted

    def refuse(*a, **k):
        raise RuntimeError("no g++ here")

    monkeypatch.setattr(build, "BINDING", str(tmp_path / "_hosted.so"))
    monkeypatch.setattr(build, "build_binding", refuse)
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(hosted, "_native", None)
    assert ap.load().approxifer_version() == ap.version() >= 100
    x = torch.zeros(2, 8, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="no g"):
        ap.approxifer_linear(x, x)
    monkeypatch.setattr(hosted.shutil, "which", lambda name: None)
    with pytest.raises(RuntimeError, match="_hosted.so is missing"):
        ap.approxifer_linear(x, x)


def test_a_binding_that_does_not_build_keeps_nobody_from_the_library(monkeypatch, tmp_path):
    from paper_2109_09868_b200 import build

    def refuse(*a, **k):
        raise RuntimeError("no g++ here")

    built = []
    monkeypatch.setattr(build, "BINDING", str(tmp_path / "_hosted.so"))
    monkeypatch.setattr(build, "build_binding", refuse)
    monkeypatch.setattr(build, "library_is_stale", lambda: True)
    monkeypatch.setattr(build, "build_library", lambda verbose=False: built.append(1))
    with pytest.raises(RuntimeError, match="no g"):
        build.build()
    assert built == [1]
