"""What block_norm, the 4-bit arrays and product and the attention behind a prefix refuse, found on the host before anything is
launched; how their Python calls deal with streams; their plain forms against differences and by hand."""
import struct

import pytest
import torch

import hosted_more_reference as ref
import paper_2109_09868_b200 as ap
from paper_2109_09868_b200 import binding

# the argument structs of the header, field by field (native alignment)
BLOCK_NORM = struct.Struct("@qiiiiiifffiPqPqPqqPPPPPqPq")
MX_ARRAY = struct.Struct("@qqiiPqPqP")
MX_LINEAR = struct.Struct("@qqqPqPPqPPPqPqiiPq")
ATTENTION = struct.Struct("@qiiiiiiiifiPqqPqqqPqqqqPqqPPPqqPq")
PREFIX = struct.Struct(ATTENTION.format + "Pqq")


def test_packed_structs_are_as_long_as_the_header_says():
    assert BLOCK_NORM.size == 16 * 8 + 10 * 4
    assert MX_ARRAY.size == 7 * 8 + 2 * 4
    assert MX_LINEAR.size == 16 * 8 + 2 * 4
    assert PREFIX.size == ATTENTION.size + 3 * 8


def norm_rc(T=3, N=16, stream=0, kind=0, after=1, before=1, act=0, a=1.0, b=1.0, eps=1e-6, reserved=0, R=16, rs=16, Y=16, ys=16, gate=0, gs=(0, 1), aw=0, ab=0, bw=0,
            bb=0, Ro=16, ros=16, X=16, xs=16):
    return ap.load().approxifer_block_norm(BLOCK_NORM.pack(T, N, stream, kind, after, before, act, a, b, eps, reserved, R, rs, Y, ys, gate, *gs, aw, ab, bw, bb, Ro, ros, X, xs), None)


def test_block_norm_refusals():
    assert norm_rc(T=0, R=0, Y=16, Ro=0, X=0) == binding.OK
    for bad in (dict(T=-1), dict(T=2 ** 31), dict(N=0), dict(N=16385, ros=16385, xs=16385), dict(rs=-1), dict(ys=-1), dict(ros=15), dict(xs=15), dict(gate=16, gs=(-1, 1)),
                dict(gate=16, gs=(0, 2)), dict(gate=16, gs=(0, -1))):
        assert norm_rc(**bad) == binding.E_RANGE, bad
    for bad in (dict(stream=2), dict(kind=-1), dict(after=3), dict(before=-1), dict(act=3), dict(eps=-1.0), dict(eps=float("nan")), dict(a=float("inf")), dict(b=float("nan")),
                dict(reserved=1), dict(Y=0), dict(Y=0, after=0, before=0), dict(Y=0, after=0, gate=16), dict(Y=0, after=0, a=0.5), dict(R=17), dict(stream=1, R=18),
                dict(kind=1, Y=18), dict(kind=1, X=18), dict(gate=17), dict(aw=17), dict(ab=17), dict(bw=17), dict(bb=17), dict(Ro=17)):
        assert norm_rc(**bad) == binding.E_PARAM, bad
    for bad in (dict(R=0), dict(Ro=0), dict(X=0), dict(Y=0, after=0, X=0)):
        assert norm_rc(**bad) == binding.E_NULL, bad
    assert ap.load().approxifer_block_norm(None, None) == binding.E_NULL


def array_rc(name, M=3, K=64, kind=0, reserved=0, X=16, xs=64, codes=16, cs=32, scales=16):
    return getattr(ap.load(), name)(MX_ARRAY.pack(M, K, kind, reserved, X, xs, codes, cs, scales), None)


@pytest.mark.parametrize("name", ["approxifer_mx_quantize", "approxifer_mx_dequantize"])
def test_mx_array_refusals(name):
    assert array_rc(name, M=0, X=0, codes=0, scales=0) == binding.OK
    for bad in (dict(M=-1), dict(M=2 ** 31), dict(K=0), dict(K=2 ** 31), dict(xs=63), dict(cs=16)):
        assert array_rc(name, **bad) == binding.E_RANGE, bad
    for bad in (dict(K=40), dict(cs=40), dict(kind=2), dict(reserved=1), dict(X=17), dict(kind=1, X=18), dict(codes=24), dict(scales=20)):
        assert array_rc(name, **bad) == binding.E_PARAM, bad
    for bad in (dict(X=0), dict(codes=0), dict(scales=0)):
        assert array_rc(name, **bad) == binding.E_NULL, bad
    assert getattr(ap.load(), name)(None, None) == binding.E_NULL


def mx(M=4, N=8, K=64, X=16, xs=32, xsc=16, W=16, ws=32, wsc=16, bias=0, R=0, rs=0, Y=16, ys=8, act=0, kind=0, room=0, bytes=0):
    return MX_LINEAR.pack(M, N, K, X, xs, xsc, W, ws, wsc, bias, R, rs, Y, ys, act, kind, room, bytes)


def test_mx_linear_refusals():
    call, size = ap.load().approxifer_mx_linear, ap.load().approxifer_mx_linear_workspace
    assert call(mx(M=0, X=0, W=0, Y=0, wsc=0), None) == binding.OK
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(M=2 ** 31), dict(N=2 ** 31), dict(K=2 ** 31), dict(xs=31), dict(xsc=0, xs=63), dict(ws=16), dict(ys=7), dict(R=16, rs=7),
                dict(bytes=-1)):
        assert call(mx(**bad), None) == binding.E_RANGE, bad
        assert size(mx(**bad)) == binding.E_RANGE, bad
    for bad in (dict(K=48), dict(xs=40), dict(ws=40), dict(act=5), dict(act=-1), dict(kind=2)):
        assert call(mx(**bad), None) == binding.E_PARAM, bad
        assert size(mx(**bad)) == binding.E_PARAM, bad
    for bad in (dict(X=24), dict(X=17, xsc=0, xs=64, room=16, bytes=2 ** 40), dict(xsc=24), dict(W=24), dict(wsc=24), dict(bias=17), dict(Y=17), dict(kind=1, Y=18),
                dict(kind=1, R=18, rs=8), dict(room=8, bytes=64)):
        assert call(mx(**bad), None) == binding.E_PARAM, bad
    for bad in (dict(X=0), dict(W=0), dict(wsc=0), dict(Y=0)):
        assert call(mx(**bad), None) == binding.E_NULL, bad
    assert call(None, None) == binding.E_NULL and size(None) == binding.E_NULL
    # codes need no workspace; many rows of bfloat16 room for their codes and scales, and with less the call is refused
    assert size(mx(M=1000)) == 0
    big = dict(M=1000, xsc=0, xs=64)
    need = size(mx(**big))
    assert need >= 1000 * 32 + 8 * 512
    assert call(mx(**big), None) == binding.E_NULL
    assert call(mx(**big, room=16, bytes=need - 1), None) == binding.E_RANGE


def prefix(T=3, batch=1, max_q=3, Hq=4, Hkv=2, D=8, page=8, window=0, sinks=0, scale=1.0, reserved=0, q=16, qs=(32, 8), kc=16, kcs=(128, 64, 8), vc=16, vcs=(128, 64, 8),
           pages=5, table=16, ts=4, tp=4, start=16, lens=16, out=16, os=(32, 8), ws=0, wb=0, first=16, fp=3, n=20):
    return PREFIX.pack(T, batch, max_q, Hq, Hkv, D, page, window, sinks, scale, reserved, q, *qs, kc, *kcs, vc, *vcs, pages, table, ts, tp, start, lens, out, *os, ws, wb,
                       first, fp, n)


def test_prefix_attention_refusals():
    call, size = ap.load().approxifer_prefix_attention, ap.load().approxifer_prefix_attention_workspace
    assert call(prefix(T=0, batch=0, q=0, kc=0, vc=0, out=0, first=0), None) == binding.OK
    for bad in (dict(T=-1), dict(batch=0), dict(max_q=0), dict(Hq=0), dict(Hkv=0), dict(D=0), dict(D=257), dict(page=0), dict(window=-1), dict(sinks=-1), dict(pages=-1),
                dict(tp=-1), dict(qs=(32, 7)), dict(os=(-32, 8)), dict(kcs=(128, 64, 7)), dict(vcs=(128, 7, 8)), dict(ts=-4), dict(wb=-1), dict(n=-1), dict(n=2 ** 31),
                dict(fp=-1), dict(fp=2 ** 31), dict(T=7, batch=2)):
        assert call(prefix(**bad), None) == binding.E_RANGE, bad
        assert size(prefix(**bad)) == binding.E_RANGE, bad
    for bad in (dict(Hq=5), dict(scale=float("nan")), dict(scale=float("inf")), dict(reserved=1), dict(window=4), dict(sinks=1)):
        assert call(prefix(**bad), None) == binding.E_PARAM, bad
        assert size(prefix(**bad)) == binding.E_PARAM, bad
    room = dict(ws=16, wb=2 ** 40)
    for bad in (dict(q=17), dict(vc=17), dict(kc=17), dict(out=17), dict(ws=8)):
        assert call(prefix(**dict(room, **bad)), None) == binding.E_PARAM, bad
    for bad in (dict(q=0), dict(kc=0), dict(vc=0), dict(table=0), dict(start=0), dict(lens=0), dict(out=0), dict(first=0)):
        assert call(prefix(**dict(room, **bad)), None) == binding.E_NULL, bad
    assert call(None, None) == binding.E_NULL and size(None) == binding.E_NULL


def test_binding_refuses_what_the_library_cannot_take():
    x = torch.zeros(2, 32, dtype=torch.bfloat16)
    codes, scales = torch.zeros(2, 16, dtype=torch.uint8), torch.zeros(1, 1, 512, dtype=torch.uint8)
    zero = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: ap.approxifer_block_norm(x), lambda: ap.approxifer_mx_quantize(x), lambda: ap.approxifer_mx_dequantize(codes, scales),
                 lambda: ap.approxifer_mx_linear(x, codes, scales),
                 lambda: ap.approxifer_prefix_attention(x.view(2, 1, 32), x.view(1, 1, 2, 32), x.view(1, 1, 2, 32), zero, 2, zero[None], zero, zero[:1], 2)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()


def test_outputs_and_workspaces_for_another_stream_come_from_that_streams_memory(monkeypatch):
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
        def __init__(self, name):
            self.name = name

        def record_stream(self, stream):
            seen.append((self.name, "kept for", stream))

    many = {"block_norm": 2, "mx_quantize": 2}

    class Native:
        def __getattr__(self, name):
            outs = tuple(Out(i) for i in range(many.get(name, 1)))
            return lambda *args: (seen.append((name, args[-1])), outs if len(outs) > 1 else outs[0])[1]

    monkeypatch.setattr(hosted, "_native", Native())
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: "user")
    s = Stream()
    calls = {"block_norm": (lambda **k: ap.approxifer_block_norm(1, 2, **k), ("residual_out", "next_out")),
             "mx_quantize": (lambda **k: ap.approxifer_mx_quantize(1, **k), ("codes", "scales")), "mx_dequantize": (lambda **k: ap.approxifer_mx_dequantize(1, 2, **k), ("X",)),
             "mx_linear": (lambda **k: ap.approxifer_mx_linear(1, 2, 3, **k), ("Y",)), "prefix_attention": (lambda **k: ap.approxifer_prefix_attention(*range(9), **k), ("out",))}
    for name, (call, outs) in calls.items():
        del seen[:]
        call(stream=s)
        assert seen == [("on", s), (name, 77), "off"] + [(i, "kept for", "user") for i in range(len(outs))]
        del seen[:]
        call(stream=s, **{outs[0]: "given"})  # (a workspace, or another output, may still be allocated)
        assert seen == [("on", s), (name, 77), "off"] + [(i, "kept for", "user") for i in range(1, len(outs))]
        del seen[:]
        call()
        assert seen == [(name, None)]


def test_the_plain_4_bit_form_by_hand():
    x = torch.zeros(1, 64)
    x[0, :8] = torch.tensor([4.0, 5.0, 5.5, 7.0, 0.25, 0.75, -1.25, -0.2])   # largest 7: scale 1
    x[0, 32:36] = torch.tensor([0.5, -0.125, 0.03, 0.9])                        # largest 0.9: scale 2^-3
    codes, scales = ref.mx_quantize(x)
    assert scales[0, 0, :4].tolist() == [127, 124, 0, 0]
    values = ref.mx_values(codes, scales)
    assert values[0, :8].tolist() == [4, 4, 6, 6, 0, 1, -1, 0]
    assert values[0, 32:36].tolist() == [0.5, -0.125, 0.0, 0.75]
    assert codes[0, :4].tolist() == [0x66, 0x77, 0x20, 0x8a]
