"""Every refusal of the adapters', normed append's and log probabilities' calls, without a GPU: all of them come before the first HIP call."""
import ctypes
import math

import pytest
import torch

import paper_2506_12024_amd as fq
from paper_2506_12024_amd import binding as B

FAKE = 0x10000000  # aligned to 256, never dereferenced
FAR = 0x40000000


def create(dtype=0, slots=3, rank=16, K=64, N=40, a=FAKE, a_stride=1024, b=FAKE, b_stride=640, ranks=None, scales=None):
    h = ctypes.c_void_p()
    return fq.lib.fq_adapters_create(ctypes.byref(h), dtype, slots, rank, K, N, a, a_stride, b, b_stride, ranks, scales), h


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), B.FQ_ERR_BITS), (dict(dtype=-1), B.FQ_ERR_BITS), (dict(slots=0), B.FQ_ERR_SHAPE), (dict(slots=16385), B.FQ_ERR_SHAPE),
    (dict(rank=0), B.FQ_ERR_SHAPE), (dict(rank=12), B.FQ_ERR_SHAPE), (dict(rank=264, a_stride=1 << 20, b_stride=1 << 20), B.FQ_ERR_SHAPE),
    (dict(K=0), B.FQ_ERR_SHAPE), (dict(K=60), B.FQ_ERR_SHAPE), (dict(K=(1 << 24) + 8), B.FQ_ERR_SHAPE), (dict(N=0), B.FQ_ERR_SHAPE),
    (dict(N=(1 << 24) + 1), B.FQ_ERR_SHAPE), (dict(a=None), B.FQ_ERR_NULL), (dict(b=None), B.FQ_ERR_NULL), (dict(a_stride=1016), B.FQ_ERR_SHAPE),
    (dict(b_stride=632), B.FQ_ERR_SHAPE), (dict(a_stride=1 << 46), B.FQ_ERR_SHAPE), (dict(a=FAKE + 8), B.FQ_ERR_ALIGN), (dict(b=FAKE + 2), B.FQ_ERR_ALIGN),
    (dict(a_stride=1028), B.FQ_ERR_ALIGN), (dict(b_stride=644), B.FQ_ERR_ALIGN), (dict(ranks=FAKE + 2), B.FQ_ERR_ALIGN), (dict(scales=FAKE + 1), B.FQ_ERR_ALIGN)])
def test_adapters_refuse(bad, code):
    rc, h = create(**bad)
    assert rc == code and not h.value and fq.fq_last_error()


def test_one_slot_needs_no_stride():
    rc, h = create(slots=1, a_stride=0, b_stride=0)
    assert rc == B.FQ_OK and fq.lib.fq_adapters_destroy(h) == B.FQ_OK


def test_adapters_handles():
    assert fq.lib.fq_adapters_create(None, 0, 1, 8, 8, 8, FAKE, 0, FAKE, 0, None, None) == B.FQ_ERR_NULL
    assert fq.lib.fq_adapters_destroy(None) == B.FQ_ERR_NULL
    junk = ctypes.create_string_buffer(256)
    assert fq.lib.fq_adapters_destroy(ctypes.addressof(junk)) == B.FQ_ERR_NULL
    assert fq.lib.fq_adapters_workspace_bytes(ctypes.addressof(junk), 1) == 0
    assert fq.lib.fq_adapters_add(None, 1, FAKE, 64, FAKE, FAKE, 40, FAR, 40, FAKE, 1 << 30, None) == B.FQ_ERR_NULL


def test_workspace_of_a_larger_call_serves_a_smaller_one():
    for shape in (dict(), dict(rank=256, K=16384, N=28672, a_stride=1 << 30, b_stride=1 << 30), dict(slots=1, rank=8, K=8, N=1)):
        _, h = create(**shape)
        last = 0
        for M in list(range(0, 700)) + [1000, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 5000, 8191, 8192, 20000, 1 << 20]:
            n = fq.lib.fq_adapters_workspace_bytes(h, M)
            assert n >= max(last, 1), (shape, M)
            last = n
        assert fq.lib.fq_adapters_workspace_bytes(h, -1) == 0 and fq.lib.fq_adapters_workspace_bytes(h, (1 << 20) + 1) == 0
        fq.lib.fq_adapters_destroy(h)


@pytest.mark.parametrize("bad,code", [
    (dict(M=-1), B.FQ_ERR_SHAPE), (dict(M=(1 << 20) + 1), B.FQ_ERR_SHAPE), (dict(x=None), B.FQ_ERR_NULL), (dict(adapter=None), B.FQ_ERR_NULL),
    (dict(y=None), B.FQ_ERR_NULL), (dict(out=None), B.FQ_ERR_NULL), (dict(ws=None), B.FQ_ERR_NULL), (dict(xs=56), B.FQ_ERR_SHAPE),
    (dict(ys=39), B.FQ_ERR_SHAPE), (dict(outs=39), B.FQ_ERR_SHAPE), (dict(xs=(1 << 40) + 8), B.FQ_ERR_SHAPE), (dict(x=FAKE + 8), B.FQ_ERR_ALIGN),
    (dict(xs=68), B.FQ_ERR_ALIGN), (dict(y=FAR + 1), B.FQ_ERR_ALIGN), (dict(out=FAR + 0x1000001), B.FQ_ERR_ALIGN), (dict(adapter=FAKE + 2), B.FQ_ERR_ALIGN),
    (dict(ws=FAKE + 16), B.FQ_ERR_ALIGN), (dict(ws_bytes=255), B.FQ_ERR_SHAPE), (dict(out=FAR + 2), B.FQ_ERR_SHAPE), (dict(out=FAR, outs=41), B.FQ_ERR_SHAPE),
    (dict(out=FAKE, outs=64), B.FQ_ERR_SHAPE), (dict(out=FAKE + 126, outs=64), B.FQ_ERR_SHAPE)])
def test_adding_refuses(bad, code):
    _, h = create()
    a = dict(M=10, x=FAKE, xs=64, adapter=FAKE, y=FAR, ys=40, out=FAR + 0x1000000, outs=40, ws=FAKE, ws_bytes=1 << 30)
    a.update(bad)
    assert fq.lib.fq_adapters_add(h, a["M"], a["x"], a["xs"], a["adapter"], a["y"], a["ys"], a["out"], a["outs"], a["ws"], a["ws_bytes"], None) == code
    assert fq.lib.fq_adapters_add(h, 0, None, 0, None, None, 0, None, 0, None, 0, None) == B.FQ_OK
    fq.lib.fq_adapters_destroy(h)


@pytest.mark.parametrize("bad,code", [
    (dict(kw=None), B.FQ_ERR_NULL), (dict(qw=None), B.FQ_ERR_NULL), (dict(ws=8), B.FQ_ERR_SHAPE), (dict(ws=-64), B.FQ_ERR_SHAPE), (dict(ws=68), B.FQ_ERR_ALIGN),
    (dict(qw=FAKE + 8), B.FQ_ERR_ALIGN), (dict(kw=FAKE + 2), B.FQ_ERR_ALIGN), (dict(eps=-1e-6), B.FQ_ERR_SHAPE), (dict(eps=math.nan), B.FQ_ERR_SHAPE),
    (dict(eps=math.inf), B.FQ_ERR_SHAPE), (dict(offset=math.inf), B.FQ_ERR_SHAPE), (dict(offset=math.nan), B.FQ_ERR_SHAPE),
    # and what fq_kv_append refuses
    (dict(tokens=-1), B.FQ_ERR_SHAPE), (dict(q=None), B.FQ_ERR_NULL), (dict(k=None), B.FQ_ERR_NULL), (dict(heads=3), B.FQ_ERR_SHAPE), (dict(rot=63), B.FQ_ERR_SHAPE),
    (dict(rot=66), B.FQ_ERR_SHAPE), (dict(freqs=None), B.FQ_ERR_NULL), (dict(amplitude=math.nan), B.FQ_ERR_SHAPE), (dict(q_out=FAKE), B.FQ_ERR_SHAPE),
    (dict(v=FAKE + 4), B.FQ_ERR_ALIGN)])
def test_normed_append_refuses(bad, code):
    kv, seqs = ctypes.c_void_p(), ctypes.c_void_p()
    assert fq.lib.fq_kv_create(ctypes.byref(kv), 0, 2, 64, 16, 5, FAKE, FAKE, 2048, 1024, 64) == B.FQ_OK
    assert fq.lib.fq_seqs_create(ctypes.byref(seqs), 2, FAKE, FAKE, FAKE, 4, None, 0) == B.FQ_OK
    a = dict(tokens=5, q=FAKE, heads=4, q_out=FAR, k=FAKE, v=FAKE, qw=FAKE, kw=FAKE, ws=0, eps=1e-6, offset=0.0, freqs=FAKE, rot=64, amplitude=1.0)
    a.update(bad)

    def go(**more):
        c = dict(a, **more)
        return fq.lib.fq_kv_append_normed(kv, seqs, c["tokens"], c["q"], 256, c["heads"], c["q_out"], 256, c["k"], 128, c["v"], 128, c["qw"], c["kw"],
                                          c["ws"], c["eps"], c["offset"], c["freqs"], c["rot"], 0, c["amplitude"], None, None)
    assert go() == code and b"fq_kv_append_normed" in fq.lib.fq_last_error()
    if "tokens" not in bad and "rot" not in bad:
        assert go(tokens=0) == B.FQ_OK
    fq.lib.fq_kv_destroy(kv), fq.lib.fq_seqs_destroy(seqs)


@pytest.mark.parametrize("name", ["fq_logprobs", "fq_logprobs_f16"])
@pytest.mark.parametrize("bad,code", [
    (dict(R=-1), B.FQ_ERR_SHAPE), (dict(V=0), B.FQ_ERR_SHAPE), (dict(V=(1 << 24) + 1, stride=1 << 25), B.FQ_ERR_SHAPE), (dict(stride=99), B.FQ_ERR_SHAPE),
    (dict(stride=(1 << 40) + 1), B.FQ_ERR_SHAPE), (dict(n=-1), B.FQ_ERR_SHAPE), (dict(n=65537), B.FQ_ERR_SHAPE), (dict(top=-1), B.FQ_ERR_SHAPE), (dict(top=65), B.FQ_ERR_SHAPE),
    (dict(x=None), B.FQ_ERR_NULL), (dict(given=None), B.FQ_ERR_NULL), (dict(lp=None), B.FQ_ERR_NULL), (dict(tok=None), B.FQ_ERR_NULL), (dict(tlp=None), B.FQ_ERR_NULL),
    (dict(ws=None), B.FQ_ERR_NULL), (dict(x=FAKE + 1), B.FQ_ERR_ALIGN), (dict(given=FAKE + 2), B.FQ_ERR_ALIGN), (dict(lp=FAKE + 2), B.FQ_ERR_ALIGN),
    (dict(tok=FAKE + 1), B.FQ_ERR_ALIGN), (dict(tlp=FAKE + 3), B.FQ_ERR_ALIGN), (dict(h=FAKE + 2), B.FQ_ERR_ALIGN), (dict(ws=FAKE + 128), B.FQ_ERR_ALIGN),
    (dict(ws_bytes=0), B.FQ_ERR_SHAPE)])
def test_logprobs_refuse(name, bad, code):
    a = dict(x=FAKE, R=4, V=100, stride=100, given=FAKE, n=2, lp=FAKE, top=5, tok=FAKE, tlp=FAKE, h=FAKE, ws=FAKE, ws_bytes=1 << 30)
    a.update(bad)
    go = lambda **c: getattr(fq.lib, name)(c["x"], c["R"], c["V"], c["stride"], c["given"], c["n"], c["lp"], c["top"], c["tok"], c["tlp"], c["h"],  # noqa: E731
                                           c["ws"], c["ws_bytes"], None)
    assert go(**a) == code and name.encode() in fq.lib.fq_last_error()
    assert go(**dict(a, R=0, V=100, stride=100, n=0, top=0, x=None)) == B.FQ_OK


def test_logprobs_workspaces():
    assert fq.fq_logprobs_workspace_bytes(0, 1) > 0
    for R, V in ((1, 1), (1, 1 << 24), (1 << 20, 128256), (2 ** 31 - 1, 32000)):
        assert 0 < fq.fq_logprobs_workspace_bytes(R, V) < 1 << 31
    for R, V in ((-1, 5), (1, 0), (1, (1 << 24) + 1)):
        with pytest.raises(fq.FlexqError):
            fq.fq_logprobs_workspace_bytes(R, V)


def test_the_binding_refuses_wrong_tensors():
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    with pytest.raises(ValueError):
        fq.Adapters(half(2, 8, 16), half(2, 10, 16))
    with pytest.raises(ValueError):
        fq.Adapters(half(2, 8, 16), half(2, 10, 8).bfloat16())
    with pytest.raises(ValueError):
        fq.Adapters(half(2, 16, 8).transpose(1, 2), half(2, 10, 8))
    with pytest.raises(ValueError):
        fq.Adapters(half(2, 8, 16), half(2, 10, 8), ranks=torch.zeros(1, dtype=torch.int32))
    h = fq.Adapters(half(2, 8, 16), half(2, 10, 8))
    ws = torch.zeros(fq.fq_adapters_workspace_bytes(h, 4), dtype=torch.uint8)
    who = torch.zeros(4, dtype=torch.int32)
    for x, y, out in ((half(4, 8), half(4, 10), half(4, 10)), (half(4, 16), half(4, 9), half(4, 10)), (half(4, 16), half(4, 10), half(3, 10)),
                      (half(4, 16).float(), half(4, 10), half(4, 10)), (half(16, 4).t(), half(4, 10), half(4, 10)),
                      (half(4, 16), half(4, 10), half(4, 10))):  # the last: not on the device
        with pytest.raises(ValueError):
            fq.fq_adapters_add(h, x, who, y, out, ws)
    logits = torch.zeros((2, 50))
    ws = torch.zeros(fq.fq_logprobs_workspace_bytes(2, 50), dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    for kw in (dict(given=i32(2, 1)), dict(given=i32(2, 1).long(), given_logprob=torch.zeros(2, 1)), dict(given=i32(3, 1), given_logprob=torch.zeros(3, 1)),
               dict(top_token=i32(2, 3), top_logprob=torch.zeros(2, 4)), dict()):  # the last: not on the device
        with pytest.raises(ValueError):
            fq.fq_logprobs(logits, 2, 50, ws, **kw)
    with pytest.raises(ValueError):
        fq.fq_logprobs_f16(logits, 2, 50, ws)
    cache = fq.KVCache(half(3, 2, 4, 64), half(3, 2, 4, 64))
    seqs = fq.Sequences(i32(2), i32(1), i32(1, 2))
    q, k, w = half(1, 4, 64), half(1, 2, 64), half(64)
    for qw, kw in ((w, half(2, 64)), (half(2, 64), half(2, 64)), (w, half(32)), (w.float(), w), (w, w)):  # the last: not on the device
        with pytest.raises(ValueError):
            fq.fq_kv_append_normed(cache, seqs, q, k, k, torch.empty_like(q), None, qw, kw)
