"""Rotary frequencies against closed forms, and every refusal of the cache, attention and sampling calls, without a GPU:
all of them come before the first HIP call."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq
from paper_2506_12024_amd import binding as B
from serve_util import draw

FAKE = 0x1000  # aligned to 256, never dereferenced


@pytest.mark.parametrize("rot", [2, 20, 64, 128, 256])
def test_plain_and_linear_frequencies(rot):
    want = np.array([10000.0 ** (-2 * i / rot) for i in range(rot // 2)])
    assert np.allclose(fq.fq_rope_freqs(rot, 10000.0), want, rtol=4e-16, atol=0)
    assert np.allclose(fq.fq_rope_freqs(rot, 10000.0, fq.FQ_ROPE_LINEAR, factor=4.0), want / 4, rtol=4e-16, atol=0)


def test_scaled_base_keeps_the_first_and_divides_the_last():
    f = fq.fq_rope_freqs(128, 10000.0, fq.FQ_ROPE_BASE, factor=8.0)
    plain = fq.fq_rope_freqs(128, 10000.0)
    assert f[0] == 1.0 and math.isclose(f[-1], plain[-1] / 8, rel_tol=1e-13)


def test_wavelength_bands():
    plain = np.array(fq.fq_rope_freqs(128, 500000.0))
    f = np.array(fq.fq_rope_freqs(128, 500000.0, fq.FQ_ROPE_WAVELENGTH, factor=8.0, low=1.0, high=4.0, original=8192))
    turns = 8192 * plain / (2 * math.pi)
    assert np.array_equal(f[turns >= 4], plain[turns >= 4])
    assert np.allclose(f[turns <= 1], plain[turns <= 1] / 8, rtol=4e-16, atol=0)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.all(f[mid] < plain[mid]) and np.all(f[mid] > plain[mid] / 8)
    a = (turns[mid] - 1) / 3
    assert np.allclose(f[mid], (1 - a) * plain[mid] / 8 + a * plain[mid], rtol=1e-14, atol=0)


def test_ramp_between_pairs():
    plain = np.array(fq.fq_rope_freqs(128, 10000.0))
    f = np.array(fq.fq_rope_freqs(128, 10000.0, fq.FQ_ROPE_RAMP, factor=16.0, low=1.0, high=32.0, original=4096))

    def pair(turns):
        return 128 * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))
    first, last = math.floor(pair(32.0)), math.ceil(pair(1.0))
    assert 0 < first < last < 64
    assert np.array_equal(f[:first + 1], plain[:first + 1])
    assert np.allclose(f[last:], plain[last:] / 16, rtol=4e-16, atol=0)
    i = np.arange(first, last)
    a = 1 - (i - first) / (last - first)
    assert np.allclose(f[i], plain[i] * (a + (1 - a) / 16), rtol=1e-14, atol=0)


@pytest.mark.parametrize("args", [(3, 1e4), (0, 1e4), (258, 1e4), (64, 1.0), (64, math.inf), (64, math.nan),
                                  (64, 1e4, 9), (64, 1e4, 1, 0.5), (64, 1e4, 1, math.nan), (2, 1e4, 2, 2.0),
                                  (64, 1e4, 3, 8.0, 4.0, 1.0, 8192), (64, 1e4, 3, 8.0, 0.0, 1.0, 8192),
                                  (64, 1e4, 4, 8.0, 1.0, 4.0, 0.0)])
def test_frequencies_refuse(args):
    with pytest.raises(fq.FlexqError) as e:
        fq.fq_rope_freqs(*args)
    assert e.value.code == B.FQ_ERR_SHAPE


def kv(dtype=0, heads=2, dim=64, page=16, pages=5, k=FAKE, v=FAKE, ps=2048, hs=1024, ts=64):
    h = ctypes.c_void_p()
    return fq.lib.fq_kv_create(ctypes.byref(h), dtype, heads, dim, page, pages, k, v, ps, hs, ts), h


def seqs(n=2, q_start=FAKE, kv_len=FAKE, table=FAKE, width=4, prefix_table=None, prefix=0):
    h = ctypes.c_void_p()
    return fq.lib.fq_seqs_create(ctypes.byref(h), n, q_start, kv_len, table, width, prefix_table, prefix), h


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), B.FQ_ERR_BITS), (dict(heads=0), B.FQ_ERR_SHAPE), (dict(dim=0), B.FQ_ERR_SHAPE),
    (dict(dim=60), B.FQ_ERR_SHAPE), (dict(dim=264), B.FQ_ERR_SHAPE), (dict(page=12), B.FQ_ERR_SHAPE),
    (dict(page=0), B.FQ_ERR_SHAPE), (dict(page=131072), B.FQ_ERR_SHAPE), (dict(pages=0), B.FQ_ERR_SHAPE),
    (dict(k=None), B.FQ_ERR_NULL), (dict(v=None), B.FQ_ERR_NULL), (dict(k=FAKE + 8), B.FQ_ERR_ALIGN),
    (dict(ps=-8), B.FQ_ERR_SHAPE), (dict(hs=32), B.FQ_ERR_SHAPE), (dict(ts=68), B.FQ_ERR_ALIGN),
    (dict(ps=1 << 45), B.FQ_ERR_SHAPE)])
def test_cache_refuses(bad, code):
    rc, h = kv(**bad)
    assert rc == code and not h.value and fq.fq_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(n=0), B.FQ_ERR_SHAPE), (dict(n=65536), B.FQ_ERR_SHAPE), (dict(width=0), B.FQ_ERR_SHAPE),
    (dict(prefix=-1), B.FQ_ERR_SHAPE), (dict(prefix=5), B.FQ_ERR_NULL), (dict(q_start=None), B.FQ_ERR_NULL),
    (dict(kv_len=None), B.FQ_ERR_NULL), (dict(table=None), B.FQ_ERR_NULL), (dict(table=FAKE + 2), B.FQ_ERR_ALIGN)])
def test_sequences_refuse(bad, code):
    rc, h = seqs(**bad)
    assert rc == code and not h.value and fq.fq_last_error()


def test_handles_are_checked():
    L = fq.lib
    assert L.fq_kv_create(None, 0, 2, 64, 16, 5, FAKE, FAKE, 2048, 1024, 64) == B.FQ_ERR_NULL
    assert L.fq_seqs_create(None, 2, FAKE, FAKE, FAKE, 4, None, 0) == B.FQ_ERR_NULL
    assert L.fq_kv_destroy(None) == B.FQ_ERR_NULL and L.fq_seqs_destroy(None) == B.FQ_ERR_NULL
    rc, c = kv()
    rc2, s = seqs()
    assert rc == rc2 == B.FQ_OK
    # a cache's handle is no batch's
    assert append(s, c) == B.FQ_ERR_NULL and append(None, s) == B.FQ_ERR_NULL and append(c, None) == B.FQ_ERR_NULL
    assert L.fq_kv_destroy(s) == B.FQ_ERR_NULL and L.fq_seqs_destroy(c) == B.FQ_ERR_NULL
    assert L.fq_kv_destroy(c) == B.FQ_OK and L.fq_seqs_destroy(s) == B.FQ_OK


def append(c, s, T=3, q=FAKE, qs=256, heads=4, o=0x2000, os=256, k=FAKE, ks=128, v=FAKE, vs=128, freqs=FAKE, rot=64,
           amplitude=1.0, positions=None):
    return fq.lib.fq_kv_append(c, s, T, q, qs, heads, o, os, k, ks, v, vs, freqs, rot, 0, amplitude, positions, None)


@pytest.mark.parametrize("bad,code", [
    (dict(T=-1), B.FQ_ERR_SHAPE), (dict(rot=63), B.FQ_ERR_SHAPE), (dict(rot=66), B.FQ_ERR_SHAPE), (dict(rot=-2), B.FQ_ERR_SHAPE),
    (dict(heads=3, qs=192, os=192), B.FQ_ERR_SHAPE), (dict(heads=-2), B.FQ_ERR_SHAPE), (dict(heads=4098), B.FQ_ERR_SHAPE),
    (dict(q=None), B.FQ_ERR_NULL), (dict(o=None), B.FQ_ERR_NULL), (dict(k=None), B.FQ_ERR_NULL), (dict(v=None), B.FQ_ERR_NULL),
    (dict(freqs=None), B.FQ_ERR_NULL), (dict(qs=248), B.FQ_ERR_SHAPE), (dict(ks=120), B.FQ_ERR_SHAPE),
    (dict(vs=132), B.FQ_ERR_ALIGN), (dict(q=FAKE + 8), B.FQ_ERR_ALIGN), (dict(o=FAKE), B.FQ_ERR_SHAPE),
    (dict(freqs=FAKE + 4), B.FQ_ERR_ALIGN), (dict(positions=FAKE + 2), B.FQ_ERR_ALIGN), (dict(amplitude=math.inf), B.FQ_ERR_SHAPE)])
def test_append_refuses(bad, code):
    (_, c), (_, s) = kv(), seqs()
    try:
        assert append(c, s, **bad) == code and fq.fq_last_error()
        assert append(c, s, T=0, q=None, k=None, v=None, o=None) == B.FQ_OK  # nothing to do, nothing is launched
    finally:
        fq.lib.fq_kv_destroy(c), fq.lib.fq_seqs_destroy(s)


def test_places_past_32_bits_are_refused():
    (_, c), (_, s) = kv(page=65536), seqs(width=32767)
    (_, s2) = seqs(width=32766, prefix_table=FAKE, prefix=65536)
    try:
        assert append(c, s) == B.FQ_ERR_SHAPE and append(c, s2) == B.FQ_ERR_SHAPE
    finally:
        fq.lib.fq_kv_destroy(c), fq.lib.fq_seqs_destroy(s), fq.lib.fq_seqs_destroy(s2)


def attend(c, s, T=3, q=FAKE, qs=256, heads=4, scale=0.1, o=0x2000, os=256, lse=None, max_q=2, max_kv=50, ws=0x10000, n=1 << 30):
    return fq.lib.fq_attend(c, s, T, q, qs, heads, scale, o, os, lse, max_q, max_kv, ws, n, None)


@pytest.mark.parametrize("bad,code", [
    (dict(T=-1), B.FQ_ERR_SHAPE), (dict(heads=3), B.FQ_ERR_SHAPE), (dict(heads=0), B.FQ_ERR_SHAPE), (dict(heads=4098), B.FQ_ERR_SHAPE),
    (dict(q=None), B.FQ_ERR_NULL), (dict(o=None), B.FQ_ERR_NULL), (dict(ws=None), B.FQ_ERR_NULL), (dict(qs=248), B.FQ_ERR_SHAPE),
    (dict(os=260), B.FQ_ERR_ALIGN), (dict(o=0x2008), B.FQ_ERR_ALIGN), (dict(lse=0x2002), B.FQ_ERR_ALIGN),
    (dict(ws=0x10080), B.FQ_ERR_ALIGN), (dict(n=8), B.FQ_ERR_SHAPE), (dict(max_q=0), B.FQ_ERR_SHAPE),
    (dict(max_q=4), B.FQ_ERR_SHAPE), (dict(max_kv=0), B.FQ_ERR_SHAPE), (dict(scale=math.nan), B.FQ_ERR_SHAPE),
    (dict(scale=math.inf), B.FQ_ERR_SHAPE), (dict(T=1 << 30, max_q=1), B.FQ_ERR_SHAPE)])
def test_attend_refuses(bad, code):
    (_, c), (_, s) = kv(), seqs()
    try:
        assert attend(c, s, **bad) == code and fq.fq_last_error()
        assert attend(c, s, T=0, q=None, o=None, ws=None) == B.FQ_OK
        assert fq.lib.fq_attend_workspace_bytes(c, s, 3, 3, 1, 9) == 0 and fq.fq_last_error()
        assert fq.lib.fq_attend_workspace_bytes(None, s, 3, 4, 1, 9) == 0
    finally:
        fq.lib.fq_kv_destroy(c), fq.lib.fq_seqs_destroy(s)


@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("heads,tokens,max_q,n,prefix", [(2, 1, 1, 1, 0), (16, 4, 1, 4, 0), (2, 4, 1, 4, 300), (64, 40, 1, 40, 5000), (32, 12, 4, 3, 0),
                                                         (32, 300, 300, 1, 0), (8, 70, 40, 5, 999)])
def test_a_workspace_serves_every_smaller_length(dim, heads, tokens, max_q, n, prefix):
    """Parts are not monotonous in the length; what the size call answers is."""
    _, c = kv(dim=dim, ps=8192, hs=4096, ts=256)
    _, s = seqs(n=n, width=4000, prefix_table=FAKE if prefix else None, prefix=prefix)
    try:
        lengths = list(range(1, 4000, 13)) + list(range(4000, 64000, 997))
        sizes = [fq.lib.fq_attend_workspace_bytes(c, s, tokens, heads, max_q, m) for m in lengths]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] >= 256
        for m in lengths[::5]:  # less than the least there is (256 bytes) is refused at every length
            rc = attend(c, s, T=tokens, qs=heads * dim, os=heads * dim, heads=heads, max_q=max_q, max_kv=m, n=255)
            assert rc == B.FQ_ERR_SHAPE
    finally:
        fq.lib.fq_kv_destroy(c), fq.lib.fq_seqs_destroy(s)


def sample(call, logits=FAKE, R=2, V=100, stride=100, u=FAKE, t=None, k=None, p=None, m=None, token=FAKE, prob=None, ws=FAKE, n=1 << 30):
    return call(logits, R, V, stride, u, t, k, p, m, token, prob, ws, n, None)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("bad,code", [
    (dict(R=-1), B.FQ_ERR_SHAPE), (dict(V=0), B.FQ_ERR_SHAPE), (dict(V=(1 << 24) + 1, stride=1 << 25), B.FQ_ERR_SHAPE),
    (dict(stride=99), B.FQ_ERR_SHAPE), (dict(stride=1 << 41), B.FQ_ERR_SHAPE), (dict(logits=None), B.FQ_ERR_NULL),
    (dict(u=None), B.FQ_ERR_NULL), (dict(token=None), B.FQ_ERR_NULL), (dict(ws=None), B.FQ_ERR_NULL),
    (dict(logits=FAKE + 1), B.FQ_ERR_ALIGN), (dict(t=FAKE + 2), B.FQ_ERR_ALIGN), (dict(k=FAKE + 1), B.FQ_ERR_ALIGN),
    (dict(p=FAKE + 2), B.FQ_ERR_ALIGN), (dict(m=FAKE + 2), B.FQ_ERR_ALIGN), (dict(prob=FAKE + 2), B.FQ_ERR_ALIGN),
    (dict(ws=FAKE + 128), B.FQ_ERR_ALIGN), (dict(n=0), B.FQ_ERR_SHAPE)])
def test_sample_refuses(half, bad, code):
    call = fq.lib.fq_sample_f16 if half else fq.lib.fq_sample
    assert sample(call, **bad) == code and fq.fq_last_error()
    assert sample(call, R=0, logits=None, ws=None) == B.FQ_OK
    assert fq.lib.fq_sample_workspace_bytes(-1, 10) == 0 and fq.lib.fq_sample_workspace_bytes(1, 0) == 0


def test_binding_refuses_other_types_and_layouts():
    half = torch.zeros((4, 2, 16, 64), dtype=torch.float16)
    i32 = torch.zeros(3, dtype=torch.int32)
    table = torch.zeros((2, 4), dtype=torch.int32)
    for k, v in ((half.float(), half.float()), (half, half.bfloat16()), (half, half[:, :, :8]),
                 (half.transpose(2, 3), half.transpose(2, 3)), (half[0], half[0])):
        with pytest.raises((ValueError, fq.FlexqError)):
            fq.KVCache(k, v)
    with pytest.raises(ValueError):
        fq.Sequences(i32.long(), i32[:2], table)
    with pytest.raises(ValueError):
        fq.Sequences(i32, i32, table)
    with pytest.raises(ValueError):
        fq.Sequences(i32, i32[:2], table[:, ::2])
    cache, s = fq.KVCache(half, half.clone()), fq.Sequences(i32, i32[:2], table)
    q, ws = torch.zeros((3, 4, 64), dtype=torch.float16), torch.zeros(4096, dtype=torch.uint8)
    for bad in (q.float(), q[:, :, :32], q.transpose(0, 1), q[:2]):
        with pytest.raises((ValueError, fq.FlexqError)):
            fq.fq_attend(cache, s, q, bad, 0.1, 1, 4, ws)
    with pytest.raises(ValueError):
        fq.fq_attend(cache, s, q, q.clone(), 0.1, 1, 4, ws, lse=torch.zeros((3, 4), dtype=torch.float64))
    kk = torch.zeros((3, 2, 64), dtype=torch.float16)
    with pytest.raises(ValueError):
        fq.fq_kv_append(cache, s, q, kk, kk, q.clone(), torch.zeros(32))
    with pytest.raises(ValueError):
        fq.fq_kv_append(cache, s, q, kk, kk, q.clone(), None, positions=torch.zeros(2, dtype=torch.int32))
    short = fq.Sequences(i32, i32[:2], table, torch.zeros(1, dtype=torch.int32), 17)
    with pytest.raises(ValueError):
        fq.fq_attend(cache, short, q, q.clone(), 0.1, 1, 4, ws)
    f, tok = torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    for logits, u, token, kw in ((torch.zeros((2, 9)).double(), f, tok, {}), (torch.zeros((9, 2)).T, f, tok, {}),
                                 (torch.zeros((2, 9)), f[:1], tok, {}), (torch.zeros((2, 9)), f, tok.long(), {}),
                                 (torch.zeros((2, 9)), f, tok, dict(top_k=f)), (torch.zeros((2, 8)), f, tok, {})):
        with pytest.raises(ValueError):
            fq.fq_sample(logits, 2, 9, u, token, ws, **kw)


def test_the_reference_draw_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3], dtype=np.float64)).astype(np.float32)
    f = np.float32
    assert [draw(x, f(u))[0] for u in (0.0, 0.05, 0.15, 0.45, 0.55, 0.65, 0.75, 0.99)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [draw(x, f(u), top_k=2)[0] for u in (0.0, 0.5, 0.6, 0.99)] == [1, 1, 3, 3]
    assert [draw(x, f(u), top_p=f(0.65))[0] for u in (0.0, 0.5, 0.6, 0.99)] == [1, 1, 3, 3]
    assert [draw(x, f(u), min_p=f(0.45))[0] for u in (0.0, 0.4, 0.5, 0.6, 0.7)] == [1, 1, 2, 2, 3]
    assert draw(x, f(0.3), temperature=f(0.0)) == (1, 1.0) and draw(np.full(4, -np.inf, f), f(0.5)) == (-1, 0.0)
    same = np.zeros(10, f)
    assert [draw(same, f(u), top_p=f(0.5))[0] for u in (0.0, 0.9)] == [0, 4]
    assert draw(same, f(0.99), top_k=3) == (2, 1 / 3)
