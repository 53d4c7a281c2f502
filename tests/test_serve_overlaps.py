"""Rows that overlap, without a GPU: an accepted call is stopped by a later check, so nothing is launched."""
import random

import pytest

import paper_2506_12024_amd as fq
from paper_2506_12024_amd import binding as B
from test_serve_pins import append, attend, kv, seqs

BASE = 0x100000


@pytest.fixture
def handles():
    (_, c), (_, s) = kv(), seqs()
    yield c, s
    fq.lib.fq_kv_destroy(c), fq.lib.fq_seqs_destroy(s)


def code(handles, **kw):
    """FQ_ERR_ALIGN (of the frequencies, looked at last) where the rows pass."""
    return append(*handles, freqs=BASE + 4, **kw)


@pytest.mark.parametrize("rot", [64, 20, 0])
@pytest.mark.parametrize("off", [-2 * 512 - 496, -1024, -512, -16, 0, 16, 256, 512, 1024, 2 * 512 + 496])
def test_rotated_queries_may_not_overlap_the_queries(handles, rot, off):
    """Three rows of four heads of 64 (512 bytes), at any distance that leaves a value in common."""
    assert code(handles, q=BASE, o=BASE + off, rot=rot) == B.FQ_ERR_SHAPE and "overlap" in fq.fq_last_error()
    for name in "kv":
        assert code(handles, q=BASE + 0x10000, o=BASE + off, rot=rot, **{name: BASE, name + "s": 256}) == (
            B.FQ_ERR_SHAPE if off < 2 * 512 + 256 else B.FQ_ERR_ALIGN)  # (their last row ends there)


@pytest.mark.parametrize("off", [-0x10000, -3 * 512, 3 * 512, 0x10000])
def test_rows_that_share_nothing_pass(handles, off):
    assert code(handles, q=BASE, o=BASE + off) == B.FQ_ERR_ALIGN
    # q, k, v and the place for the turned queries as parts of one row
    row = dict(qs=768, os=768, ks=768, vs=768)
    assert code(handles, q=BASE, o=BASE + 512, k=BASE + 1024, v=BASE + 1280, **row) == B.FQ_ERR_ALIGN
    assert code(handles, q=BASE, o=BASE + 528, k=BASE + 1024, v=BASE + 1280, **row) == B.FQ_ERR_SHAPE
    assert code(handles, q=BASE, o=BASE + 768, k=BASE + 1024, v=BASE + 1280, **row) == B.FQ_ERR_SHAPE


def test_overlaps_as_counted_value_by_value(handles):
    rng = random.Random(3)
    met = [0, 0]
    for _ in range(3000):
        T = rng.randint(1, 9)
        place = {n: BASE + 16 * rng.randint(0, 400) for n in "qkvo"}
        stride = {n: (256 if n in "qo" else 128) + 8 * rng.choice([0, rng.randint(0, 80)]) for n in "qkvo"}
        if rng.random() < 0.5:
            stride = dict.fromkeys("qkvo", 256 + 8 * rng.randint(0, 100))
        held = {n: {place[n] // 16 + stride[n] // 8 * t + i for t in range(T) for i in range(32 if n in "qo" else 16)} for n in "qkvo"}
        meets = any(held["o"] & held[n] for n in "qkv")
        met[meets] += 1
        rc = code(handles, T=T, q=place["q"], o=place["o"], k=place["k"], v=place["v"], qs=stride["q"], os=stride["o"], ks=stride["k"],
                  vs=stride["v"])
        assert rc == (B.FQ_ERR_SHAPE if meets else B.FQ_ERR_ALIGN), (T, place, stride)
    assert min(met) > 300


def test_strides_of_any_size(handles):
    far = 1 << 62
    assert code(handles, q=BASE, o=BASE + 512, qs=far, os=far) == B.FQ_ERR_ALIGN
    assert code(handles, q=BASE, o=BASE + 256, qs=far, os=far) == B.FQ_ERR_SHAPE
    assert code(handles, T=0x7fffffff, q=BASE, o=BASE + 512, qs=far, os=far, ks=far, vs=far) == B.FQ_ERR_ALIGN


def test_results_may_not_partly_overlap_the_queries(handles):
    def refused(o, **kw):  # (the scale, looked at last, stops a call that passes)
        assert attend(*handles, q=BASE, o=o, scale=float("nan"), **kw) == B.FQ_ERR_SHAPE
        return "overlap" in fq.fq_last_error()
    for off in (-1520, -1024, -512, -16, 16, 512, 1024, 1520):
        assert refused(BASE + off)
    assert refused(BASE, os=264) and refused(BASE + 512, qs=504, os=504) and refused(BASE - 16, qs=1000, os=264)
    row = dict(qs=768, os=768)
    assert not any(refused(o, **kw) for o, kw in ((BASE, {}), (BASE + 512, row), (BASE + 1024, row), (BASE - 1536, {}), (BASE + 1536, {})))
    assert refused(BASE + 496, **row) and refused(BASE + 1040, **row)
