"""fq_attend against a 64-bit reference: types, head counts and widths, ragged batches, prefixes, holes, garbage in what is
not looked at, empty rows, strides, streams and capture."""
import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq
from serve_util import TYPES, Batch, attend, attend_tolerance, lse_tolerance, pool

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def f64(t):
    return t.double().cpu().numpy()


def call(batch, cache, q, scale, max_q=None, max_kv=None, out=None, lse=True, stream=None, seqs=None):
    T, heads, dim = q.shape
    max_q = max_q or max(max(batch.new), 1)
    max_kv = max_kv or max(max(batch.kv), 1)
    seqs = seqs or batch.sequences()
    if out is None:
        out = torch.full((T, heads, dim), 9.0, dtype=q.dtype, device=DEV)
    lse = torch.full((T, heads), 9.0, dtype=torch.float32, device=DEV) if lse else None
    ws = torch.empty(fq.fq_attend_workspace_bytes(cache, seqs, T, heads, max_q, max_kv), dtype=torch.uint8, device=DEV)
    fq.fq_attend(cache, seqs, q, out, scale, max_q, max_kv, ws, lse=lse, stream=stream)
    return out, lse, ws


def check(batch, out, lse, q, kc, vc, scale, max_kv=None):
    dim = q.shape[2]
    want, want_lse, size, steep, mass = attend(batch, f64(q), f64(kc), f64(vc), scale, max_kv)
    got = f64(out)
    assert np.all(np.isfinite(got))
    err, tol = np.abs(got - want), attend_tolerance(q.dtype, want, size, steep, mass, dim)
    assert np.all(err <= tol), "off by %g of the tolerance at %s" % ((err / tol).max(), np.unravel_index((err / tol).argmax(), err.shape))
    if lse is not None:
        got = f64(lse)
        empty = np.isinf(want_lse)
        assert np.array_equal(got[empty], want_lse[empty])
        tol = lse_tolerance(want_lse[~empty], steep[~empty], dim, batch.prefix + max(batch.kv))
        assert np.all(np.abs(got[~empty] - want_lse[~empty]) <= tol)


def run(batch, q_heads, kv_heads, dim, dtype, token_major=False, spread=1.5, scale=None, garbage=True, max_q=None, max_kv=None,
        lse=True):
    gen = torch.Generator().manual_seed(11)
    kc, vc = (pool(gen, batch.pages, kv_heads, batch.page, dim, dtype, token_major) for _ in range(2))
    if garbage:  # whatever no row may look at is NaN or infinite
        used = np.zeros((batch.pages, batch.page), dtype=bool)
        for b in range(len(batch.new)):
            pages, slots, hole = batch.slots(b)
            used[pages[~hole], slots[~hole]] = True
        dead = torch.from_numpy(~used).to(DEV)[:, None, :, None].expand(kc.shape)
        kc.masked_fill_(dead, float("nan"))
        vc.masked_fill_(dead, float("inf"))
    q = (spread * torch.randn((batch.tokens, q_heads, dim), generator=gen)).to(dtype).to(DEV)
    scale = dim ** -0.5 if scale is None else scale
    out, l, _ = call(batch, fq.KVCache(kc, vc), q, scale, max_q, max_kv, lse=lse)
    torch.cuda.synchronize()
    check(batch, out, l, q, torch.nan_to_num(kc), torch.nan_to_num(vc), scale, max_kv)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (8, 1), (6, 2), (32, 2), (40, 2), (5, 5)])
@pytest.mark.parametrize("dim", [8, 64, 80, 96, 128, 136, 256])
def test_heads_and_widths_of_single_tokens(dtype, heads, dim):
    run(Batch([1, 1, 1, 1], [70, 1, 33, 200], 16), heads[0], heads[1], dim, TYPES[dtype], token_major=dim == 80)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (8, 1), (6, 2), (40, 2)])
@pytest.mark.parametrize("dim", [8, 64, 80, 128, 192, 256])
def test_heads_and_widths_of_chunks(dtype, heads, dim):
    run(Batch([30, 1, 7], [75, 1, 140], 16), heads[0], heads[1], dim, TYPES[dtype], token_major=dim == 80)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1023, 1025])
def test_lengths_around_tiles(n):
    run(Batch([1], [n], 16), 4, 2, 64, torch.float16)
    run(Batch([min(n, 70)], [n], 8), 2, 1, 128, torch.bfloat16)


@pytest.mark.parametrize("page", [1, 2, 8, 32, 64, 128, 1024])
def test_pages(page):
    run(Batch([1, 1], [300, 77], page), 8, 2, 128, torch.float16)
    run(Batch([40, 3], [300, 77], page), 4, 4, 64, torch.float16, token_major=True)


@pytest.mark.parametrize("new", [1, 2, 5, 20, 90])
def test_long_histories(new):
    run(Batch([new], [5000 + new], 32), 8, 2, 64, torch.float16, spread=3.0)
    run(Batch([new, 1, new], [2000, 1, 3 + new], 16), 4, 4, 128, torch.bfloat16)


@pytest.mark.parametrize("prefix", [1, 15, 16, 64, 100, 257, 1500])
@pytest.mark.parametrize("heads,seqs", [((8, 1), 3), ((4, 4), 3), ((8, 2), 40), ((16, 1), 40)])
def test_shared_prefixes(prefix, heads, seqs):
    kv = [(7 * i) % 40 + 1 for i in range(seqs)]
    run(Batch([1] * seqs, kv, 16, prefix=prefix), heads[0], heads[1], 64, torch.float16)


@pytest.mark.parametrize("new", [[1, 2, 3], [4, 0, 30], [100, 1, 65]])
def test_ragged_chunks_behind_a_prefix(new):
    run(Batch(new, [n + 9 for n in new], 8, prefix=203), 4, 2, 64, torch.float16, lse=False)


@pytest.mark.parametrize("dim,heads", [(64, (8, 2)), (128, (4, 4)), (80, (2, 1)), (256, (2, 2))])
def test_prompts_among_single_tokens(dim, heads):
    """Row blocks of many sequences follow each other: empty ones, more than 64, prompts first, last and between."""
    for new in ([150, 1, 1, 40, 0, 0, 7], [0, 0, 1, 300], [1] * 70 + [130, 0, 33] + [2] * 60, [90] * 3):
        kv = [n + (13 * i) % 50 for i, n in enumerate(new)]
        run(Batch(new, kv, 16), heads[0], heads[1], dim, torch.float16)
    run(Batch([150, 1, 0, 40], [160, 300, 0, 40], 16), heads[0], heads[1], dim, torch.bfloat16, max_q=151)


@pytest.mark.parametrize("new", [[1, 2, 3], [4, 0, 30], [100, 1, 65]])
def test_shared_prefixes_of_chunks(new):
    run(Batch(new, [n + 9 for n in new], 8, prefix=203), 4, 2, 128, torch.float16)
    run(Batch(new, new, 8, prefix=64), 8, 2, 64, torch.bfloat16)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads,dim", [((4, 2), 64), ((8, 1), 128), ((2, 2), 80), ((2, 1), 256)])
@pytest.mark.parametrize("new,kv", [([4], [200]), ([3, 1], [64, 9]), ([40], [40]), ([150], [390]), ([70, 5], [70, 300])])
def test_new_tokens_that_are_not_finite_reach_no_earlier_row(dtype, heads, dim, new, kv):
    """Infinities and NaNs in K and V of a chunk's later tokens: rows before them are as if they were not there, rows that see
    a NaN are NaN."""
    batch = Batch(new, kv, 8)
    gen = torch.Generator().manual_seed(21)
    kc, vc = (pool(gen, batch.pages, heads[1], 8, dim, TYPES[dtype]) for _ in range(2))
    q = torch.randn((batch.tokens, heads[0], dim), generator=gen).to(TYPES[dtype]).to(DEV)
    first_bad = [n - n // 2 for n in new]  # of the new tokens
    for b, (n, m) in enumerate(zip(new, kv)):
        for j in range(first_bad[b], n):
            p = m - n + j
            vc[int(batch.table[b, p // 8]), :, p % 8, j % dim] = [float("nan"), float("inf"), -float("inf")][j % 3]
            if j % 2:
                kc[int(batch.table[b, p // 8]), :, p % 8, 3] = float("nan")
    out, lse, _ = call(batch, fq.KVCache(kc, vc), q, 0.1)
    torch.cuda.synchronize()
    keep = np.concatenate([np.arange(n) < f for n, f in zip(new, first_bad)])
    want, want_lse, size, steep, mass = attend(batch, f64(q), f64(torch.nan_to_num(kc, 0, 0, 0)), f64(torch.nan_to_num(vc, 0, 0, 0)), 0.1)
    got, tol = f64(out), attend_tolerance(q.dtype, want, size, steep, mass, dim)
    assert np.all(np.abs(got[keep] - want[keep]) <= tol[keep])
    assert np.all(np.abs(f64(lse)[keep] - want_lse[keep]) <= lse_tolerance(want_lse[keep], steep[keep], dim, max(kv)))
    for b, (n, f) in enumerate(zip(new, first_bad)):
        for j in range(f, n):  # every row from the first bad token on sees that one's V
            assert not np.isfinite(got[batch.q_start[b] + j, :, f % dim]).any()


@pytest.mark.parametrize("new", [1, 40])
def test_an_infinite_value_that_is_seen_stays_one(new):
    batch = Batch([new], [100 + new], 16)
    gen = torch.Generator().manual_seed(22)
    kc, vc = (pool(gen, batch.pages, 2, 16, 64, torch.float16) for _ in range(2))
    vc[int(batch.table[0, 0]), 1, 5, 7] = float("inf")
    q = torch.randn((new, 4, 64), generator=gen).half().to(DEV)
    out, _, _ = call(batch, fq.KVCache(kc, vc), q, 0.1)
    torch.cuda.synchronize()
    assert torch.all(out[:, 2:, 7] == float("inf"))
    out[:, 2:, 7] = 0
    assert torch.all(torch.isfinite(out))


def test_rows_that_see_nothing():
    """Lengths of zero, more new tokens than length, no own keys behind a prefix."""
    run(Batch([1, 1, 1], [0, 5, 0], 4), 4, 2, 64, torch.float16)
    run(Batch([6, 0, 70], [2, 0, 3], 4), 4, 2, 64, torch.float16)
    run(Batch([1, 1], [0, 0], 4, prefix=9), 4, 2, 64, torch.float16)
    run(Batch([6, 70], [2, 0], 4, prefix=9), 4, 2, 64, torch.float16)


@pytest.mark.parametrize("new", [1, 40])
def test_holes(new):
    batch = Batch([new, new], [200, 100], 16, prefix=70)
    batch.table[0, 1], batch.table[0, 2], batch.table[0, 12] = -1, batch.pages, 2 ** 31 - 1
    batch.table[1, :] = -(2 ** 31)
    batch.prefix_table[2] = -5
    run(batch, 4, 2, 64, torch.float16)
    batch.prefix_table[:] = -1  # the second sequence now sees nothing at all
    run(batch, 8, 2, 64, torch.bfloat16)


def test_bounds_given_by_the_caller():
    run(Batch([1, 1], [200, 40], 16, width=20), 4, 2, 64, torch.float16, max_kv=10 ** 9)
    run(Batch([3, 1], [200, 40], 16), 4, 2, 64, torch.float16, max_q=4, max_kv=50)  # keys beyond are not seen
    run(Batch([1, 1], [200, 40], 16), 4, 2, 64, torch.float16, max_kv=1, lse=False)


@pytest.mark.parametrize("heads,new,prefix", [((32, 32), [1], 0), ((8, 2), [1, 1, 1], 700), ((8, 1), [4, 2], 0), ((4, 4), [130], 0)])
def test_one_workspace_for_all_lengths(heads, new, prefix):
    """Sized for the longest, used for every length: the launch asks for no more, and writes no further."""
    width = 260
    gen = torch.Generator().manual_seed(31)
    long = Batch(new, [4100] * len(new), 16, prefix=prefix, width=width)
    kc, vc = (pool(gen, long.pages, heads[1], 16, 64, torch.float16) for _ in range(2))
    cache = fq.KVCache(kc, vc)
    q = torch.randn((long.tokens, heads[0], 64), generator=gen).half().to(DEV)
    seqs = long.sequences()
    need = fq.fq_attend_workspace_bytes(cache, seqs, long.tokens, heads[0], max(new), 4100)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(q), torch.empty((long.tokens, heads[0]), device=DEV)
    for m in (130, 400, 900, 1500, 2500, 3100, 4100):
        seqs._keep[1].fill_(m)
        fq.fq_attend(cache, seqs, q, out, 0.125, max(new), m, ws[:need], lse=lse)
        torch.cuda.synchronize()
        long.kv = [m] * len(new)
        check(long, out, lse, q, kc, vc, 0.125)
        assert torch.all(ws[need:] == 77)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0, 30.0])
def test_scales(scale):
    run(Batch([1, 5], [300, 77], 16), 8, 2, 64, torch.float16, scale=scale)
    run(Batch([50], [300], 16), 8, 2, 64, torch.bfloat16, scale=scale)


@pytest.mark.parametrize("new", [1, 40])
def test_rows_apart_and_rows_beyond_max_q(new):
    batch = Batch([new, new + 2], [90, 80], 16)
    gen = torch.Generator().manual_seed(3)
    kc, vc = (pool(gen, batch.pages, 2, 16, 64, torch.float16) for _ in range(2))
    wide = torch.randn((batch.tokens, 9, 64), generator=gen).half().to(DEV)
    q, out = wide[:, 1:5], torch.full((batch.tokens, 6, 64), 9.0, dtype=torch.float16, device=DEV)
    o, lse, _ = call(batch, fq.KVCache(kc, vc), q, 0.125, out=out[:, 2:])
    torch.cuda.synchronize()
    check(batch, o, lse, q, kc, vc, 0.125)
    assert torch.all(out[:, :2] == 9.0)
    o, lse, _ = call(batch, fq.KVCache(kc, vc), q, 0.125, max_q=new)
    torch.cuda.synchronize()
    assert torch.all(o[2 * new:] == 9.0) and torch.all(lse[2 * new:] == 9.0) and not torch.any(o[:2 * new] == 9.0)


def test_scores_that_overflow_the_type_and_equal_keys():
    """Large scores keep their softmax (binary32 statistics); equal keys give the mean of the values."""
    batch = Batch([1, 33], [100, 70], 16)
    run(batch, 4, 2, 128, torch.float16, spread=60.0, scale=1.0)
    gen = torch.Generator().manual_seed(5)
    kc = torch.ones((batch.pages, 2, 16, 64), dtype=torch.float16, device=DEV)
    vc = pool(gen, batch.pages, 2, 16, 64, torch.float16)
    q = torch.randn((34, 4, 64), generator=gen).half().to(DEV)
    out, lse, _ = call(batch, fq.KVCache(kc, vc), q, 0.1)
    torch.cuda.synchronize()
    check(batch, out, lse, q, kc, vc, 0.1)


def test_equal_calls_give_equal_bits_on_any_stream_and_in_a_graph():
    for batch, heads in ((Batch([1] * 5, [900, 3, 77, 450, 1], 16, prefix=300), (8, 2)), (Batch([70, 9], [200, 9], 16), (4, 4))):
        gen = torch.Generator().manual_seed(4)
        kc, vc = (pool(gen, batch.pages, heads[1], 16, 64, torch.float16) for _ in range(2))
        cache, seqs = fq.KVCache(kc, vc), batch.sequences()
        q = torch.randn((batch.tokens, heads[0], 64), generator=gen).half().to(DEV)
        first, first_lse, _ = call(batch, cache, q, 0.2, seqs=seqs)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        again, again_lse, keep = call(batch, cache, q, 0.2, stream=side, seqs=seqs)
        side.synchronize()
        assert torch.equal(first, again) and torch.equal(first_lse, again_lse)
        T = batch.tokens
        out, lse = torch.empty_like(q), torch.empty((T, heads[0]), device=DEV)
        max_q, max_kv = max(batch.new), max(batch.kv)
        ws = torch.empty(fq.fq_attend_workspace_bytes(cache, seqs, T, heads[0], max_q, max_kv), dtype=torch.uint8, device=DEV)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=torch.cuda.Stream()):
            fq.fq_attend(cache, seqs, q, out, 0.2, max_q, max_kv, ws, lse=lse)
        for step in range(4):
            ws.fill_(255)  # nothing is expected of what an earlier call left
            g.replay()
            torch.cuda.synchronize()
            eager, eager_lse, _ = call(batch, cache, q, 0.2, seqs=seqs)
            torch.cuda.synchronize()
            assert torch.equal(out, eager) and torch.equal(lse, eager_lse)
            q.mul_(1.1)
            seqs._keep[1].sub_(1).clamp_(min=0)  # shorter sequences in the same graph
            out.zero_()


def test_pages_past_32_bits():
    """A pool of more than 2^32 elements: the last pages hold the sequence."""
    page, heads, dim = 64, 8, 128
    pages = (1 << 32) // (page * heads * dim) + 9
    kc = torch.empty((pages, heads, page, dim), dtype=torch.float16, device=DEV)
    vc = torch.empty_like(kc)
    batch = Batch([2, 1], [150, 64], page, spare=0)
    gen = torch.Generator().manual_seed(6)
    small = [pool(gen, batch.pages, heads, page, dim, torch.float16) for _ in range(2)]
    kc[-batch.pages:], vc[-batch.pages:] = small[0], small[1]
    q = torch.randn((3, 16, dim), generator=gen).half().to(DEV)
    far = Batch([2, 1], [150, 64], page, spare=0)
    far.table = far.table + np.int32(pages - batch.pages)
    out, lse, _ = call(far, fq.KVCache(kc, vc), q, 0.1)
    torch.cuda.synchronize()
    check(batch, out, lse, q, small[0], small[1], 0.1)
    # and the append finds its way there
    k = torch.randn((3, heads, dim), generator=gen).half().to(DEV)
    fq.fq_kv_append(fq.KVCache(kc, vc), far.sequences(), None, k, k, None, None)
    torch.cuda.synchronize()
    for t, (b, p) in enumerate(far.places()):
        assert torch.equal(kc[int(far.table[b, p // page]), :, p % page], k[t])
