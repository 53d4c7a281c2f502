"""fq_attend at the ends of its arithmetic, against the same 64-bit reference: scores of any size, weights of any size."""
import copy
import math

import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq
from serve_util import EPS, TYPES, Batch, attend, attend_tolerance, lse_tolerance, pool
from test_gpu_attend import call, check, f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("new,prefix", [([1, 1, 1], 0), ([1, 2, 1], 100), ([40], 0), ([150, 9], 70)])
@pytest.mark.parametrize("scale", [1.0, -0.37, 300.0])
def test_equal_largest_scores_of_any_size(dtype, dim, new, prefix, scale):
    equal_largest_scores(dtype, dim, new, prefix, scale, False)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("new,prefix", [([2, 3, 2], 0), ([40], 0), ([150, 9], 70)])
@pytest.mark.parametrize("scale", [1.0, -0.37, 300.0])
def test_equal_largest_scores_beside_values_that_are_not_finite(dtype, new, prefix, scale):
    equal_largest_scores(dtype, 64, new, prefix, scale, True)


def equal_largest_scores(dtype, dim, new, prefix, scale, odd):
    """Scores that are exact in binary32 (one product), from 10^5 to 10^12: the largest ones of a row are equal and share
    its weight, everything else is further down than any weight reaches.  odd: each last new token's value is NaN."""
    batch = Batch(new, [n + 150 for n in new], 16, prefix=prefix)
    gen = torch.Generator().manual_seed(41)
    vc = pool(gen, batch.pages, 2, 16, dim, TYPES[dtype])
    near = torch.rand((batch.pages, 2, 16), generator=gen) < 0.05
    near[batch.table[:, 0], :, 0] = True  # the first key of every sequence among them
    sign = 1.0 if scale > 0 else -1.0
    kc = torch.zeros((batch.pages, 2, 16, dim), dtype=TYPES[dtype])
    kc[..., 3] = torch.where(near, sign * 49152.0, sign * 512.0).to(TYPES[dtype])
    q = torch.zeros((batch.tokens, 4, dim), dtype=TYPES[dtype])
    sizes = np.exp(np.linspace(math.log(4.0), math.log(60000.0), batch.tokens * 4)).reshape(batch.tokens, 4)
    q[..., 3] = torch.from_numpy(sizes).to(TYPES[dtype])
    kc, q = kc.to(DEV), q.to(DEV)
    if odd:
        for b, n in enumerate(batch.kv):
            vc[int(batch.table[b, (n - 1) // 16]), :, (n - 1) % 16] = float("nan")
    out, lse, _ = call(batch, fq.KVCache(kc, vc), q, scale)
    torch.cuda.synchronize()
    keep = np.ones(batch.tokens, dtype=bool)
    if odd:
        keep[batch.q_start[1:] - 1] = False
    want, want_lse, size, _, _ = (x[keep] for x in attend(batch, f64(q), f64(kc), f64(vc), float(np.float32(scale))))
    out, lse = f64(out)[keep], f64(lse)[keep]
    # the scores are exact and equal, so are their weights: the roundings of these (binary32, then the type) and of the result
    half = EPS[TYPES[dtype]] / 2
    tol = half * (1 + half) * (np.abs(want) + size) + 2.0 ** -20 * size + 2.0 ** -25
    share = np.abs(out - want) / tol
    assert np.all(share <= 1), "off by %g of the tolerance at %s" % (share.max(), np.unravel_index(share.argmax(), share.shape))
    assert np.all(np.abs(lse - want_lse) <= 32 * 2.0 ** -24 * (1 + np.abs(want_lse)))


@pytest.mark.parametrize("new", [[1, 1], [3], [40, 1]])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -121, -(2.0 ** -119), 2.0 ** -126, 2.0 ** -140, -(2.0 ** -149)])
@pytest.mark.parametrize("dim", [64, 128])
def test_smallest_scales_of_the_largest_products(new, scale, dim):
    """bfloat16 queries and keys of 2^58: products of 2^120 under scales down to the smallest binary32 value and 0."""
    batch = Batch(new, [n + 150 for n in new], 16)
    gen = torch.Generator().manual_seed(43)
    kc, vc = (pool(gen, batch.pages, 2, 16, dim, torch.bfloat16) for _ in range(2))
    kc.mul_(2.0 ** 58)
    q = (2.0 ** 58 * torch.randn((batch.tokens, 4, dim), generator=gen)).bfloat16().to(DEV)
    out, lse, _ = call(batch, fq.KVCache(kc, vc), q, scale)
    torch.cuda.synchronize()
    check(batch, out, lse, q, kc, vc, scale)


def strong_and_weak(dtype, fall, new, kv, odd=False):
    """The first key of every sequence has a score of 0 and a value of 0, the others -fall (in powers of two) and values about
    1; odd: the last new token's value is NaN.  For three rows (result, lse, and what serve_util.attend says of it), one at a
    time: a row's keys, of the first and the last head."""
    heads, dim = 32, 64
    batch = Batch(new, kv, 64)
    gen = torch.Generator().manual_seed(47)
    shape = (batch.pages, heads, 64, dim)
    kc = torch.zeros(shape, dtype=dtype, device=DEV)
    vc = (1.0 + 0.25 * torch.randn((batch.pages, 1, 64, dim), generator=gen)).to(dtype).to(DEV).expand(shape).contiguous()
    kc[..., 5] = -fall * math.log(2.0) / 8.0
    first = torch.from_numpy(batch.table[:, 0]).long().to(DEV)
    kc[first, :, 0], vc[first, :, 0] = 0.0, 0.0
    q = torch.zeros((batch.tokens, heads, dim), dtype=dtype, device=DEV)
    q[..., 5] = 8.0
    some, rows = [0, heads - 1], (0, batch.tokens // 2 + 5, batch.tokens - 1)
    if odd:
        rows = [batch.tokens - n for n in (2, 50, 100)]
        vc[int(batch.table[0, (kv[0] - 1) // 64]), :, (kv[0] - 1) % 64] = float("nan")
    out, lse, _ = call(batch, fq.KVCache(kc, vc), q, 1.0)
    torch.cuda.synchronize()
    k64, v64 = f64(kc[:, some]), f64(vc[:, some])
    for row in rows:
        b, place = batch.places()[row]
        one = copy.copy(batch)
        one.new, one.kv, one.table, one.q_start = [1], [place + 1], batch.table[b:b + 1], np.array([0, 1])
        yield f64(out[row:row + 1, some]), f64(lse[row:row + 1, some]), place + 1, attend(one, f64(q[row:row + 1, some]), k64, v64, 1.0)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("fall", [0.0, 5.0, 12.3, 24.3])
@pytest.mark.parametrize("new,kv,odd", [([1024], [32768], False), ([1024], [32768], True), ([1] * 24, [8192] * 24, False)])
def test_sums_of_long_rows_lose_nothing(dtype, fall, new, kv, odd):
    """Tens of thousands of equal weights beside a large one, in every kernel and (odd) on the way round values that are not
    finite: the sum is as good as one of few."""
    for out, lse, keys, (want, want_lse, size, steep, mass) in strong_and_weak(TYPES[dtype], fall, new, kv, odd):
        off = np.abs(lse - want_lse) / lse_tolerance(want_lse, steep, 64, keys)
        assert np.all(off <= 1), "lse off by %g of the tolerance" % off.max()
        if odd:
            off = np.abs(out - want) / attend_tolerance(TYPES[dtype], want, size, steep, mass, 64)
            assert np.all(off <= 1), "off by %g of the tolerance" % off.max()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("fall", [12.3, 20.4, 24.3, 27.5])
@pytest.mark.parametrize("new,kv", [([1024], [32768]), ([1] * 24, [8192] * 24)])
def test_weak_keys_beside_a_strong_one_keep_their_share(dtype, fall, new, kv):
    """The result is what the weak keys hold, the strong one's value being 0.  A weight errs by half a step of its type, in
    binary16 by 2^-25 at least, where the largest is 2^7 and more: 2^-32 of the largest, 2^7 less than beside a largest of 1."""
    for out, _, _, (want, _, size, steep, mass) in strong_and_weak(TYPES[dtype], fall, new, kv):
        off = np.abs(out - want) / attend_tolerance(TYPES[dtype], want, size, steep, mass / 128, 64)
        assert np.all(off <= 1), "off by %g of the tolerance" % off.max()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads,dim", [((4, 2), 64), ((8, 1), 128), ((2, 2), 80), ((2, 1), 256)])
@pytest.mark.parametrize("new,own", [([4], 0), ([3, 1], 60), ([40], 90), ([150], 9), ([70, 5], 30)])
def test_values_that_are_not_finite_behind_a_prefix(dtype, heads, dim, new, own):
    """A chunk's later tokens hold infinities and NaNs, and it stands behind a prefix with a hole: rows before them see prefix
    and cache as if they were not there."""
    batch = Batch(new, [n + own for n in new], 8, prefix=77)
    batch.prefix_table[3] = -1
    gen = torch.Generator().manual_seed(51)
    kc, vc = (pool(gen, batch.pages, heads[1], 8, dim, TYPES[dtype]) for _ in range(2))
    q = torch.randn((batch.tokens, heads[0], dim), generator=gen).to(TYPES[dtype]).to(DEV)
    first_bad = [n - n // 2 for n in new]
    for b, n in enumerate(new):
        for j in range(first_bad[b], n):
            p = own + j
            vc[int(batch.table[b, p // 8]), :, p % 8, j % dim] = [float("nan"), float("inf"), -float("inf")][j % 3]
            if j % 2:
                kc[int(batch.table[b, p // 8]), :, p % 8, 3] = float("nan")
    out, lse, _ = call(batch, fq.KVCache(kc, vc), q, 0.1)
    torch.cuda.synchronize()
    keep = np.concatenate([np.arange(n) < f for n, f in zip(new, first_bad)])
    want, want_lse, size, steep, mass = attend(batch, f64(q), f64(torch.nan_to_num(kc, 0, 0, 0)), f64(torch.nan_to_num(vc, 0, 0, 0)), 0.1)
    got, tol = f64(out), attend_tolerance(q.dtype, want, size, steep, mass, dim)
    assert np.all(np.abs(got[keep] - want[keep]) <= tol[keep])
    assert np.all(np.abs(f64(lse)[keep] - want_lse[keep]) <= lse_tolerance(want_lse[keep], steep[keep], dim, 77 + max(batch.kv)))
    for b, (n, f) in enumerate(zip(new, first_bad)):
        for j in range(f, n):
            assert not np.isfinite(got[batch.q_start[b] + j, :, f % dim]).any()


@pytest.mark.parametrize("new,kv,prefix,odd", [([1, 1, 1], [900, 3, 70], 0, False), ([1, 2], [40, 50], 300, False), ([40, 3], [60, 300], 0, False),
                                               ([300, 0, 5], [999, 0, 5], 70, False), ([4, 130], [30, 400], 0, True)])
@pytest.mark.parametrize("heads,dim", [((8, 2), 64), ((4, 4), 128), ((2, 1), 256)])
def test_results_in_the_place_of_the_queries(new, kv, prefix, odd, heads, dim):
    """The same bits as with a tensor of its own, in rows that lie apart too, and past values that are not finite."""
    batch = Batch(new, kv, 16, prefix=prefix)
    gen = torch.Generator().manual_seed(57)
    kc, vc = (pool(gen, batch.pages, heads[1], 16, dim, torch.float16) for _ in range(2))
    if odd:
        for b, n in enumerate(kv):
            vc[int(batch.table[b, (n - 1) // 16]), :, (n - 1) % 16] = float("nan")
    wide = torch.randn((batch.tokens, heads[0] + 1, dim), generator=gen).half().to(DEV)
    kept, q = wide[:, -1].clone(), wide[:, :heads[0]]
    cache = fq.KVCache(kc, vc)
    want, want_lse, _ = call(batch, cache, q.contiguous(), 0.2)
    out, lse, _ = call(batch, cache, q, 0.2, out=q)
    torch.cuda.synchronize()
    assert torch.equal(out.nan_to_num(7.0), want.nan_to_num(7.0)) and torch.equal(lse, want_lse)
    assert torch.equal(wide[:, -1], kept)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("heads,dim", [((8, 2), 64), ((4, 4), 128), ((2, 2), 80), ((2, 1), 256)])
@pytest.mark.parametrize("new,own,prefix", [([3], 200, 0), ([2, 3], 40, 90), ([40], 300, 0), ([200, 3], 100, 50)])
def test_an_old_infinite_value_is_an_infinity_in_every_row_that_sees_it(dtype, heads, dim, new, own, prefix):
    """In the cache (all rows see it), in the prefix, and in a new token, each in a column of its own; a column with both
    signs is NaN; all other columns are as if the infinities were not there."""
    batch = Batch(new, [n + own for n in new], 16, prefix=prefix)
    gen = torch.Generator().manual_seed(61)
    kc, vc = (pool(gen, batch.pages, heads[1], 16, dim, TYPES[dtype]) for _ in range(2))
    inf = float("inf")
    late = [n + own - 1 - n // 3 for n in new]  # the place of a new token of each sequence
    for b in range(len(new)):
        vc[int(batch.table[b, 0]), :, 3, 5] = inf
        vc[int(batch.table[b, late[b] // 16]), :, late[b] % 16, 6] = -inf
        vc[int(batch.table[b, 1]), :, 2, 7] = inf
        vc[int(batch.table[b, late[b] // 16]), :, late[b] % 16, 7] = -inf
    if prefix:
        vc[int(batch.prefix_table[0]), :, 0, 4] = -inf
    q = torch.randn((batch.tokens, heads[0], dim), generator=gen).to(TYPES[dtype]).to(DEV)
    out, lse, _ = call(batch, fq.KVCache(kc, vc), q, 0.1)
    torch.cuda.synchronize()
    got = f64(out)
    want, want_lse, size, steep, mass = attend(batch, f64(q), f64(kc), f64(torch.nan_to_num(vc, 0, 0, 0)), 0.1)
    odd = np.zeros(dim, dtype=bool)
    odd[[5, 6, 7] + ([4] if prefix else [])] = True
    tol = attend_tolerance(q.dtype, want, size, steep, mass, dim)
    assert np.all(np.abs(got - want)[..., ~odd] <= tol[..., ~odd])
    assert np.all(np.abs(f64(lse) - want_lse) <= lse_tolerance(want_lse, steep, dim, prefix + max(batch.kv)))
    assert np.all(got[..., 5] == inf) and (not prefix or np.all(got[..., 4] == -inf))
    for t, (b, place) in enumerate(batch.places()):
        if place >= late[b]:
            assert np.all(got[t, :, 6] == -inf) and np.all(np.isnan(got[t, :, 7]))
        else:
            assert np.all(np.abs(got[t, :, 6] - want[t, :, 6]) <= tol[t, :, 6]) and np.all(got[t, :, 7] == inf)


@pytest.mark.parametrize("place", [5, 1500])
def test_values_that_are_not_finite_take_no_other_time(place):
    """One infinity among 2048 keys, in an old token and in a new one: a prompt takes a few times what it takes without at most
    (500 times where such calls were computed row by row)."""
    batch = Batch([1024], [2048], 16)
    gen = torch.Generator(device=DEV).manual_seed(63)
    kc, vc = (torch.randn((batch.pages, 8, 16, 128), generator=gen, device=DEV).half() for _ in range(2))
    q = torch.randn((1024, 64, 128), generator=gen, device=DEV).half()
    cache, seqs, out = fq.KVCache(kc, vc), batch.sequences(), torch.empty_like(q)
    ws = torch.empty(fq.fq_attend_workspace_bytes(cache, seqs, 1024, 64, 1024, 2048), dtype=torch.uint8, device=DEV)

    def least():
        times = []
        for _ in range(6):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            fq.fq_attend(cache, seqs, q, out, 0.1, 1024, 2048, ws)
            end.record()
            end.synchronize()
            times.append(begin.elapsed_time(end))
        return min(times)
    without = least()
    vc[int(batch.table[0, place // 16]), :, place % 16, 9] = float("inf")
    assert least() < 20 * without
