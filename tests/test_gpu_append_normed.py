"""fq_kv_append_normed against a 64-bit reference: layouts, parts of a head, weights, strides, bad pages, magnitudes, capture."""
import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq
from serve_util import EPS, TYPES, Batch, pool, turn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def f64(t):
    return t.double().cpu().numpy()


def normed(x, w, eps, offset):
    return x / np.sqrt((x ** 2).mean(axis=2, keepdims=True) + eps) * (w + offset)


def run(batch, q_heads, kv_heads, dim, rot, interleaved, dtype, token_major=False, fused=False, positions=None, amplitude=1.0,
        with_q=True, each=False, offset=0.0, eps=1e-6, size=3.0):
    gen = torch.Generator().manual_seed(7)
    T = batch.tokens
    kc, vc = (pool(gen, batch.pages, kv_heads, batch.page, dim, dtype, token_major) for _ in range(2))
    k0, v0 = f64(kc), f64(vc)
    row = (size * torch.randn((T, q_heads + 2 * kv_heads, dim), generator=gen, dtype=torch.float64)).to(dtype).to(DEV)
    q, k, v = row[:, :q_heads], row[:, q_heads:q_heads + kv_heads], row[:, q_heads + kv_heads:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    qw, kw = ((1.0 - offset + 0.3 * torch.randn((n, dim) if each else (dim,), generator=gen)).to(dtype).to(DEV)
              for n in (q_heads, kv_heads))
    q_out = torch.full((T, q_heads, dim), 9.0, dtype=dtype, device=DEV)
    freqs = fq.fq_rope_freqs(rot, 10000.0) if rot else []
    pos = np.array([p + batch.prefix for _, p in batch.places()]) if positions is None else positions
    fq.fq_kv_append_normed(fq.KVCache(kc, vc), batch.sequences(), q if with_q else None, k, v, q_out if with_q else None,
                           torch.tensor(freqs, dtype=torch.float64, device=DEV) if rot else None, qw if with_q else None, kw, eps, offset,
                           interleaved, amplitude, None if positions is None else torch.from_numpy(positions).int().to(DEV))
    torch.cuda.synchronize()
    nq, nk = normed(f64(q), f64(qw), eps, offset), normed(f64(k), f64(kw), eps, offset)
    if rot:
        want_q, size_q = turn(nq, pos, freqs, rot, interleaved, amplitude)
        want_k, size_k = turn(nk, pos, freqs, rot, interleaved, amplitude)
    else:
        want_q, want_k, size_q, size_k = nq, nk, 0.0 * nq, 0.0 * nk
    size_q, size_k = size_q + np.abs(nq), size_k + np.abs(nk)
    # a binary32 sum of dim squares under a root (half its error), sine and cosine of a binary32 fraction of a turn and a few
    # roundings: under 2^-20 + dim 2^-25 of what went in; then one rounding to the type, whose smallest step is 2^-25 twice in binary16
    part = 2.0 ** -20 + dim * 2.0 ** -25

    def close(got, want, size):
        assert np.all(np.abs(f64(got) - want) <= EPS[dtype] / 2 * np.abs(want) + part * size + 2.0 ** -25)
    where_k, written = k0, np.zeros(k0.shape, dtype=bool)
    size_kc, want_vc, v64 = np.zeros_like(k0), v0, f64(v)
    for t, (b, p) in enumerate(batch.places()):
        page = batch.table[b, p // batch.page] if p >= 0 else -1
        if 0 <= page < batch.pages:
            at = (page, slice(None), p % batch.page)
            where_k[at], size_kc[at], want_vc[at], written[at] = want_k[t], size_k[t], v64[t], True
    if with_q:
        close(q_out, want_q, size_q)
    close(kc, where_k, size_kc)
    assert np.array_equal(f64(kc)[~written], where_k[~written])
    assert np.array_equal(f64(vc), want_vc)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (64, 64), (64, 32), (80, 20), (8, 2), (96, 0), (256, 256), (40, 38), (96, 96), (72, 16),
                                     (104, 104), (200, 64), (256, 6), (16, 16), (24, 8), (120, 48)])
def test_layouts_and_parts_of_a_head(dtype, interleaved, dim, rot):
    run(Batch([3, 1, 5], [20, 1, 5], 4), 4, 2, dim, rot, interleaved, TYPES[dtype], fused=True, token_major=dim == 80, each=dim == 64,
        offset=1.0 if dim == 80 else 0.0)


@pytest.mark.parametrize("heads", [(1, 1), (32, 32), (64, 8), (7, 1), (40, 40)])
@pytest.mark.parametrize("new,kv,page", [([1], [1], 16), ([1], [1000], 16), ([300], [300], 64), ([1] * 70, list(range(1, 71)), 8),
                                         ([0, 3, 0, 0, 2, 0], [5, 3, 0, 7, 9, 0], 1)])
def test_batches(heads, new, kv, page):
    run(Batch(new, kv, page, spare=1), heads[0], heads[1], 128, 64, False, torch.float16)


def test_a_long_prompt():
    run(Batch([2048], [2048], 64), 16, 2, 128, 128, False, torch.bfloat16, each=True)


def test_positions_of_their_own_and_far_ones():
    batch = Batch([4, 4], [9, 4], 8)
    run(batch, 4, 4, 128, 128, False, torch.float16, positions=np.array([0, 1, 131071, 1000003, -5, 2 ** 31 - 1, 77, 2 ** 30]))
    run(batch, 4, 4, 128, 128, True, torch.bfloat16, positions=np.arange(8) + 10 ** 6, amplitude=1.2772588722239782)


def test_the_prefix_counts_in_the_position():
    run(Batch([2, 1], [9, 4], 8, prefix=37), 4, 2, 64, 64, False, torch.float16)


def test_keys_and_values_only():
    run(Batch([2, 1], [9, 4], 8), 4, 2, 64, 64, False, torch.float16, with_q=False, each=True)


@pytest.mark.parametrize("size,eps", [(1e-6, 1e-6), (1e-6, 0.0), (2000.0, 1e-5), (1e-3, 1.0)])
def test_magnitudes_binary16(size, eps):
    run(Batch([5], [5], 8), 4, 2, 128, 128, False, torch.float16, size=size, eps=eps)


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e18, 1e22, 1e37])
@pytest.mark.parametrize("interleaved", [False, True])
def test_magnitudes_bfloat16(size, interleaved):
    """Squares of these values leave binary32, the norm does not."""
    run(Batch([5], [5], 8), 4, 2, 128, 128, interleaved, torch.bfloat16, size=size, eps=0.0)
    run(Batch([5], [5], 8), 4, 2, 80, 20, interleaved, torch.bfloat16, size=size, eps=1e-6)


def test_heads_of_zeros_are_zeros():
    dtype, cache = torch.float16, [torch.full((2, 2, 4, 64), 5.0, dtype=torch.float16, device=DEV) for _ in range(2)]
    batch = Batch([3], [3], 4, spare=1)
    z = torch.zeros((3, 2, 64), dtype=dtype, device=DEV)
    out = torch.full_like(z, 9.0)
    w = torch.ones(64, dtype=dtype, device=DEV)
    fq.fq_kv_append_normed(fq.KVCache(*cache), batch.sequences(), z, z, z, out, None, w, w)
    assert torch.all(out == 0) and int((cache[0] == 0).sum()) == 3 * 2 * 64


def test_values_that_are_not_finite_stay_in_their_heads():
    batch = Batch([4], [4], 4)
    gen = torch.Generator().manual_seed(3)
    for bad in (float("inf"), float("nan")):
        outs = []
        for spoil in (False, True):
            kc, vc = (pool(torch.Generator().manual_seed(1), batch.pages, 2, 4, 64, torch.float16) for _ in range(2))
            q = torch.randn((4, 4, 64), generator=gen.manual_seed(4)).half().to(DEV)
            k = torch.randn((4, 2, 64), generator=gen.manual_seed(5)).half().to(DEV)
            if spoil:
                q[1, 2, 7], k[2, 1, 9] = bad, bad
            out = torch.empty_like(q)
            w = torch.ones(64, dtype=torch.float16, device=DEV)
            fq.fq_kv_append_normed(fq.KVCache(kc, vc), batch.sequences(), q, k, k, out, torch.tensor(fq.fq_rope_freqs(64, 1e4), dtype=torch.float64, device=DEV), w, w)
            torch.cuda.synchronize()
            outs.append((out, kc[int(batch.table[0, 0])]))
        (o, c), (o2, c2) = outs
        assert torch.all(torch.isnan(o2[1, 2]) | (o2[1, 2] == 0)) and torch.any(torch.isnan(o2[1, 2]))
        assert torch.any(torch.isnan(c2[1, 2]))
        o2[1, 2], c2[1, 2] = o[1, 2], c[1, 2]
        assert torch.equal(o, o2) and torch.equal(c, c2)


@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1, None])
def test_bad_pages_are_not_written(bad):
    batch = Batch([5, 6], [13, 6], 4)
    batch.table[0, 2] = batch.pages if bad is None else bad
    batch.table[1, 0] = batch.pages + 1 if bad is None else bad
    run(batch, 4, 2, 64, 64, False, torch.float16)


def test_tables_and_caches_that_are_not_on_the_device_are_refused():
    dtype, gen = torch.float16, torch.Generator().manual_seed(1)
    kc, vc = (pool(gen, 4, 2, 8, 64, dtype) for _ in range(2))
    k, w = torch.randn((3, 2, 64), generator=gen).to(dtype).to(DEV), torch.ones(64, dtype=dtype, device=DEV)
    tables = [torch.tensor(v, dtype=torch.int32) for v in ([0, 3], [3], [[0, 1]])]
    near, far = fq.Sequences(*(t.to(DEV) for t in tables)), fq.Sequences(*tables)
    for cache, seqs, weight in ((fq.KVCache(kc.cpu(), vc.cpu()), near, w), (fq.KVCache(kc, vc), far, w), (fq.KVCache(kc, vc), near, w.cpu())):
        with pytest.raises(ValueError):
            fq.fq_kv_append_normed(cache, seqs, None, k, k, None, None, None, weight)


def test_more_new_tokens_than_length_have_no_place():
    run(Batch([6], [4], 4), 4, 2, 64, 64, False, torch.float16)


def test_rows_that_no_sequence_owns_stay():
    dtype, gen = torch.float16, torch.Generator().manual_seed(1)
    kc, vc = (pool(gen, 4, 2, 8, 64, dtype) for _ in range(2))
    k0 = kc.clone()
    k = torch.randn((6, 2, 64), generator=gen).to(dtype).to(DEV)
    q_out = torch.full((6, 2, 64), 9.0, dtype=dtype, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    w = torch.ones(64, dtype=dtype, device=DEV)
    # rows 0 and 1 belong to nobody, the second sequence ends past the rows, its length past its pages
    seqs = fq.Sequences(torch.tensor([2, 4, 99], **i32), torch.tensor([-7, 1000], **i32), torch.tensor([[0, 1], [2, 3]], **i32))
    freqs = torch.tensor(fq.fq_rope_freqs(64, 10000.0), dtype=torch.float64, device=DEV)
    fq.fq_kv_append_normed(fq.KVCache(kc, vc), seqs, k, k, k, q_out, freqs, w, w)
    torch.cuda.synchronize()
    assert torch.all(q_out[:2] == 9.0) and not torch.any(q_out[2:] == 9.0)
    want, _ = turn(normed(f64(k)[4:], 1.0, 1e-6, 0.0), np.array([14, 15]), freqs.cpu().numpy(), 64, False)
    assert np.abs(f64(kc)[3, :, 6:].transpose(1, 0, 2) - want).max() < 2e-3 * np.abs(want).max()
    assert torch.equal(kc[:3], k0[:3]) and torch.equal(kc[3, :, :6], k0[3, :, :6])


def test_with_unit_weights_of_normed_heads_it_is_the_plain_append():
    """Heads whose mean square is 1 exactly, eps 0: both calls turn the same values."""
    batch = Batch([7, 2], [30, 2], 8)
    gen = torch.Generator().manual_seed(2)
    sign = lambda *shape: (2.0 * torch.randint(0, 2, shape, generator=gen) - 1.0).half().to(DEV)  # noqa: E731
    q, k = sign(9, 4, 64), sign(9, 2, 64)
    w = torch.ones(64, dtype=torch.float16, device=DEV)
    freqs = torch.tensor(fq.fq_rope_freqs(64, 10000.0), dtype=torch.float64, device=DEV)
    got = []
    for call in (fq.fq_kv_append, fq.fq_kv_append_normed):
        kc, vc = (pool(torch.Generator().manual_seed(1), batch.pages, 2, 8, 64, torch.float16) for _ in range(2))
        out = torch.empty_like(q)
        call(fq.KVCache(kc, vc), batch.sequences(), q, k, k, out, freqs, *(() if call is fq.fq_kv_append else (w, w, 0.0)))
        got.append((out, kc, vc))
    # (the square root of 1 and the products with it are exact)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_captured_step_follows_the_tables():
    dtype, gen = torch.bfloat16, torch.Generator().manual_seed(2)
    batch = Batch([1, 1], [20, 20], 4)
    kc, vc = (pool(gen, batch.pages, 2, 4, 64, dtype) for _ in range(2))
    cache = fq.KVCache(kc, vc)
    q = torch.randn((2, 4, 64), generator=gen).to(dtype).to(DEV)
    k = torch.randn((2, 2, 64), generator=gen).to(dtype).to(DEV)
    w = torch.rand(64, generator=gen).to(dtype).to(DEV)
    freqs = torch.tensor(fq.fq_rope_freqs(64, 10000.0), dtype=torch.float64, device=DEV)
    seqs = batch.sequences()
    kv_len = seqs._keep[1]
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        fq.fq_kv_append_normed(cache, seqs, q, k, k, out, freqs, w, w)
    for step in range(1, 5):
        kv_len.copy_(torch.tensor([3 * step, 5 * step - 4], dtype=torch.int32))
        q.add_(0.25)
        w.mul_(0.5)
        g.replay()
        torch.cuda.synchronize()
        got = [out.clone(), kc.clone(), vc.clone()]
        kc.zero_(), vc.zero_(), out.zero_()
        fq.fq_kv_append_normed(cache, seqs, q, k, k, out, freqs, w, w)
        torch.cuda.synchronize()
        assert torch.equal(got[0], out)
        for t, (b, p) in enumerate(zip((0, 1), (3 * step - 1, 5 * step - 5))):
            page = int(batch.table[b, p // 4])
            assert torch.equal(got[1][page, :, p % 4], kc[page, :, p % 4]) and torch.any(kc[page, :, p % 4] != 0)
            assert torch.equal(got[2][page, :, p % 4], k[t])
