"""fq_adapters_add against a 64-bit reference: ranks, sizes, strides, rows without an adapter, contents that do not count, capture."""
import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq
from serve_util import EPS, TYPES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def f64(t):
    return t.double().cpu().numpy()


def want(x, y, a, b, adapter, ranks, scales):
    """(out, magnitude of what went into it, bound of the error apart from the last rounding), float64."""
    out, err = y.copy(), 2.0 ** -24 * np.abs(y)
    for m, s in enumerate(adapter):
        r = ranks[s] if 0 <= s < len(a) else 0
        if r <= 0:
            err[m] = 0.0
            continue
        A, B = a[s, :r], b[s][:, :r]
        low, size = A @ x[m], np.abs(A) @ np.abs(x[m])
        out[m] += scales[s] * (B @ low)
        # x A^T: K binary32 additions at most.  It enters the second product as two numbers of the type: 2^-17 of it, and of the
        # row's largest 2^-30 (binary16's smallest step); then 2 rank binary32 additions and a few roundings
        part = (len(x[m]) + 8) * 2.0 ** -24 * size + 2.0 ** -17 * np.abs(low) + 2.0 ** -30 * np.abs(low).max()
        err[m] += abs(scales[s]) * (np.abs(B) @ (part + (2 * r + 8) * 2.0 ** -24 * np.abs(low))) * (1 + 2.0 ** -10)
    return out, err


def check(got, ref, err, dtype):
    half = EPS[dtype] / 2
    tol = half * np.abs(ref) + (1 + half) * err + np.where(err > 0, 2.0 ** -25, 0.0)
    off = np.abs(f64(got) - ref)
    assert np.all(off <= tol), (off - tol).max()


def data(M, K, N, slots, rank, dtype, seed=0, ranks=None, spare=True):
    gen = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    a = (torch.randn((slots, rank, K), generator=gen) / K ** 0.5).to(dtype)
    b = torch.randn((slots, N, rank), generator=gen).to(dtype)
    x, y = torch.randn((M, K), generator=gen).to(dtype), torch.randn((M, N), generator=gen).to(dtype)
    if ranks is None:
        ranks = [rank] + [int(v) for v in rng.integers(0 if spare else 1, rank + 1, slots - 1)]
    scales = rng.uniform(-2.0, 2.0, slots).astype(np.float32)
    adapter = rng.integers(-1 if spare else 0, slots, M).astype(np.int32)
    return a, b, x, y, ranks, scales, adapter


def add(a, b, x, y, ranks, scales, adapter, out=None, workspace=None):
    h = fq.Adapters(a, b, None if ranks is None else torch.tensor(ranks, dtype=torch.int32).to(DEV),
                    None if scales is None else torch.from_numpy(scales).to(DEV))
    M = x.shape[0]
    need = fq.fq_adapters_workspace_bytes(h, M)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV) if workspace is None else workspace
    out = torch.full_like(y, 9.0) if out is None else out
    fq.fq_adapters_add(h, x, torch.from_numpy(adapter).to(DEV), y, out, ws[:need])
    torch.cuda.synchronize()
    assert torch.all(ws[need:] == 255)
    return out


def run(M, K, N, slots, rank, dtype, **kw):
    d = data(M, K, N, slots, rank, dtype, **kw)
    a, b, x, y, ranks, scales, adapter = d
    got = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, scales, adapter)
    check(got, *want(f64(x), f64(y), f64(a), f64(b), adapter, ranks, scales.astype(np.float64)), dtype)
    return d, got


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("M,K,N,slots,rank", [
    (1, 8, 1, 1, 8), (1, 4096, 4096, 2, 16), (3, 40, 17, 2, 8), (16, 512, 64, 1, 16), (17, 264, 65, 3, 24), (33, 1000, 130, 5, 32),
    (64, 128, 256, 40, 16), (65, 136, 72, 7, 16), (100, 256, 100, 3, 64), (300, 520, 200, 4, 40), (257, 64, 33, 300, 8),
    (5, 256, 72, 3, 256), (130, 104, 48, 2, 136), (700, 384, 320, 9, 128)])
def test_sizes(dtype, M, K, N, slots, rank):
    run(M, K, N, slots, rank, TYPES[dtype])


@pytest.mark.parametrize("M", [1, 2, 15, 16, 31, 32, 48, 63, 64, 66, 128, 129, 255, 256, 300, 1000, 2500])
def test_row_counts(M):
    run(M, 136, 72, 6, 16, torch.float16, seed=M)
    run(M, 136, 72, 6, 16, torch.float16, seed=M, spare=False)


@pytest.mark.parametrize("M,K,N,slots,rank", [(4095, 40, 24, 5, 8), (4097, 40, 24, 5, 8), (5000, 72, 33, 3, 40), (300, 64, 33, 1500, 8), (700, 264, 48, 1023, 16),
                                              (10, 40, 24, 3000, 72), (257, 8, 5, 16384, 8), (9000, 16, 12, 2, 256), (4200, 24, 8, 1200, 8)])
def test_many_rows_and_many_slots(M, K, N, slots, rank):
    run(M, K, N, slots, rank, torch.float16, seed=M)


@pytest.mark.parametrize("M,K,rank", [(3, 8192, 32), (40, 8200, 32), (40, 16392, 16), (66, 1000, 136), (70, 12, 8), (400, 2056, 24), (3, 264, 72)])
def test_long_sums_and_their_ends(M, K, rank):
    """K at and beside the ends of the pieces that the products take, in one launch and in several."""
    K = -(-K // 8) * 8
    run(M, K, 52, 3, rank, torch.bfloat16, seed=K)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("M,K,N,slots,rank", [(300, 4104, 200, 4, 128), (90, 4360, 72, 3, 256), (1500, 2304, 1100, 5, 32), (520, 1544, 6200, 7, 64), (600, 520, 6148, 3, 48),
                                              (70, 1288, 260, 3, 8), (90, 2056, 132, 20, 40), (1, 2304, 40, 2, 200), (64, 4096, 40, 64, 64), (1100, 768, 66, 3, 16)])
def test_parts_added_by_one_launch_or_by_all_workgroups(dtype, M, K, N, slots, rank):
    run(M, K, N, slots, rank, TYPES[dtype], seed=M)


@pytest.mark.parametrize("M", [16, 64, 100, 256])
@pytest.mark.parametrize("slots,K,N", [(1, 8192, 40), (2, 64, 16384), (33, 8200, 36), (70, 256, 8200)])
def test_sets_of_few_and_of_many_slots(M, slots, K, N):
    run(M, K, N, slots, 16, torch.float16, seed=M)


def test_a_prompt_beside_single_tokens():
    """Rows of one slot side by side and apart, tiles that end between them, rows of none among them."""
    a, b, x, y, ranks, scales, _ = data(1000, 136, 72, 6, 24, torch.float16)
    adapter = np.concatenate([np.full(333, 2), np.full(130, -1), np.full(64, 0), np.arange(473) % 7 - 1]).astype(np.int32)
    got = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, scales, adapter)
    check(got, *want(f64(x), f64(y), f64(a), f64(b), adapter, ranks, scales.astype(np.float64)), torch.float16)


def test_rows_have_the_same_bits_wherever_they_stand():
    """A row's sums do not depend on the rows beside it, among calls of one shape."""
    for M in (40, 150, 700):
        a, b, x, y, ranks, scales, adapter = data(M, 520, 72, 4, 16, torch.float16)
        one = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, scales, adapter)
        order = np.random.default_rng(1).permutation(M)
        two = add(a.to(DEV), b.to(DEV), x[order].to(DEV), y[order].to(DEV), ranks, scales, adapter[order])
        assert torch.equal(one[torch.from_numpy(order).to(DEV)], two)


def test_two_streams_at_once():
    sets = [data(M, 264, 136, 4, 16, torch.float16, seed=M) for M in (300, 301)]
    whole = [add(d[0].to(DEV), d[1].to(DEV), d[2].to(DEV), d[3].to(DEV), *d[4:]) for d in sets]
    streams, outs, keep = [torch.cuda.Stream() for _ in sets], [], []
    for d, s in zip(sets, streams):
        h = fq.Adapters(d[0].to(DEV), d[1].to(DEV), torch.tensor(d[4], dtype=torch.int32).to(DEV), torch.from_numpy(d[5]).to(DEV))
        keep.append((h, d[2].to(DEV), torch.from_numpy(d[6]).to(DEV), d[3].to(DEV), torch.empty_like(d[3], device=DEV),
                     torch.empty(fq.fq_adapters_workspace_bytes(h, d[2].shape[0]), dtype=torch.uint8, device=DEV)))
    torch.cuda.synchronize()
    for _ in range(10):
        for k, s in zip(keep, streams):
            fq.fq_adapters_add(*k, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(k[4], w) for k, w in zip(keep, whole))


@pytest.mark.parametrize("ranks", [[16, 1], [1, 15], [0, 0], [7, 9], [-5, 99]])
def test_ranks_and_what_lies_beyond_them(ranks):
    """Rows of A and columns of B behind a slot's rank, and slots that no row names, hold NaNs."""
    dtype = torch.float16
    a, b, x, y, _, scales, adapter = data(40, 136, 72, 3, 16, dtype, ranks=[0, 0, 0])
    adapter = np.where(adapter == 2, 0, adapter).astype(np.int32)
    held = [min(max(r, 0), 16) for r in ranks] + [16]
    for s in range(2):
        a[s, held[s]:] = float("nan")
        b[s, :, held[s]:] = float("inf")
    a[2], b[2] = float("nan"), float("nan")
    got = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks + [16], scales, adapter)
    check(got, *want(f64(x), f64(y), np.nan_to_num(f64(a)), np.nan_to_num(f64(b), posinf=0.0), adapter, held, scales.astype(np.float64)), dtype)


def test_no_ranks_and_no_scales():
    a, b, x, y, _, _, adapter = data(20, 64, 48, 3, 8, torch.bfloat16)
    got = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), None, None, adapter)
    check(got, *want(f64(x), f64(y), f64(a), f64(b), adapter, [8] * 3, np.ones(3)), torch.bfloat16)


@pytest.mark.parametrize("M", [7, 90])
def test_rows_without_an_adapter_keep_their_bits(M):
    a, b, x, y, ranks, scales, adapter = data(M, 64, 50, 3, 8, torch.float16, ranks=[8, 3, 0])
    adapter[::2] = [(-1, 3, 2, 2 ** 31 - 1, -2 ** 31)[i % 5] for i in range(len(adapter[::2]))]
    y.view(torch.int16)[::2] = torch.randint(-2 ** 15, 2 ** 15, y[::2].shape, dtype=torch.int16)  # NaNs of all kinds among them
    got = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, scales, adapter)
    assert torch.equal(got[::2].view(torch.int16).cpu(), y[::2].view(torch.int16))
    odd = slice(1, None, 2)
    check(got[odd], *want(f64(x)[odd], f64(y)[odd], f64(a), f64(b), adapter[odd], ranks, scales.astype(np.float64)), torch.float16)


@pytest.mark.parametrize("M", [5, 200])
@pytest.mark.parametrize("pad,lead", [(0, 0), (1, 1), (8, 3), (24, 8)])
def test_rows_that_lie_apart_and_in_place(M, pad, lead):
    dtype, K, N = torch.float16, 72, 61
    a, b, x, y, ranks, scales, adapter = data(M, K, N, 4, 16, dtype)
    ref = want(f64(x), f64(y), f64(a), f64(b), adapter, ranks, scales.astype(np.float64))
    wide_x = torch.zeros((M, K + 16), dtype=dtype, device=DEV)
    wide_x[:, 8:8 + K] = x.to(DEV)
    row = torch.full((M, N + lead + pad), 7.0, dtype=dtype, device=DEV)
    here = row[:, lead:lead + N]
    here.copy_(y)
    add(a.to(DEV), b.to(DEV), wide_x[:, 8:8 + K], here, ranks, scales, adapter, out=here)
    check(here, *ref, dtype)
    assert torch.all(row[:, :lead] == 7.0) and torch.all(row[:, lead + N:] == 7.0)
    out = torch.full((M, N + lead + pad), 7.0, dtype=dtype, device=DEV)
    add(a.to(DEV), b.to(DEV), wide_x[:, 8:8 + K], y.to(DEV), ranks, scales, adapter, out=out[:, lead:lead + N])
    assert torch.equal(out[:, lead:lead + N], here)
    assert torch.all(out[:, :lead] == 7.0) and torch.all(out[:, lead + N:] == 7.0)


def test_one_row_in_place_has_no_stride():
    a, b, x, y, ranks, scales, adapter = data(1, 64, 40, 2, 8, torch.float16, spare=False)
    h = fq.Adapters(a.to(DEV), b.to(DEV), scales=torch.from_numpy(scales).to(DEV))
    one, who, x, y = torch.empty_like(y, device=DEV), torch.from_numpy(adapter).to(DEV), x.to(DEV), y.to(DEV)
    ws = torch.empty(fq.fq_adapters_workspace_bytes(h, 1), dtype=torch.uint8, device=DEV)
    fq.fq_adapters_add(h, x, who, y, one, ws)
    assert fq.lib.fq_adapters_add(h.handle, 1, x.data_ptr(), 64, who.data_ptr(), y.data_ptr(), 40, y.data_ptr(), 48, ws.data_ptr(), ws.numel(), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(one, y)


def test_tensors_that_are_not_on_the_device_are_refused():
    a, b, x, y, ranks, scales, adapter = data(3, 64, 40, 2, 8, torch.float16)
    h, far = fq.Adapters(a.to(DEV), b.to(DEV)), fq.Adapters(a, b)
    ws = torch.empty(fq.fq_adapters_workspace_bytes(h, 3), dtype=torch.uint8, device=DEV)
    good = [h, x.to(DEV), torch.from_numpy(adapter).to(DEV), y.to(DEV), torch.empty_like(y, device=DEV), ws]
    for i, bad in enumerate([far, x, torch.from_numpy(adapter), y, y, ws.cpu()]):
        with pytest.raises(ValueError):
            fq.fq_adapters_add(*good[:i], bad, *good[i + 1:])


def test_slots_that_lie_apart():
    dtype = torch.bfloat16
    a, b, x, y, ranks, scales, adapter = data(30, 64, 40, 3, 16, dtype)
    wide_a, wide_b = torch.full((3, 20, 64), 5.0, dtype=dtype, device=DEV), torch.full((3, 41, 16), 5.0, dtype=dtype, device=DEV)
    wide_a[:, 2:18], wide_b[:, 1:] = a.to(DEV), b.to(DEV)
    got = add(wide_a[:, 2:18], wide_b[:, 1:], x.to(DEV), y.to(DEV), ranks, scales, adapter)
    check(got, *want(f64(x), f64(y), f64(a), f64(b), adapter, ranks, scales.astype(np.float64)), dtype)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("M", [6, 150])
@pytest.mark.parametrize("power", [-12, 8])
def test_sums_outside_binary16(dtype, M, power):
    """x A^T of 2^20 and more, or of 2^-26 and less in most ranks beside a large one, and B that brings it back."""
    dtype = TYPES[dtype]
    a, b, x, y, ranks, scales, adapter = data(M, 512, 40, 2, 16, dtype, spare=False)
    a = (a.double() * 2.0 ** power).to(dtype)
    if power > 0:
        x, b = (x.double() * 2.0 ** 10).to(dtype), (b.double() * 2.0 ** -14).to(dtype)
    else:
        a[:, 0] = 8.0
        b[:, :, 0] = (b[:, :, 0].double() * 2.0 ** -12).to(dtype)
    got = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, scales, adapter)
    check(got, *want(f64(x), f64(y), f64(a), f64(b), adapter, ranks, scales.astype(np.float64)), dtype)


@pytest.mark.parametrize("M", [12, 180])
def test_values_that_are_not_finite_stay_in_their_rows(M):
    dtype = torch.float16
    a, b, x, y, ranks, scales, adapter = data(M, 64, 48, 2, 16, dtype, ranks=[16, 16], spare=False)
    clean = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, np.abs(scales), adapter)
    x[3, 5], x[7, 9], y[9, 2] = float("inf"), float("nan"), float("-inf")
    got = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, np.abs(scales), adapter)
    other = [m for m in range(M) if m not in (3, 7, 9)]
    assert torch.equal(got[other], clean[other])
    assert torch.all(torch.isnan(got[7])) and not torch.any(torch.isfinite(got[3]))
    assert got[9, 2] == float("-inf") and torch.equal(got[9, 3:], clean[9, 3:])


def test_an_infinite_sum_of_one_sign_is_infinite():
    """x A^T infinite in one rank alone, B of one sign there: the result is the infinity, not NaN."""
    a, b, x = torch.zeros((1, 8, 16)), torch.ones((1, 24, 8)), torch.ones((2, 16))
    a[0, 0, 0] = 1.0
    x[0, 0] = float("inf")
    x[0, 1:] = 0.0
    b[0, 12:, 0] = -2.0
    got = add(a.half().to(DEV), b.half().to(DEV), x.half().to(DEV), torch.zeros((2, 24)).half().to(DEV), None, None, np.zeros(2, np.int32))
    # (the other ranks of row 0 are 0 times the infinity, NaN: only a rank whose A is not 0 there is infinite)
    assert torch.all(torch.isnan(got[0])) and torch.equal(got[1].cpu(), torch.tensor([1.0] * 12 + [-2.0] * 12).half())
    a[0, :, 0] = 1.0
    got = add(a.half().to(DEV), b.half().to(DEV), x.half().to(DEV), torch.zeros((2, 24)).half().to(DEV), None, None, np.zeros(2, np.int32))
    assert torch.all(got[0, :12] == float("inf")) and torch.all(torch.isnan(got[0, 12:]))


def test_equal_calls_give_equal_bits():
    for M in (9, 400):
        a, b, x, y, ranks, scales, adapter = data(M, 256, 136, 5, 32, torch.float16)
        one = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, scales, adapter)
        for _ in range(3):
            assert torch.equal(add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, scales, adapter), one)


@pytest.mark.parametrize("M", [4, 150])
def test_a_captured_call_follows_adapters_and_slots(M):
    dtype = torch.float16
    a, b, x, y, ranks, scales, adapter = data(M, 136, 80, 4, 16, dtype)
    a, b, x, y = (t.to(DEV) for t in (a, b, x, y))
    ranks, scales, adapter = torch.tensor(ranks, dtype=torch.int32).to(DEV), torch.from_numpy(scales).to(DEV), torch.from_numpy(adapter).to(DEV)
    h = fq.Adapters(a, b, ranks, scales)
    ws = torch.empty(fq.fq_adapters_workspace_bytes(h, M), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        fq.fq_adapters_add(h, x, adapter, y, out, ws)
    gen = torch.Generator(device=DEV).manual_seed(5)
    for step in range(4):
        adapter.copy_(torch.randint(-1, 4, (M,), generator=gen, device=DEV))
        ranks.copy_(torch.randint(0, 17, (4,), generator=gen, device=DEV))
        a.copy_(a.roll(1, 0))
        x.mul_(-0.5)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.fill_(3.0)
        fq.fq_adapters_add(h, x, adapter, y, out, ws)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.any(got != y)


def test_on_another_stream_and_workspaces_of_larger_calls():
    a, b, x, y, ranks, scales, adapter = data(200, 136, 72, 4, 16, torch.float16)
    whole = add(a.to(DEV), b.to(DEV), x.to(DEV), y.to(DEV), ranks, scales, adapter)
    h = fq.Adapters(a.to(DEV), b.to(DEV), torch.tensor(ranks, dtype=torch.int32).to(DEV), torch.from_numpy(scales).to(DEV))
    ws = torch.empty(fq.fq_adapters_workspace_bytes(h, 200), dtype=torch.uint8, device=DEV)
    x, y, who = x.to(DEV), y.to(DEV), torch.from_numpy(adapter).to(DEV)
    out = torch.zeros_like(y)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for M in (200, 199, 65, 64, 3, 0):
        fq.fq_adapters_add(h, x[:M], who[:M], y[:M], out[:M], ws, stream=s)
        s.synchronize()
        assert torch.allclose(out[:M].float(), whole[:M].float(), rtol=2.0 ** -9, atol=2.0 ** -9)
