"""fq_adapters_add by more rows than one launch takes: what test_gpu_adapters.py asks of few rows, of the routes of several launches."""
import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq
from serve_util import TYPES
from test_gpu_adapters import add, check, data, f64, want

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16 = torch.float16
# M, K, N, slots, rank: rows counted by every workgroup, parts of x A^T added by every workgroup of the last launch; the same where rows of y are not
# aligned to 8 bytes; parts added by a launch of their own, for ranks up to 64 and beyond; rows sorted by a launch of their own, of sets of many slots and in calls
# whose set and rank give many workgroups
ROUTES = {"all_add": (300, 136, 72, 4, 16), "odd": (300, 264, 61, 5, 24), "join_64": (300, 4096, 5504, 4, 64), "join_136": (300, 2056, 72, 4, 136),
          "sorted": (300, 136, 72, 1100, 16), "many_rows": (4200, 72, 40, 6, 32),
          "sorted_few": (64, 4096, 72, 64, 128)}
routes = pytest.mark.parametrize("route", sorted(ROUTES))


def device(*tensors):
    return [t.to(DEV) for t in tensors]


@routes
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_ranks_and_what_lies_beyond_them(route, dtype):
    """Rows of A and columns of B behind a slot's rank, and a slot that no row names, hold NaNs and infinities."""
    M, K, N, slots, rank = ROUTES[route]
    a, b, x, y, _, scales, adapter = data(M, K, N, slots, rank, TYPES[dtype], ranks=[0] * slots)
    adapter = np.where(adapter == slots - 1, 0, adapter).astype(np.int32)
    ranks = [(rank, 1, rank - 1, rank + 99, 0, rank // 2 + 1, -5)[s % 7] for s in range(slots)]
    held = [min(max(r, 0), rank) for r in ranks]
    for s in range(slots):
        a[s, held[s]:] = float("nan")
        b[s, :, held[s]:] = float("inf") if s % 2 else float("nan")
    a[slots - 1], b[slots - 1] = float("nan"), float("nan")
    got = add(*device(a, b, x, y), ranks, scales, adapter)
    check(got, *want(f64(x), f64(y), np.nan_to_num(f64(a)), np.nan_to_num(f64(b), posinf=0.0), adapter, held, scales.astype(np.float64)), TYPES[dtype])


@routes
def test_rows_without_an_adapter_keep_their_bits(route):
    M, K, N, slots, rank = ROUTES[route]
    a, b, x, y, ranks, scales, adapter = data(M, K, N, slots, rank, F16)
    ranks[1] = 0
    adapter[::2] = [(-1, slots, 1, 2 ** 31 - 1, -2 ** 31)[i % 5] for i in range(len(adapter[::2]))]
    y.view(torch.int16)[::2] = torch.randint(-2 ** 15, 2 ** 15, y[::2].shape, dtype=torch.int16)  # NaNs of all kinds among them
    ref = want(f64(x)[1::2], f64(y)[1::2], f64(a), f64(b), adapter[1::2], ranks, scales.astype(np.float64))
    here = y.to(DEV)
    for out in (None, here):
        got = add(a.to(DEV), b.to(DEV), x.to(DEV), here, ranks, scales, adapter, out=out)
        assert torch.equal(got[::2].view(torch.int16).cpu(), y[::2].view(torch.int16))
        check(got[1::2], *ref, F16)


@routes
@pytest.mark.parametrize("pad,lead", [(0, 0), (1, 1), (4, 4), (24, 8)])
def test_rows_that_lie_apart_and_in_place(route, pad, lead):
    M, K, N, slots, rank = ROUTES[route]
    a, b, x, y, ranks, scales, adapter = data(M, K, N, slots, rank, F16)
    ref = want(f64(x), f64(y), f64(a), f64(b), adapter, ranks, scales.astype(np.float64))
    wide_x = torch.full((M, K + 16), float("nan"), dtype=F16, device=DEV)
    wide_x[:, 8:8 + K] = x.to(DEV)
    row = torch.full((M, N + lead + pad), 7.0, dtype=F16, device=DEV)
    here = row[:, lead:lead + N]
    here.copy_(y)
    add(a.to(DEV), b.to(DEV), wide_x[:, 8:8 + K], here, ranks, scales, adapter, out=here)
    check(here, *ref, F16)
    out = torch.full((M, N + lead + pad), 7.0, dtype=F16, device=DEV)
    add(a.to(DEV), b.to(DEV), wide_x[:, 8:8 + K], y.to(DEV), ranks, scales, adapter, out=out[:, lead:lead + N])
    assert torch.equal(out[:, lead:lead + N], here)
    for t in (row, out):
        assert torch.all(t[:, :lead] == 7.0) and torch.all(t[:, lead + N:] == 7.0)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("M", [1, 7, 40, 64, 100, 256])
def test_few_rows_in_place(M, dtype):
    """The main use: y and out are one tensor whose rows are aligned."""
    a, b, x, y, ranks, scales, adapter = data(M, 264, 136, 5, 16, TYPES[dtype], seed=M)
    here = y.to(DEV)
    add(a.to(DEV), b.to(DEV), x.to(DEV), here, ranks, scales, adapter, out=here)
    check(here, *want(f64(x), f64(y), f64(a), f64(b), adapter, ranks, scales.astype(np.float64)), TYPES[dtype])


@routes
def test_slots_that_lie_apart_without_ranks_or_scales(route):
    M, K, N, slots, rank = ROUTES[route]
    dtype = torch.bfloat16
    a, b, x, y, _, _, adapter = data(M, K, N, slots, rank, dtype)
    wide_a, wide_b = torch.full((slots, rank + 4, K), 5.0, dtype=dtype, device=DEV), torch.full((slots, N + 1, rank), 5.0, dtype=dtype, device=DEV)
    wide_a[:, 2:rank + 2], wide_b[:, 1:] = a.to(DEV), b.to(DEV)
    got = add(wide_a[:, 2:rank + 2], wide_b[:, 1:], x.to(DEV), y.to(DEV), None, None, adapter)
    check(got, *want(f64(x), f64(y), f64(a), f64(b), adapter, [rank] * slots, np.ones(slots)), dtype)


@routes
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("power", [-12, 8])
def test_sums_outside_binary16(route, dtype, power):
    """x A^T of 2^20 and more, or of 2^-26 and less in most ranks beside a large one, and B that brings it back."""
    M, K, N, slots, rank = ROUTES[route]
    dtype = TYPES[dtype]
    a, b, x, y, ranks, scales, adapter = data(M, K, N, slots, rank, dtype, spare=False)
    a = (a.double() * 2.0 ** power).to(dtype)
    if power > 0:
        x, b = (x.double() * 2.0 ** 10).to(dtype), (b.double() * 2.0 ** -14).to(dtype)
    else:
        a[:, 0] = 8.0
        b[:, :, 0] = (b[:, :, 0].double() * 2.0 ** -12).to(dtype)
    got = add(*device(a, b, x, y), ranks, scales, adapter)
    check(got, *want(f64(x), f64(y), f64(a), f64(b), adapter, ranks, scales.astype(np.float64)), dtype)


@routes
def test_values_that_are_not_finite_stay_in_their_rows(route):
    M, K, N, slots, rank = ROUTES[route]
    a, b, x, y, _, scales, adapter = data(M, K, N, slots, rank, F16, spare=False)
    ranks, scales = [rank] * slots, np.abs(scales)
    clean = add(*device(a, b, x, y), ranks, scales, adapter)
    x[3, 5], x[7, 9], y[9, 2] = float("inf"), float("nan"), float("-inf")
    got = add(*device(a, b, x, y), ranks, scales, adapter)
    other = [m for m in range(M) if m not in (3, 7, 9)]
    assert torch.equal(got[other], clean[other])
    assert torch.all(torch.isnan(got[7])) and not torch.any(torch.isfinite(got[3]))
    assert got[9, 2] == float("-inf") and torch.equal(got[9, 3:], clean[9, 3:])


@routes
def test_a_captured_call_follows_adapters_and_slots(route):
    M, K, N, slots, rank = ROUTES[route]
    a, b, x, y, ranks, scales, adapter = data(M, K, N, slots, rank, F16)
    a, b, x, y, scales, adapter = device(a, b, x, y, torch.from_numpy(scales), torch.from_numpy(adapter))
    ranks = torch.tensor(ranks, dtype=torch.int32).to(DEV)
    h = fq.Adapters(a, b, ranks, scales)
    ws = torch.empty(fq.fq_adapters_workspace_bytes(h, M), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        fq.fq_adapters_add(h, x, adapter, y, out, ws)
    gen = torch.Generator(device=DEV).manual_seed(5)
    for step in range(4):
        adapter.copy_(torch.randint(-1, slots, (M,), generator=gen, device=DEV))
        ranks.copy_(torch.randint(0, rank + 1, (slots,), generator=gen, device=DEV))
        a.copy_(a.roll(1, 0))
        x.mul_(-0.5)
        out.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        ws.fill_(step)
        out.fill_(3.0)
        fq.fq_adapters_add(h, x, adapter, y, out, ws)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.any(got != y)


@routes
def test_equal_calls_give_equal_bits_wherever_rows_stand(route):
    M, K, N, slots, rank = ROUTES[route]
    a, b, x, y, ranks, scales, adapter = data(M, K, N, slots, rank, F16)
    one = add(*device(a, b, x, y), ranks, scales, adapter)
    assert torch.equal(add(*device(a, b, x, y), ranks, scales, adapter), one)
    order = np.random.default_rng(1).permutation(M)
    two = add(*device(a, b, x[order], y[order]), ranks, scales, adapter[order])
    assert torch.equal(one[torch.from_numpy(order).to(DEV)], two)


def test_workspaces_of_larger_calls_and_rows_behind_the_last():
    """Every call writes its rows and no other ones, in the workspace of the largest."""
    a, b, x, y, ranks, scales, adapter = data(700, 520, 72, 4, 40, F16)
    ref = want(f64(x), f64(y), f64(a), f64(b), adapter, ranks, scales.astype(np.float64))
    a, b, x, y, scales, who = device(a, b, x, y, torch.from_numpy(scales), torch.from_numpy(adapter))
    h = fq.Adapters(a, b, torch.tensor(ranks, dtype=torch.int32).to(DEV), scales)
    ws = torch.full((fq.fq_adapters_workspace_bytes(h, 700),), 255, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(y)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for M in (700, 699, 300, 257, 256, 200, 199, 65, 64, 3, 1, 0):
            out.fill_(9.0)
            fq.fq_adapters_add(h, x[:M], who[:M], y[:M], out[:M], ws)
            s.synchronize()
            check(out[:M], ref[0][:M], ref[1][:M], F16)
            assert torch.all(out[M:] == 9.0), M


def test_two_streams_at_once():
    sets = [data(M, 264, 136, 4, 136, F16, seed=M) for M in (300, 301)]
    whole = [add(*device(*d[:4]), *d[4:]) for d in sets]
    streams, keep = [torch.cuda.Stream() for _ in sets], []
    for d in sets:
        h = fq.Adapters(*device(d[0], d[1], torch.tensor(d[4], dtype=torch.int32), torch.from_numpy(d[5])))
        keep.append((h, *device(d[2], torch.from_numpy(d[6]), d[3], torch.full_like(d[3], 9.0)),
                     torch.empty(fq.fq_adapters_workspace_bytes(h, d[2].shape[0]), dtype=torch.uint8, device=DEV)))
    torch.cuda.synchronize()
    for _ in range(10):
        for k, s in zip(keep, streams):
            fq.fq_adapters_add(*k, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(k[4], w) for k, w in zip(keep, whole))
