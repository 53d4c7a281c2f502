"""Which launches fq_adapters_add takes, a choice of the host that needs no device."""
import ctypes

import pytest

import paper_2506_12024_amd as fq


class _View(ctypes.Structure):  # FqAdaptersView
    _fields_ = ([("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("a_stride", ctypes.c_longlong), ("b_stride", ctypes.c_longlong),
                 ("ranks", ctypes.c_void_p), ("scales", ctypes.c_void_p)] + [(n, ctypes.c_int) for n in ("slots", "rank", "K", "N", "bf16")])


class _Route(ctypes.Structure):  # FqAdaptersRoute
    _fields_ = [(n, ctypes.c_int) for n in ("few", "listed", "workgroups", "out_tiles")]


_route = fq.lib["_Z17fq_adapters_routeRK14FqAdaptersViewi"]
_route.restype, _route.argtypes = _Route, [ctypes.c_void_p, ctypes.c_int]


def route(M, K, N, slots, rank):
    v = _View(slots=slots, rank=rank, K=K, N=N)
    r = _route(ctypes.byref(v), M)
    return r.few, r.listed, r.workgroups, r.out_tiles


@pytest.mark.parametrize("rank", [16, 32, 64])
def test_few_rows_take_no_more_workgroups_than_compute_units(rank):
    """A unit that has two workgroups takes twice as long."""
    for M in range(1, 65):
        for N in (64, 4096, 11008, 28672):
            few, _, groups, _ = route(M, (1 << 17) // rank, N, 64, rank)
            assert few and M <= groups <= 256, (M, N)


@pytest.mark.parametrize("rank", [64, 128])
def test_a_tile_is_on_one_chiplet_only_where_that_pays(rank):
    """Eight tiles to a row of the grid, and all of a tile's workgroups meet on one of eight chiplets: for wide outputs not by chance."""
    for M in (8, 16, 24, 32, 64, 200, 512, 1000, 4096):
        for slots in (7, 15, 16, 31, 64, 300):
            for N in (4096, 6144, 8192, 11008):
                few, _, _, tiles = route(M, 8192, N, slots, rank)
                most = M // 64 + min(M, slots + 1)
                assert not few and most <= tiles < most + 8
                assert tiles % 8 == 0 if N <= 6144 else tiles % 2 == 1, (M, slots, N)


@pytest.mark.parametrize("K,N,rank", [(5120, 5120, 32), (5120, 13824, 32), (3200, 4096, 64)])
def test_decode_batches_of_many_slots_are_one_launch(K, N, rank):
    """A and a tile's x together up to 2^18 values: sets whose slots may give most rows a tile of their own."""
    for M, slots in ((16, 16), (24, 64), (32, 16), (32, 32), (32, 64), (40, 1000), (64, 32), (64, 64)):
        assert route(M, K, N, slots, rank)[0], (M, slots)
    for M, slots in ((1, 64), (8, 64), (32, 8), (64, 8), (64, 31)):
        assert not route(M, K, N, slots, rank)[0], (M, slots)


@pytest.mark.parametrize("K,rank", [(11008, 16), (14336, 16), (8192, 32), (4096, 64)])
def test_decode_batches_of_nearly_as_many_slots_as_rows_are_one_launch(K, rank):
    """Up to 2^18 values of A."""
    for M, slots in ((28, 28), (32, 32), (32, 1000), (40, 32), (64, 52), (64, 64)):
        assert route(M, K, 4096, slots, rank)[0], (M, slots)
        assert route(M, K, 8192, slots, rank)[0] == (min(M, slots) >= 40), (M, slots)
    for M, slots in ((1, 64), (16, 64), (27, 64), (32, 16), (64, 32), (64, 51)):
        assert not route(M, K, 4096, slots, rank)[0], (M, slots)


@pytest.mark.parametrize("M,K,N,rank,slots,few", [
    (16, 5456, 4096, 32, 16, 1), (16, 5464, 4096, 32, 16, 0), (32, 5456, 9000, 32, 16, 1), (33, 5456, 4096, 32, 16, 0), (15, 5456, 9000, 32, 64, 0),
    (28, 8192, 6144, 32, 28, 1), (39, 8192, 6145, 32, 64, 0), (40, 8192, 6145, 32, 40, 1), (64, 8200, 4096, 32, 64, 0),
    (1, 8192, 4096, 16, 1, 1), (64, 4096, 4096, 32, 8, 1), (256, 4096, 4096, 16, 64, 1), (257, 4096, 4096, 16, 64, 0), (1, 64, 4096, 72, 1, 0)])
def test_where_one_launch_ends(M, K, N, rank, slots, few):
    assert route(M, K, N, slots, rank)[0] == few


@pytest.mark.parametrize("M,K,N,slots,rank,listed", [
    (701, 11008, 4096, 12, 16, 0), (2048, 8192, 8192, 4, 64, 0), (300, 4096, 4096, 32, 16, 0), (4096, 4096, 4096, 64, 16, 0), (10, 4096, 4096, 1000, 128, 0),
    # sets of many slots, of which a call may name a few: most workgroups have no tile
    (701, 4096, 4096, 1000, 16, 1), (257, 4096, 4096, 300, 16, 1), (257, 4096, 1024, 300, 256, 1), (4096, 4096, 4096, 1000, 16, 1), (100, 4096, 4096, 64, 256, 1),
    (2048, 4096, 4096, 300, 16, 1), (64, 4096, 4096, 1000, 128, 1), (4097, 64, 64, 1, 16, 1), (300, 64, 64, 1024, 16, 1)])
def test_many_workgroups_find_their_rows_in_a_list(M, K, N, slots, rank, listed):
    assert route(M, K, N, slots, rank)[:2] == (0, listed)
