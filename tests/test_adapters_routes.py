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
