"""fq_adapters_add at the ends of its numbers: infinities of B, sums beyond the types, scales of any size."""
import numpy as np
import pytest
import torch

from serve_util import TYPES
from test_gpu_adapters import DEV, add, check, f64, want

pytestmark = pytest.mark.gpu


def device(*tensors):
    return [t.to(DEV) for t in tensors]


@pytest.mark.parametrize("M,rank", [(5, 8), (5, 32), (5, 64), (300, 8), (300, 64), (300, 136)])
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("N", [40, 41])
def test_an_infinity_of_b_is_one_of_the_result(M, rank, dtype, N):
    """u B with an infinite value of B is the infinity of the product's sign, whatever digits u has; beside 0 or the other infinity NaN."""
    dtype = TYPES[dtype]
    gen = torch.Generator().manual_seed(3)
    a, b = torch.rand((1, rank, 16), generator=gen).to(dtype) + 0.25, torch.randn((1, N, rank), generator=gen).to(dtype)
    x, y = torch.rand((M, 16), generator=gen).to(dtype) + 0.25, torch.randn((M, N), generator=gen).to(dtype)
    a[0, 1], x[1] = 1.0, 1.0  # (row 1, rank 1: 16 exactly)
    x[2] = -x[2]
    x[3] = 0.0
    clean = add(*device(a, b, x, y), None, None, np.zeros(M, np.int32))
    inf = float("inf")
    b[0, 5, rank - 1], b[0, 17, 1], b[0, 30, 0] = inf, -inf, float("nan")
    b[0, 39, 0], b[0, 39, 1] = inf, -inf
    got, here = add(*device(a, b, x, y), None, None, np.zeros(M, np.int32)), y.to(DEV)
    add(*device(a, b, x), here, None, None, np.zeros(M, np.int32), out=here)
    assert torch.equal(here.view(torch.int16), got.view(torch.int16))
    sign = torch.ones(M, device=DEV)
    sign[2] = -1.0
    rows = [m for m in range(M) if m != 3]
    assert torch.equal(got[rows, 5].float(), (inf * sign)[rows]) and torch.equal(got[rows, 17].float(), (-inf * sign)[rows])
    assert torch.all(torch.isnan(got[:, [30, 39]])) and torch.all(torch.isnan(got[3, [5, 17]]))
    other = [n for n in range(N) if n not in (5, 17, 30, 39)]
    assert torch.equal(got[:, other], clean[:, other])


@pytest.mark.parametrize("M", [2, 300])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_sums_beyond_the_largest_bfloat16_are_numbers(M, sign):
    """x A^T between the largest bfloat16 and the largest binary32, and a scale that brings it back."""
    dtype = torch.bfloat16
    a, b, x = torch.zeros((1, 8, 8)), torch.zeros((1, 12, 8)), torch.zeros((M, 8))
    x[:, 0], a[0, 0, 0] = sign * 1.9921875 * 2.0 ** 64, 2.0 ** 63
    x[:, 1], a[0, 0, 1] = sign * 1.5 * 2.0 ** 60, 2.0 ** 59  # u = 2^127 (255 / 128 + 3 / 512)
    b[0, :, 0] = 1.0
    scales, y, adapter = np.array([2.0 ** -120], dtype=np.float32), torch.zeros((M, 12)), np.zeros(M, np.int32)
    a, b, x, y = (t.to(dtype) for t in (a, b, x, y))
    got = add(*device(a, b, x, y), None, scales, adapter)
    check(got, *want(f64(x), f64(y), f64(a), f64(b), adapter, [8], scales.astype(np.float64)), dtype)


@pytest.mark.parametrize("M", [2, 300])
@pytest.mark.parametrize("scale", [2.0 ** 100, -2.0 ** 127, 2.0 ** -140])
def test_scales_of_any_size_beside_sums_of_any_size(M, scale):
    """The power of two that a row's x A^T is held by does not take a finite scale out of binary32: a product of 0 stays 0."""
    a, b, x = torch.full((1, 8, 512), 2.0 ** 15), torch.zeros((1, 12, 8)), torch.full((M, 512), 2.0 ** 15)
    b[0, 6:] = 1.0
    y = torch.randn((M, 12), generator=torch.Generator().manual_seed(1))
    a, b, x, y = (t.half() for t in (a, b, x, y))
    got = add(*device(a, b, x, y), None, np.array([scale], dtype=np.float32), np.zeros(M, np.int32)).cpu()
    assert torch.equal(got[:, :6], y[:, :6])
    assert torch.equal(got[:, 6:], y[:, 6:]) if abs(scale) < 1.0 else torch.all(got[:, 6:] == scale * float("inf"))
