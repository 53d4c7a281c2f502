"""fq_attend at the ends of its arithmetic, against the same 64-bit reference: scores of any size, weights of any size."""
import math

import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq
from serve_util import EPS, TYPES, Batch, attend, pool
from test_gpu_attend import call, check, f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("new,prefix", [([1, 1, 1], 0), ([1, 2, 1], 100), ([40], 0), ([150, 9], 70)])
@pytest.mark.parametrize("scale", [1.0, -0.37, 300.0])
def test_equal_largest_scores_of_any_size(dtype, dim, new, prefix, scale):
    """Scores that are exact in binary32 (one product), from 10^5 to 10^12: the largest ones of a row are equal and share
    its weight, everything else is further down than any weight reaches."""
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
    out, lse, _ = call(batch, fq.KVCache(kc, vc), q, scale)
    torch.cuda.synchronize()
    want, want_lse, size, _, _ = attend(batch, f64(q), f64(kc), f64(vc), float(np.float32(scale)))
    # the scores are exact and equal, so are their weights: the roundings of these (binary32, then the type) and of the result
    half = EPS[TYPES[dtype]] / 2
    tol = half * (1 + half) * (np.abs(want) + size) + 2.0 ** -20 * size + 2.0 ** -25
    share = np.abs(f64(out) - want) / tol
    assert np.all(share <= 1), "off by %g of the tolerance at %s" % (share.max(), np.unravel_index(share.argmax(), share.shape))
    assert np.all(np.abs(f64(lse) - want_lse) <= 32 * 2.0 ** -24 * (1 + np.abs(want_lse)))


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
