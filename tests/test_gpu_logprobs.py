"""fq_logprobs and fq_logprobs_f16 against 64 bits: sizes, alignments, ties, masks, values that are not finite, capture."""
import math

import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF, SINGLE = torch.float16, torch.float32


def reference(x, given, top_n):
    """One row, float64: (entropy, given, tokens, top, bounds of the errors of a log probability and of the entropy)."""
    V = len(x)
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    order = np.lexsort((np.arange(V), -x))
    if top == -np.inf:
        return 0.0, np.full(len(given), -np.inf), np.full(top_n, -1), np.full(top_n, -np.inf), 0.0, 0.0
    with np.errstate(invalid="ignore", under="ignore"):
        far = np.where(x == top, 0.0, -np.inf if top == np.inf else x - top)
        w = np.exp(far)
    far = np.where(w > 0, far, 0.0)
    rest = w.sum() - 1.0 if w.sum() > 1.5 else np.delete(w, order[0]).sum()
    log_sum = math.log1p(rest)
    lp = np.where(w > 0, far, -np.inf) - log_sum
    with np.errstate(invalid="ignore"):
        lp = np.where((w == 0) & (x > -np.inf) & (top < np.inf), x - top - log_sum, lp)
    entropy = log_sum - (w * far).sum() / (1 + rest)
    tokens, best = np.full(top_n, -1), np.full(top_n, -np.inf)
    kept = [i for i in order[:top_n] if lp[i] > -np.inf]
    tokens[:len(kept)], best[:len(kept)] = kept, lp[kept]
    # a weight: its difference and that times log2 e rounded (|t| 2^-24 each), 8 steps for the exponential; a thread's sum of V / 256
    # weights and some more, each step rounded
    step = 2.0 ** -24
    each = 2 * np.abs(far) + 8 + V / 256 + 32
    without = w.copy()
    without[order[0]] = 0.0
    err = step * (without * each).sum()
    err_turned = step * (w * np.abs(far) * each).sum()
    err_lp = err / (1 + rest)
    return entropy, np.array([lp[g] if 0 <= g < V else -np.inf for g in given]), tokens, best, err_lp, \
        err_lp + (err_turned + np.abs((w * far).sum()) * err / (1 + rest)) / (1 + rest)


def call(logits, given, top_n, R, V, canary=True):
    n = given.shape[1]
    need = fq.fq_logprobs_workspace_bytes(R, V)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)
    outs = dict(given=torch.from_numpy(given).to(DEV) if n else None, given_logprob=torch.full((R, n), 7.0, device=DEV) if n else None,
                top_token=torch.full((R, top_n), 7, dtype=torch.int32, device=DEV) if top_n else None,
                top_logprob=torch.full((R, top_n), 7.0, device=DEV) if top_n else None, entropy=torch.full((R + 1,), 7.0, device=DEV))
    (fq.fq_logprobs if logits.dtype is SINGLE else fq.fq_logprobs_f16)(logits, R, V, ws[:need], **outs)
    torch.cuda.synchronize()
    assert torch.all(ws[need:] == 255) and outs["entropy"][R] == 7.0
    return outs


def check(logits, given, top_n, rows=None):
    """logits [R][V] on the device, any strides."""
    R, V = logits.shape
    got = call(logits, given, top_n, R, V)
    got = {k: None if v is None else v.cpu().numpy() for k, v in got.items()}
    x = logits.double().cpu().numpy()
    step = 2.0 ** -24
    for r in (range(R) if rows is None else rows):
        entropy, lp, tokens, best, err_lp, err_h = reference(x[r], given[r], top_n)

        def near(a, b, err):
            a = a.astype(np.float64)
            with np.errstate(over="ignore"):  # a difference of two binary32 values may pass binary32 (2 * 3.4e38): it rounds to -inf there
                b = np.where(np.isinf(b.astype(np.float32)), b.astype(np.float32), b)
            same = (a == b) | (np.abs(a - np.where(np.isfinite(b), b, 0.0)) <= 2 * step * np.abs(np.where(np.isfinite(b), b, 0.0)) + err)
            assert np.all(same & (np.isinf(a) == np.isinf(b))), (r, a, b, err)
        near(got["entropy"][r:r + 1], np.array([entropy]), err_h + 2.0 ** -126)
        if given.shape[1]:
            near(got["given_logprob"][r], lp, err_lp + 2.0 ** -126)
        if top_n:
            assert np.array_equal(got["top_token"][r], tokens), (r, got["top_token"][r], tokens)
            near(got["top_logprob"][r], best, err_lp + 2.0 ** -126)


def rows_of(R, V, dtype, seed=0, deviation=3.0):
    gen = torch.Generator().manual_seed(seed)
    return (deviation * torch.randn((R, V), generator=gen)).to(dtype)


def some(R, V, n, seed=0):
    return np.random.default_rng(seed).integers(0, V, (R, n)).astype(np.int32)


@pytest.mark.parametrize("dtype", [SINGLE, HALF])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 31, 63, 64, 65, 127, 500, 1000, 1024, 4097, 10000, 32000, 50257, 128256])
@pytest.mark.parametrize("R,top_n", [(1, 5), (3, 64)])
def test_vocabularies(dtype, V, R, top_n):
    check(rows_of(R, V, dtype, V).to(DEV), some(R, V, 2), top_n)


@pytest.mark.parametrize("dtype", [SINGLE, HALF])
@pytest.mark.parametrize("R,V", [(1, 200000), (2, 152064), (16, 32000), (17, 32001), (64, 4096), (65, 5000), (130, 32000), (300, 999), (520, 128),
                                 (1100, 2049), (3000, 70)])
def test_row_counts(dtype, R, V):
    check(rows_of(R, V, dtype, R).to(DEV), some(R, V, 1), 20, rows=range(0, R, max(1, R // 60)))


@pytest.mark.parametrize("top_n", [0, 1, 2, 3, 10, 20, 33, 63, 64])
@pytest.mark.parametrize("R", [1, 150])
def test_numbers_of_alternatives(top_n, R):
    check(rows_of(R, 5000, SINGLE, top_n).to(DEV), some(R, 5000, 1), top_n, rows=range(0, R, 10))


@pytest.mark.parametrize("dtype", [SINGLE, HALF])
@pytest.mark.parametrize("lead", range(9))
@pytest.mark.parametrize("V", [1, 64, 777, 33001])
def test_rows_begin_anywhere(dtype, lead, V):
    """What stands between the rows would win."""
    wide = torch.full((3, V + lead + 5), 99.0, dtype=dtype)
    wide[:, lead:lead + V] = rows_of(3, V, dtype, lead)
    wide = wide.to(DEV)
    check(wide[:, lead:lead + V], some(3, V, 1), 7)
    check(wide[1:2, lead:lead + V], some(1, V, 1), 7)


@pytest.mark.parametrize("dtype", [SINGLE, HALF])
@pytest.mark.parametrize("R,V", [(1, 59999), (1, 60000), (64, 60001), (65, 60001), (7, 262143), (3, 131072)])
def test_long_rows_begin_anywhere(dtype, R, V):
    """Rows of small batches are taken in pieces from 60000 logits on."""
    gen = torch.Generator(device=DEV).manual_seed(V)
    for lead in (0, 1, 5):
        wide = torch.full((R, V + lead + 3), 99.0, dtype=dtype, device=DEV)
        wide[:, lead:lead + V].normal_(0.0, 3.0, generator=gen)
        check(wide[:, lead:lead + V], some(R, V, 1), 20, rows=sorted({0, R // 2, R - 1}))


def test_more_rows_than_a_launch_takes():
    R, V = (1 << 20) + 3, 5
    x = torch.randn((R, V), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    given = np.ascontiguousarray(np.broadcast_to(np.arange(R, dtype=np.int32)[:, None] % V, (R, 1)))
    check(x, given, 2, rows=(0, 1, (1 << 20) - 1, 1 << 20, R - 1))


def test_two_streams_at_once():
    xs = [rows_of(3, 128256, SINGLE, seed).to(DEV) for seed in (1, 2)]
    whole = [call(x, some(3, 128256, 1), 9, 3, 128256) for x in xs]
    streams, outs = [torch.cuda.Stream() for _ in xs], [{k: None if v is None else v.clone() for k, v in w.items()} for w in whole]
    spaces = [torch.empty(fq.fq_logprobs_workspace_bytes(3, 128256), dtype=torch.uint8, device=DEV) for _ in xs]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, o, ws, s in zip(xs, outs, spaces, streams):
            fq.fq_logprobs(x, 3, 128256, ws, stream=s, **o)
    torch.cuda.synchronize()
    assert all(torch.equal(o[k], w[k]) for o, w in zip(outs, whole) for k in w)


ROWS = {"equal": lambda V, g: torch.zeros(V), "ascending": lambda V, g: torch.arange(V) / V * 30, "descending": lambda V, g: -torch.arange(V) / V * 30,
        "few_values": lambda V, g: torch.randint(0, 4, (V,), generator=g).float(),
        "two_values": lambda V, g: (torch.rand(V, generator=g) < 0.01).float() * 5,
        "cluster": lambda V, g: torch.randn(V, generator=g) + 40.0 * (torch.arange(V) // 300 == V // 700),
        "outlier": lambda V, g: torch.randn(V, generator=g) + 60000.0 * (torch.arange(V) == V // 3),
        "lowest": lambda V, g: torch.where(torch.rand(V, generator=g) < 0.02, torch.randn(V, generator=g), torch.tensor(-65504.0)),
        "few_above_lowest": lambda V, g: torch.where(torch.arange(V) % 4001 == 17, torch.randn(V, generator=g), torch.tensor(-65504.0)),
        "masked": lambda V, g: torch.where(torch.arange(V) % 4001 == 17, torch.randn(V, generator=g), torch.tensor(-math.inf)),
        "one_left": lambda V, g: torch.where(torch.arange(V) == V - 1, 3.0, -math.inf),
        "nothing": lambda V, g: torch.full((V,), -math.inf),
        "nan": lambda V, g: torch.where(torch.rand(V, generator=g) < 0.3, math.nan, torch.randn(V, generator=g)),
        "only_nan": lambda V, g: torch.full((V,), math.nan),
        "nan_first": lambda V, g: torch.where(torch.arange(V) < V // 2, math.nan, torch.randn(V, generator=g)),
        "infinite": lambda V, g: torch.where(torch.arange(V) % 1000 == 5, math.inf, torch.randn(V, generator=g)),
        "infinite_and_nan": lambda V, g: torch.where(torch.arange(V) == V // 2, math.inf, torch.full((V,), math.nan)),
        "sure": lambda V, g: torch.randn(V, generator=g) + 25.0 * (torch.arange(V) == V // 2),
        "very_sure": lambda V, g: 0.01 * torch.randn(V, generator=g) + 60.0 * (torch.arange(V) == 1),
        "signed_zeros": lambda V, g: torch.where(torch.arange(V) % 2 == 0, -0.0, 0.0)}


@pytest.mark.parametrize("dtype", [SINGLE, HALF])
@pytest.mark.parametrize("kind", sorted(ROWS))
@pytest.mark.parametrize("V", [1, 5, 777, 32000, 130001])
def test_rows_of_all_kinds(dtype, kind, V):
    g = torch.Generator().manual_seed(V)
    row = ROWS[kind](V, g).to(dtype)
    given = np.array([[0, V // 2, V - 1, min(17, V - 1)]] * 3, dtype=np.int32)
    rows = torch.stack([row, row.flip(0), rows_of(1, V, dtype)[0]]).to(DEV)
    for top_n in (20, 64):
        check(rows, given, top_n)
        check(rows[:1], given[:1], top_n)
    many = rows.repeat(100, 1)
    check(many, np.repeat(given[:1], 300, 0), 5, rows=(0, 1, 2, 298, 299))


@pytest.mark.parametrize("dtype,words,ints", [(SINGLE, [0x7f800001, 0x7fc00000, -0x7fffff, -1], torch.int32), (HALF, [0x7c01, 0x7e00, -0x3ff, -1], torch.int16)])
@pytest.mark.parametrize("R,V", [(1, 777), (3, 32000), (2, 70001)])
def test_nans_of_all_kinds_are_as_minus_infinity(dtype, words, ints, R, V):
    """Quiet and signalling, of both signs."""
    gen = torch.Generator().manual_seed(V)
    x = torch.randn((R, V), generator=gen).to(dtype)
    at = torch.rand((R, V), generator=gen) < 0.1
    which = torch.randint(0, len(words), (R, V), generator=gen)
    bad = torch.where(at, torch.tensor(words, dtype=ints)[which], x.view(ints)).view(dtype)
    assert torch.equal(torch.isnan(bad), at)
    outs = []
    for logits in (bad.to(DEV), torch.where(at, -torch.inf, x).to(DEV)):
        token, best = torch.empty((R, 20), dtype=torch.int32, device=DEV), torch.empty((R, 20), device=DEV)
        given = torch.arange(R * 9, dtype=torch.int32, device=DEV).view(R, 9)
        lp, h = torch.empty((R, 9), device=DEV), torch.empty(R, device=DEV)
        ws = torch.empty(fq.fq_logprobs_workspace_bytes(R, V), dtype=torch.uint8, device=DEV)
        (fq.fq_logprobs if dtype == SINGLE else fq.fq_logprobs_f16)(logits, R, V, ws, given, lp, token, best, h)
        outs.append((token, best, lp, h))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("size", [1e-30, 1e4, 1e30, 3e38])
def test_magnitudes_of_binary32(size):
    x = torch.rand((2, 5000), generator=torch.Generator().manual_seed(1), dtype=torch.float64) * 2 - 1
    check((x * size).float().to(DEV), some(2, 5000, 3), 20)


def test_a_token_that_is_nearly_certain_keeps_its_digits():
    x = torch.full((2, 30000), -10.0)
    x[0, 11], x[1, 29999] = 30.0, 40.0
    got = call(x.to(DEV), np.array([[11], [29999]], dtype=np.int32), 1, 2, 30000)
    for r, top in ((0, 30.0), (1, 40.0)):
        want = -math.log1p(29999 * math.exp(-10.0 - top))
        assert abs(float(got["given_logprob"][r, 0]) / want - 1) < 1e-4
        assert abs(float(got["entropy"][r]) / (-want + 29999 * math.exp(-10.0 - top) * (top + 10.0)) - 1) < 1e-4


def test_given_tokens_of_all_kinds():
    V = 3001
    odd = np.array([[-1, 0, V - 1, V, 2 ** 31 - 1, -2 ** 31, 5, 5]] * 4, dtype=np.int32)
    check(rows_of(4, V, HALF).to(DEV), odd, 0)
    check(rows_of(2, V, SINGLE).to(DEV), some(2, V, 2000), 3)


def test_only_some_outputs():
    x = rows_of(5, 4000, SINGLE).to(DEV)
    ws = torch.empty(fq.fq_logprobs_workspace_bytes(5, 4000), dtype=torch.uint8, device=DEV)
    whole = call(x, some(5, 4000, 1), 4, 5, 4000)
    one = torch.empty(5, device=DEV)
    fq.fq_logprobs(x, 5, 4000, ws, given=whole["given"][:, 0].contiguous(), given_logprob=one)
    h = torch.empty(5, device=DEV)
    fq.fq_logprobs(x, 5, 4000, ws, entropy=h)
    t, p = torch.empty((5, 4), dtype=torch.int32, device=DEV), torch.empty((5, 4), device=DEV)
    fq.fq_logprobs(x, 5, 4000, ws, top_token=t, top_logprob=p)
    fq.fq_logprobs(x, 5, 4000, ws)
    fq.fq_logprobs(x, 0, 4000, ws)
    assert torch.equal(one, whole["given_logprob"][:, 0]) and torch.equal(h, whole["entropy"][:5])
    assert torch.equal(t, whole["top_token"]) and torch.equal(p, whole["top_logprob"])


@pytest.mark.parametrize("dtype,V", [(HALF, 1 << 24), (SINGLE, 3000001)])
def test_the_longest_rows(dtype, V):
    gen = torch.Generator(device=DEV).manual_seed(4)
    x = torch.empty((1, V), dtype=SINGLE, device=DEV).normal_(0.0, 3.0, generator=gen).to(dtype)
    check(x, some(1, V, 1), 20)
    x[0, V - 3] = 30.0
    check(x, some(1, V, 1), 64)


@pytest.mark.parametrize("R,V", [(1, 128256), (300, 5000)])
def test_equal_calls_give_equal_bits_and_a_captured_one_follows_its_inputs(R, V):
    x, given = rows_of(R, V, SINGLE).to(DEV), torch.from_numpy(some(R, V, 2)).to(DEV)
    outs = dict(given=given, given_logprob=torch.empty((R, 2), device=DEV), top_token=torch.empty((R, 9), dtype=torch.int32, device=DEV),
                top_logprob=torch.empty((R, 9), device=DEV), entropy=torch.empty(R, device=DEV))
    ws = torch.full((fq.fq_logprobs_workspace_bytes(R, V),), 255, dtype=torch.uint8, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        fq.fq_logprobs(x, R, V, ws, **outs)
    for step in range(4):
        x.copy_(x.roll(step + 1, 1) * 0.9)
        given.add_(1)
        g.replay()
        torch.cuda.synchronize()
        first = {k: v.clone() for k, v in outs.items()}
        for k, v in outs.items():
            if k != "given":
                v.fill_(3)
        ws.fill_(step)
        fq.fq_logprobs(x, R, V, ws, **outs)
        torch.cuda.synchronize()
        assert all(torch.equal(first[k], outs[k]) for k in outs)


def test_the_entropy_is_that_of_fq_entropy_kl():
    x = rows_of(40, 32000, SINGLE).to(DEV)
    other = torch.empty(40, device=DEV)
    fq.fq_entropy_kl(x, None, 40, 32000, other, None)
    got = call(x, some(40, 32000, 1), 0, 40, 32000)["entropy"][:40]
    assert torch.allclose(got, other, rtol=1e-5, atol=0)
