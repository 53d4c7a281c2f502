"""fq_logprobs of many rows of long vocabularies, whose blocks of logits are doubled, and its accuracy by the number of logits that a thread adds up."""
import math

import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq
from test_gpu_logprobs import ROWS, call, check, rows_of, some

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF, SINGLE = torch.float16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [SINGLE, HALF])


def normal(R, V, dtype, lead, seed):
    """Rows that begin anywhere; what stands between them would win."""
    wide = torch.full((R, V + lead + 3), 99.0, dtype=dtype, device=DEV)
    wide[:, lead:lead + V].normal_(0.0, 3.0, generator=torch.Generator(device=DEV).manual_seed(seed))
    return wide[:, lead:lead + V]


@TYPES
@pytest.mark.parametrize("R,V", [(65, 131064), (65, 131073), (65, 200000), (300, 152064), (300, 262145), (90, 600001)])
def test_many_rows_of_long_vocabularies(dtype, R, V):
    for lead, top_n in ((0, 20), (1, 64), (5, 5), (0, 0)):
        check(normal(R, V, dtype, lead, V + lead), some(R, V, 3), top_n, rows=sorted({0, R // 2, R - 1}))


@TYPES
@pytest.mark.parametrize("R", [65, 300])
@pytest.mark.parametrize("kind", sorted(ROWS))
def test_rows_of_all_kinds_among_many(dtype, R, kind):
    V = 151937
    row = ROWS[kind](V, torch.Generator().manual_seed(V)).to(dtype)
    x = normal(R, V, dtype, 3, 1)
    x[1], x[R - 1] = row.to(DEV), row.flip(0).to(DEV)
    given = np.tile(np.array([[0, V // 2, V - 1, 17]], dtype=np.int32), (R, 1))
    for top_n in (20, 64):
        check(x, given, top_n, rows=(0, 1, 2, R - 1))


@TYPES
def test_all_of_the_best_in_one_block_and_at_both_ends(dtype):
    R, V = 70, 200001
    x = normal(R, V, dtype, 1, 2)
    x[0, 64 * 1000:64 * 1000 + 128] += 40.0
    x[1, :64] += 40.0
    x[2, V - 70:] += 40.0
    x[3] = torch.where(torch.arange(V, device=DEV) % 3000 == 1, 30.0, -20.0).to(dtype)
    check(x, some(R, V, 1), 64, rows=range(5))


@pytest.mark.parametrize("R", [70, 3])
def test_a_captured_call_of_long_vocabularies(R):
    V = 200000
    x, given = rows_of(R, V, HALF).to(DEV), torch.from_numpy(some(R, V, 2)).to(DEV)
    outs = dict(given=given, given_logprob=torch.empty((R, 2), device=DEV), top_token=torch.empty((R, 9), dtype=torch.int32, device=DEV),
                top_logprob=torch.empty((R, 9), device=DEV), entropy=torch.empty(R, device=DEV))
    ws = torch.full((fq.fq_logprobs_workspace_bytes(R, V),), 255, dtype=torch.uint8, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        fq.fq_logprobs_f16(x, R, V, ws, **outs)
    for step in range(4):
        x.copy_(x.roll(step + 1, 1) * 0.9)
        given.add_(1)
        for k, v in outs.items():
            if k != "given":
                v.fill_(5)
        g.replay()
        torch.cuda.synchronize()
        first = {k: v.clone() for k, v in outs.items()}
        for k, v in outs.items():
            if k != "given":
                v.fill_(3)
        ws.fill_(step)
        fq.fq_logprobs_f16(x, R, V, ws, **outs)
        torch.cuda.synchronize()
        assert all(torch.equal(first[k], outs[k]) for k in outs)


@pytest.mark.parametrize("R,V", [(3, 128256), (70, 151936)])
def test_two_streams_at_once_write_all_of_their_outputs(R, V):
    xs = [rows_of(R, V, SINGLE, seed).to(DEV) for seed in (1, 2)]
    given = some(R, V, 1)
    whole = [call(x, given, 9, R, V) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    outs = [{k: v.clone() if k == "given" else torch.full_like(v, 9) for k, v in w.items()} for w in whole]
    spaces = [torch.full((fq.fq_logprobs_workspace_bytes(R, V),), 255, dtype=torch.uint8, device=DEV) for _ in xs]
    for o in outs:
        o["entropy"] = o["entropy"][:R]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, o, ws, s in zip(xs, outs, spaces, streams):
            fq.fq_logprobs(x, R, V, ws, stream=s, **o)
    torch.cuda.synchronize()
    assert all(torch.equal(o[k], w[k][:R]) for o, w in zip(outs, whole) for k in w)


def loads_of_a_thread(R, V, per):
    """16-byte loads that a thread adds up in binary32: pieces of rows for up to 64 long ones, else a workgroup to a row (256 compute units)."""
    loads = (V + per - 1) // per + 1
    if R <= 64 and V >= 60000:
        ahead, threads = 32 // per, 512
        units = -(-loads // (threads * ahead))
        pieces = max(1, min(64, 2 * 256 // R))
        return ahead * -(-units // pieces)
    threads = 64 if loads <= 256 else 1024 if R < 256 and loads > 4096 else 256 if loads <= 2048 else 512
    return -(-loads // threads) + 32 // per


@TYPES
@pytest.mark.parametrize("R,V", [(1, 1000), (1, 32000), (3, 128256), (1, 1 << 24), (64, 65536), (65, 65536), (70, 600001), (65, 1 << 22), (300, 50257), (300, 151936)])
def test_accuracy_by_what_a_thread_adds_up(dtype, R, V):
    """Sums of weights and of weights times distance, every step of a binary32 sum rounded."""
    per = 4 if dtype is SINGLE else 8
    x = torch.empty((R, V), device=DEV, dtype=SINGLE).normal_(0.0, 3.0, generator=torch.Generator(device=DEV).manual_seed(V)).to(dtype)
    got = call(x, some(R, V, 2), 1, R, V)
    given = some(R, V, 2)
    loads, step = loads_of_a_thread(R, V, per), 2.0 ** -24
    for r in sorted({0, R // 2, R - 1}):
        row = x[r].double().cpu().numpy()
        first = int(np.argmax(row))
        far = row - row[first]
        w = np.exp(far)
        without = w.copy()
        without[first] = 0.0
        rest, turned = without.sum(), (w * far).sum()
        # a weight: its distance and that times log2 e (|far| steps each), 8 for the exponential; the sum of a load's weights (per - 1 at
        # most) and of the thread's loads; a raise of the running maximum takes the sum times a power, 10 steps, a turn of
        # 32 / per loads at most one; four sums over lanes
        each = 2 * np.abs(far) + 8 + (per - 1) + loads + 10 * -(-loads // (32 // per)) + 4
        err = step * (without * each).sum()
        err_turned = step * (w * np.abs(far) * (each + 1)).sum()
        err_lp = err / (1 + rest)
        for j, g in enumerate(given[r]):
            ref = far[g] - math.log1p(rest)
            assert abs(float(got["given_logprob"][r, j]) - ref) <= err_lp + 2 * step * abs(ref), (r, j)
        assert abs(float(got["top_logprob"][r, 0]) + math.log1p(rest)) <= err_lp + 2 * step * math.log1p(rest)
        entropy = math.log1p(rest) - turned / (1 + rest)
        err_h = err_lp + (err_turned + abs(turned) * err / (1 + rest)) / (1 + rest)
        assert abs(float(got["entropy"][r]) - entropy) <= err_h + 2 * step * entropy
