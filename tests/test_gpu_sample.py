"""fq_sample and fq_sample_f16 against whole-number arithmetic on the host: tokens are equal."""
import numpy as np
import pytest
import torch

import paper_2506_12024_amd as fq
from serve_util import draw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def run(x, u, temperature=None, top_k=None, top_p=None, min_p=None, half=False, stride=None, stream=None):
    """x numpy [R][V]; the settings arrays or None.  Compares every row with the reference and returns the tokens."""
    R, V = x.shape
    dtype = torch.float16 if half else torch.float32
    x = x.astype(np.float16 if half else np.float32)
    store = torch.full((R, stride or V), float("nan"), dtype=dtype, device=DEV)
    store[:, :V] = torch.from_numpy(x.astype(np.float32)).to(DEV).to(dtype)
    dev = [None if a is None else torch.from_numpy(np.asarray(a, dtype=t)).to(DEV) for a, t in
           ((u, np.float32), (temperature, np.float32), (top_k, np.int32), (top_p, np.float32), (min_p, np.float32))]
    token = torch.full((R,), -7, dtype=torch.int32, device=DEV)
    prob = torch.full((R,), -7.0, dtype=torch.float32, device=DEV)
    ws = torch.empty(fq.fq_sample_workspace_bytes(R, V), dtype=torch.uint8, device=DEV)
    (fq.fq_sample_f16 if half else fq.fq_sample)(store[:, :V], R, V, dev[0], token, ws, dev[1], dev[2], dev[3], dev[4], prob, stream)
    torch.cuda.synchronize()
    token, prob = token.cpu().numpy(), prob.cpu().numpy()
    for r in range(R):
        at = lambda a, off, t: off if a is None else t(a[r])
        want, p = draw(x[r].astype(np.float32), np.float32(u[r]), at(temperature, np.float32(1), np.float32), at(top_k, 0, int),
                       at(top_p, np.float32(1), np.float32), at(min_p, np.float32(0), np.float32))
        assert token[r] == want, (r, token[r], want)
        assert abs(prob[r] - p) <= 2.0 ** -23 * p, (r, prob[r], p)
    return token


def settings(rng, R):
    return dict(temperature=rng.choice([0.0, 0.3, 0.7, 1.0, 1.5, 30.0], R), top_k=rng.choice([-1, 0, 1, 2, 40, 1000, 1 << 30], R),
                top_p=rng.choice([0.0, 0.1, 0.5, 0.9, 0.999, 1.0, 2.0], R), min_p=rng.choice([0.0, 1e-6, 0.05, 0.7, 1.0, 3.0], R))


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 1000, 1023, 1025, 4097, 32000])
def test_all_settings_at_once(V, half):
    rng = np.random.default_rng(V)
    R = 24
    run(rng.normal(0, 3, (R, V)), rng.random(R, dtype=np.float32), half=half, **settings(rng, R))


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("name,value", [("temperature", 0.7), ("top_k", 1), ("top_k", 50), ("top_k", 3000), ("top_p", 0.02),
                                        ("top_p", 0.9), ("min_p", 0.1)])
def test_one_setting_alone(name, value, half):
    rng = np.random.default_rng(5)
    for R, V in ((1, 32000), (6, 5001)):
        run(rng.normal(0, 2, (R, V)), rng.random(R, dtype=np.float32), half=half, **{name: [value] * R})
    run(rng.normal(0, 2, (3, 700)), rng.random(3, dtype=np.float32), half=half)


@pytest.mark.parametrize("V", [128256, 152064, 300001])
def test_large_vocabularies(V):
    rng = np.random.default_rng(V)
    R = 5
    run(rng.normal(0, 3, (R, V)), rng.random(R, dtype=np.float32), temperature=[1, 0.8, 1, 1.2, 0],
        top_k=[0, 0, 64, 2000, 0], top_p=[1, 0.9, 0.95, 1, 1], min_p=[0, 0, 0, 0.01, 0])
    run(rng.normal(0, 0.01, (2, V)), rng.random(2, dtype=np.float32), top_p=[0.7, 0.999])
    run(rng.normal(0, 40, (2, V)), rng.random(2, dtype=np.float32), top_p=[0.7, 0.999])


@pytest.mark.parametrize("V", [10, 1000, 40000])
def test_ties_go_to_the_lowest_index(V):
    """Equal logits, logits on a coarse grid, zeros of both signs."""
    rng = np.random.default_rng(9)
    u = np.array([0.0, 0.25, 0.5, 0.999, 0.75], dtype=np.float32)
    same = np.zeros((5, V))
    run(same, u)
    run(same, u, top_k=[1, 2, 5, 7, 9])
    run(same, u, top_p=[0.5, 0.5, 0.25, 0.1, 0.3], min_p=[1.0] * 5)
    run(np.where(rng.random((5, V)) < 0.5, 0.0, -0.0), u, top_k=[3] * 5)
    coarse = np.round(rng.normal(0, 1, (5, V)))
    run(coarse, u, top_k=[0, 1, 4, V // 2, V - 1], top_p=[0.5, 0.9, 0.9, 0.3, 0.99])
    run(coarse, u, temperature=[0.0, -1.0, np.nan, 1.0, 2.0], half=True)


def test_infinities_and_nan():
    V, inf, nan = 3000, np.inf, np.nan
    rng = np.random.default_rng(2)
    x = rng.normal(0, 2, (8, V))
    x[0, :] = -inf                       # nothing to draw
    x[1, :] = nan
    x[2, :] = -inf
    x[2, 1234] = -50.0                   # one entry
    x[3, rng.random(V) < 0.5] = -inf
    x[4, rng.random(V) < 0.5] = nan
    x[5, [7, 900, 2999]] = inf           # three entries hold everything
    x[6, :] = np.finfo(np.float32).min   # equal, at the type's lowest
    x[7, ::2] = np.finfo(np.float32).min
    u = rng.random(8, dtype=np.float32)
    none = run(x, u)
    assert none[0] == none[1] == -1 and none[2] == 1234 and none[5] in (7, 900, 2999)
    run(x, u, top_k=[5, 5, 5, 1900, 1900, 2, 3, 2000], top_p=[0.9] * 8, min_p=[0.01] * 8)
    run(x, u, temperature=[0.0] * 8)
    run(x, u, temperature=[np.inf] * 8)
    run(x, u, temperature=[1e-40, 1e-38, 1e-30, 1e30, 1e38, 1e-20, 1.0, 1e-45])


def test_temperatures_and_logits_of_any_size():
    """Logits far from 0, steps of binary32 wider than the temperature, weights that are all 1 or all 0 but one."""
    V = 2500
    rng = np.random.default_rng(12)
    u = rng.random(10, dtype=np.float32)
    scale = np.array([1e-40, 1e-30, 1e-6, 1.0, 1e4, 1e8, 1e20, 1e30, 1e37, 5e37])[:, None]
    x = (rng.normal(0, 1, (10, V)) * scale).astype(np.float32)
    offset = x + np.float32(1e4)
    for t in (1e-40, 1e-30, 1e-6, 0.01, 1.0, 1e6, 1e30, 1e38):
        run(x, u, temperature=[t] * 10)
        run(x, u, temperature=[t] * 10, top_p=[0.9] * 10)
        run(x, u, temperature=[t] * 10, top_k=[40] * 10, min_p=[0.3] * 10)
    for t in (0.01, 0.5, 1.0, 1e6, 1e30):
        run(offset, u, temperature=[t] * 10)
        run(offset, u, temperature=[t] * 10, top_p=[0.9] * 10)
    x[:, ::3] = -np.inf
    x[:, 5] = np.nan
    run(x, u, temperature=[np.inf] * 10, top_k=[7] * 10)
    run(x, u, temperature=[np.inf] * 10, top_p=[0.3] * 10)
    run(x, u, temperature=[1e30] * 10, top_p=[0.3] * 10, min_p=[1e-3] * 10)


def test_numbers_at_the_ends():
    rng = np.random.default_rng(3)
    x = rng.normal(0, 3, (6, 2000))
    x[:, 0], x[:, 1999] = -200.0, -200.0  # too light to be drawn at either end
    run(x, np.array([0.0, 1.0 - 2.0 ** -24, 2.0 ** -24, 2.0 ** -60, 1e-45, 0.5], dtype=np.float32))
    run(x, np.array([1.0, 5.0, -1.0, -0.0, 0.0, 1e-30], dtype=np.float32), top_k=[3] * 6)


@pytest.mark.parametrize("half", [False, True])
def test_rows_apart_and_unaligned(half):
    rng = np.random.default_rng(4)
    for V, stride in ((1000, 1001), (1000, 1003), (32000, 32002), (5, 9)):
        run(rng.normal(0, 3, (7, V)), rng.random(7, dtype=np.float32), half=half, stride=stride, top_p=[0.9] * 7)


def test_many_rows():
    rng = np.random.default_rng(6)
    run(rng.normal(0, 3, (700, 257)), rng.random(700, dtype=np.float32), **settings(rng, 700))


def test_frequencies_of_tokens():
    """Over evenly spread numbers every token comes as often as its probability says."""
    x = np.log(np.array([0.05, 0.4, 0.25, 0.3]))
    R = 4000
    token = run(np.tile(x, (R, 1)), ((np.arange(R) + 0.5) / R).astype(np.float32))
    assert np.abs(np.bincount(token, minlength=4) / R - [0.05, 0.4, 0.25, 0.3]).max() < 1e-3


def test_streams_and_graphs():
    rng = np.random.default_rng(8)
    R, V = 3, 40000
    x = torch.from_numpy(rng.normal(0, 3, (R, V)).astype(np.float32)).to(DEV)
    u = torch.from_numpy(rng.random(R, dtype=np.float32)).to(DEV)
    kw = dict(top_k=torch.tensor([0, 50, 0], dtype=torch.int32, device=DEV), top_p=torch.tensor([0.9, 1.0, 1.0], device=DEV))
    ws = torch.empty(fq.fq_sample_workspace_bytes(R, V), dtype=torch.uint8, device=DEV)
    ws2 = torch.empty_like(ws)
    token, prob = torch.empty(R, dtype=torch.int32, device=DEV), torch.empty(R, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        fq.fq_sample(x, R, V, u, token, ws, prob=prob, **kw)
    side = torch.cuda.Stream()
    for _ in range(4):
        g.replay()
        torch.cuda.synchronize()
        t2, p2 = torch.empty_like(token), torch.empty_like(prob)
        fq.fq_sample(x, R, V, u, t2, ws2, prob=p2, stream=side, **kw)
        torch.cuda.synchronize()
        assert torch.equal(token, t2) and torch.equal(prob, p2)
        x.mul_(0.9)
        u.mul_(0.7).add_(0.2)
        ws.fill_(255)
        torch.cuda.synchronize()
