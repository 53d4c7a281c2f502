"""What a server adds to a decoder's step on this library: its cases and plain forms.

Three operators, in the order in which a step meets them: low-rank adapters of many requests beside the projection that
they share (``adapters``), norms of the heads of queries and keys with the rotary positions and the append to a paged
cache (``normed``), and log probabilities of given tokens with entropy and the likeliest alternatives (``logprobs``).
Sizes are those of the 7B-, 13B- and 70B-shaped stacks of ``synth`` and of the entropy workloads, and generic ones.

``run`` computes an operator in its plain form, elementary torch operations in 32 or 64 bits; with ``own`` set it makes
the library's calls instead.  ``exact`` is a second writing in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
THETA = 500000.0
EPS = 1e-6


def listed():
    return [
        # one token of a request with an adapter, beside the 7B query projection: launch and latency
        dict(name="adapters_token_7b", kind="adapters", type="f16", rows=1, mix="own", spare=0, adapters=8, rank=16,
             K=4096, N=4096),
        # a decode step of 32 requests with adapters of all ranks up to 32, some without, beside the 7B gate projection
        dict(name="adapters_batch32_7b", kind="adapters", type="f16", rows=32, mix="own", spare=4, adapters=24, rank=32,
             K=4096, N=11008),
        # chunks of some prompts and the single tokens of others in one call, beside the 7B down projection
        dict(name="adapters_mixed_7b", kind="adapters", type="f16", rows=701, mix="both", spare=1, adapters=12, rank=16,
             K=11008, N=4096),
        # one long prompt beside a 70B projection
        dict(name="adapters_prompt_70b", kind="adapters", type="bf16", rows=2048, mix="runs", spare=0, adapters=4,
             rank=64, K=8192, N=8192),
        # one token goes into the cache: launch and latency
        dict(name="normed_token", kind="normed", type="f16", seqs=1, new=1, kv=1000, q_heads=32, kv_heads=8, dim=128,
             rot=128, interleaved=False, page=16, token_major=False, fused=True, each=False, offset=0.0, far=False),
        # a decode step of 32 sequences far into their contexts, weights of each head's own
        dict(name="normed_batch32_70b", kind="normed", type="bf16", seqs=32, new=1, kv=1024, q_heads=64, kv_heads=8,
             dim=128, rot=128, interleaved=True, page=16, token_major=False, fused=False, each=True, offset=0.0, far=True),
        # chunks of nine prompts, narrow heads of which a quarter rotates, weights kept as their distance from one
        dict(name="normed_chunks_80", kind="normed", type="f16", seqs=9, new=300, kv=700, q_heads=32, kv_heads=32, dim=80,
             rot=20, interleaved=False, page=32, token_major=True, fused=True, each=False, offset=1.0, far=False),
        # a long prompt of the 70B shapes
        dict(name="normed_prompt_70b", kind="normed", type="f16", seqs=1, new=2048, kv=2048, q_heads=64, kv_heads=8,
             dim=128, rot=128, interleaved=False, page=64, token_major=False, fused=False, each=False, offset=0.0, far=False),
        # the drawn token of one request and five alternatives: launch and latency
        dict(name="logprobs_token", kind="logprobs", type="f32", rows=1, vocab=32000, given=1, top=5, masked=False),
        # a batch's drawn tokens with twenty alternatives, some requests held to a grammar, logits as fq_linear leaves them
        dict(name="logprobs_batch32_f16", kind="logprobs", type="f16", rows=32, vocab=128256, given=1, top=20, masked=True),
        # the tokens of a prompt scored, no alternatives
        dict(name="logprobs_prompt_f16", kind="logprobs", type="f16", rows=2048, vocab=32000, given=1, top=0, masked=False),
        # positions of several texts scored for four continuations each, with alternatives
        dict(name="logprobs_scoring", kind="logprobs", type="f32", rows=500, vocab=128256, given=4, top=20, masked=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["adapters", "adapters", "normed", "logprobs"])
    if kind == "logprobs":
        vocab = _log(rng, 50, 200000)
        return dict(kind=kind, type=rng.choice(["f32", "f16"]), rows=min(_log(rng, 1, 3000), max(1, 60000000 // vocab)),
                    vocab=vocab, given=rng.choice([0, 1, 1, rng.randint(2, 9)]), top=rng.choice([0, 1, 5, 20, rng.randint(1, 64)]),
                    masked=rng.random() < 0.3)
    if kind == "adapters":
        K, N = 8 * _log(rng, 8, 2048), _log(rng, 16, 28672)
        rank = rng.choice([8, 16, 16, 32, 64, 128])
        rows = min(_log(rng, 1, 4096), max(1, 50000000 // (K + 2 * N)))
        adapters = max(1, min(_log(rng, 1, 64), 60000000 // (rank * (K + N))))
        return dict(kind=kind, type=rng.choice(["f16", "bf16"]), rows=rows, mix=rng.choice(["own", "runs", "both"]),
                    spare=rng.choice([0, 0, 1, 4]), adapters=adapters, rank=rank, K=K, N=N)
    dim = rng.choice([64, 80, 96, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 32])
    q_heads = kv_heads * (rng.choice([1, 2]) if kv_heads == 32 else rng.choice([1, 2, 3, 4, 8]))
    new = rng.choice([1, _log(rng, 1, 1500)])
    seqs = max(1, min(_log(rng, 1, 64), 4000 // new, 16000000 // (new * q_heads * dim)))
    kv = new + _log(rng, 1, 1000)
    return dict(kind=kind, type=rng.choice(["f16", "bf16"]), seqs=seqs, new=new, kv=min(kv, new + 40000 * 8 // (seqs * kv_heads)),
                q_heads=q_heads, kv_heads=kv_heads, dim=dim, rot=rng.choice([dim, dim, dim // 2, 20]),
                interleaved=rng.random() < 0.5, page=rng.choice([8, 16, 32, 64, 128]), token_major=rng.random() < 0.3,
                fused=rng.random() < 0.4, each=rng.random() < 0.3, offset=rng.choice([0.0, 0.0, 1.0]), far=rng.random() < 0.4)


def _rng_of(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    """(new tokens, length with them) of each sequence; the last one is the longest the case allows."""
    rng = _rng_of(case)
    new, kv = [], []
    for _ in range(case["seqs"] - 1):
        n = rng.randint(1, case["new"])
        new.append(n)
        kv.append(n + rng.randint(0, case["kv"] - case["new"]))
    return new + [case["new"]], kv + [case["kv"]]


def _requests(case):
    """(adapter of each row, or -1; rank of each adapter).  "own": a request to a row, "runs": a few prompts' rows in a
    piece, "both": the pieces first, then requests of a row each.  One of `spare` + 1 requests has none with spare > 0."""
    rng = _rng_of(case)
    rows, n = case["rows"], case["adapters"]
    inside = {"own": 0, "runs": rows, "both": rows - rows // 8}[case["mix"]]

    def one():
        return -1 if case["spare"] and rng.randrange(case["spare"] + 4) == 0 else rng.randrange(n)
    of = []
    while len(of) < inside:
        of += [one()] * min(inside - len(of), rng.randint(max(1, inside // 4), inside))
    of += [one() for _ in range(rows - inside)]
    return of, [case["rank"]] + [rng.choice([case["rank"], case["rank"], case["rank"] // 2, max(1, case["rank"] // 4)])
                                 for _ in range(n - 1)]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = random.Random(seed)
    return {"adapters": _prepare_adapters, "normed": _prepare_normed, "logprobs": _prepare_logprobs}[case["kind"]](case, g, rng)


def _normal(g, shape, dtype, deviation=1.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, deviation, generator=g)


def _prepare_adapters(case, g, rng):
    dtype, n, rank, K, N, M = TYPES[case["type"]], case["adapters"], case["rank"], case["K"], case["N"], case["rows"]
    of, ranks = _requests(case)
    s = dict(case=case, x=_normal(g, (M, K), dtype), y=_normal(g, (M, N), dtype),
             a=_normal(g, (n, rank, K), dtype, 1.0 / math.sqrt(K)), b=_normal(g, (n, N, rank), dtype),
             adapter=torch.tensor(of, dtype=torch.int32).to(DEV), ranks=torch.tensor(ranks, dtype=torch.int32).to(DEV),
             scales=torch.tensor([rng.uniform(0.2, 2.0) / math.sqrt(r) for r in ranks], dtype=torch.float32).to(DEV),
             out=torch.empty((M, N), dtype=dtype, device=DEV))
    if own:
        import paper_2506_12024_amd as fq
        s["fq"] = fq
        s["handle"] = fq.Adapters(s["a"], s["b"], s["ranks"], s["scales"])
        s["workspace"] = torch.empty(fq.fq_adapters_workspace_bytes(s["handle"], M), dtype=torch.uint8, device=DEV)
    return s


def _prepare_normed(case, g, rng):
    dtype, page, heads, dim, Hq = TYPES[case["type"]], case["page"], case["kv_heads"], case["dim"], case["q_heads"]
    new, kv = _lengths(case)
    held = [-(-n // page) for n in kv]
    pages = sum(held) + 3
    order = list(range(pages))
    rng.shuffle(order)
    table = torch.zeros((case["seqs"], max(held) + 1), dtype=torch.int32)
    for b, n in enumerate(held):
        table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    T = sum(new)

    def pool():
        shape = (pages, page, heads, dim) if case["token_major"] else (pages, heads, page, dim)
        t = _normal(g, shape, dtype)
        return t.permute(0, 2, 1, 3) if case["token_major"] else t  # [page][head][token][dim] either way

    s = dict(case=case, new=new, kv=kv, q_start=torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32).to(DEV),
             kv_len=torch.tensor(kv, dtype=torch.int32).to(DEV), table=table.to(DEV), k_cache=pool(), v_cache=pool(),
             q_out=torch.empty((T, Hq, dim), dtype=dtype, device=DEV), positions=None)
    if case["fused"]:
        row = _normal(g, (T, Hq + 2 * heads, dim), dtype, 3.0)
        s["q"], s["k"], s["v"] = row[:, :Hq], row[:, Hq:Hq + heads], row[:, Hq + heads:]
    else:
        s["q"], s["k"], s["v"] = (_normal(g, (T, n, dim), dtype, 3.0) for n in (Hq, heads, heads))
    for name, n in (("q_weight", Hq), ("k_weight", heads)):
        w = 1.0 - case["offset"] + 0.3 * torch.randn((n, dim) if case["each"] else (dim,), device=DEV, generator=g)
        s[name] = w.to(dtype)
    # positions of their own where the cache holds the end of a longer context
    if case["far"]:
        s["positions"] = torch.cat([torch.arange(n, dtype=torch.int32) + rng.randint(10000, 120000) for n in new]).to(DEV)
    s["freqs"] = torch.tensor([THETA ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)], dtype=torch.float64).to(DEV)
    if own:
        import paper_2506_12024_amd as fq
        s["fq"] = fq
        s["cache"] = fq.KVCache(s["k_cache"], s["v_cache"])
        s["sequences"] = fq.Sequences(s["q_start"], s["kv_len"], s["table"])
    return s


def _prepare_logprobs(case, g, rng):
    R, V, n, top = case["rows"], case["vocab"], case["given"], case["top"]
    logits = _normal(g, (R, V), torch.float32, 3.0)
    # a confident row stands out by some nats, as after a word's first half
    sure = torch.randint(0, V, (R,), device=DEV, generator=g)
    logits[torch.arange(R, device=DEV), sure] += 20.0 * torch.rand(R, device=DEV, generator=g) ** 2
    if case["masked"]:  # every fourth request may go on with some hundreds of the tokens at most
        some = torch.rand((len(range(0, R, 4)), V), device=DEV, generator=g) * V >= rng.choice([8, 50, 300])
        logits[::4] = logits[::4].masked_fill(some, -math.inf)
        logits[::4, rng.randrange(V)] = 1.0
    s = dict(case=case, logits=logits.to(TYPES[case["type"]]), given=None, given_logprob=None, top_token=None, top_logprob=None,
             entropy=torch.empty(R, dtype=torch.float32, device=DEV))
    if n:
        s["given"] = torch.randint(0, V, (R, n), device=DEV, generator=g, dtype=torch.int32)
        s["given"][:, 0] = sure
        s["given_logprob"] = torch.empty((R, n), dtype=torch.float32, device=DEV)
    if top:
        s["top_token"] = torch.empty((R, top), dtype=torch.int32, device=DEV)
        s["top_logprob"] = torch.empty((R, top), dtype=torch.float32, device=DEV)
    if own:
        import paper_2506_12024_amd as fq
        s["fq"] = fq
        s["workspace"] = torch.empty(fq.fq_logprobs_workspace_bytes(R, V), dtype=torch.uint8, device=DEV)
    return s


def run(s):
    case = s["case"]
    if own:
        fq = s["fq"]
        if case["kind"] == "adapters":
            fq.fq_adapters_add(s["handle"], s["x"], s["adapter"], s["y"], s["out"], s["workspace"])
            return s["out"]
        if case["kind"] == "normed":
            fq.fq_kv_append_normed(s["cache"], s["sequences"], s["q"], s["k"], s["v"], s["q_out"], s["freqs"], s["q_weight"],
                                   s["k_weight"], eps=EPS, offset=case["offset"], interleaved=case["interleaved"],
                                   positions=s["positions"])
            return s["q_out"], s["k_cache"], s["v_cache"]
        call = fq.fq_logprobs if case["type"] == "f32" else fq.fq_logprobs_f16
        call(s["logits"], case["rows"], case["vocab"], s["workspace"], given=s["given"], given_logprob=s["given_logprob"],
             top_token=s["top_token"], top_logprob=s["top_logprob"], entropy=s["entropy"])
        return [s[k] for k in ("entropy", "given_logprob", "top_token", "top_logprob") if s[k] is not None]
    return {"adapters": _plain_adapters, "normed": _plain_normed, "logprobs": _plain_logprobs}[case["kind"]](s)


def _plain_adapters(s):
    """Every row through all adapters at once, the others' part of the row masked: y + ((x A^T) * mask * scale) B^T."""
    n, rank, K = s["a"].shape
    of = s["adapter"].long()[:, None]
    column = torch.arange(n * rank, device=DEV)
    kept = (column[None, :] // rank == of) & ((column % rank) < s["ranks"].long()[column // rank])[None, :]
    low = torch.matmul(s["x"].float(), s["a"].reshape(n * rank, K).float().t())
    low = torch.where(kept, low * s["scales"][column // rank][None, :], 0.0)
    added = torch.matmul(low, s["b"].float().transpose(1, 2).reshape(n * rank, -1))
    return (s["y"].float() + added).to(s["y"].dtype)


def _plain_normed(s):
    case, page, rot = s["case"], s["case"]["page"], s["case"]["rot"]
    T = s["q"].shape[0]
    t = torch.arange(T, device=DEV)
    seq = torch.searchsorted(s["q_start"][1:].long(), t, right=True)
    place = s["kv_len"].long()[seq] - (s["q_start"].long()[seq + 1] - t)
    where = place if s["positions"] is None else s["positions"]
    angle = where.double()[:, None, None] * s["freqs"]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def normed(x, weight):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * (weight.float() + case["offset"])
        head, tail = x[..., :rot], x[..., rot:]
        if case["interleaved"]:
            a, b = head[..., 0::2], head[..., 1::2]
            head = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
        else:
            a, b = head[..., :rot // 2], head[..., rot // 2:]
            head = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
        return torch.cat((head, tail), dim=-1).to(s["q"].dtype)

    at = s["table"].long()[seq, place // page]
    s["k_cache"].permute(0, 2, 1, 3)[at, place % page] = normed(s["k"], s["k_weight"])
    s["v_cache"].permute(0, 2, 1, 3)[at, place % page] = s["v"]
    return normed(s["q"], s["q_weight"]), s["k_cache"], s["v_cache"]


def _plain_logprobs(s):
    x = s["logits"].float()
    far = x - x.amax(dim=1, keepdim=True)
    w = torch.exp(far)
    total = w.sum(dim=1, keepdim=True)
    logprob = far - torch.log(total)
    p = w / total
    outs = [-torch.where(p > 0, p * logprob, 0.0).sum(dim=1)]
    if s["given"] is not None:
        outs.append(logprob.gather(1, s["given"].long()))
    if s["top_token"] is not None:
        n = min(s["top_token"].shape[1], x.shape[1])
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :n]
        best = torch.full(s["top_token"].shape, -math.inf, device=DEV)
        token = torch.full(s["top_token"].shape, -1, dtype=torch.int32, device=DEV)
        best[:, :n] = logprob.gather(1, order)
        token[:, :n] = torch.where(best[:, :n] > -math.inf, order, -1).int()
        outs += [token, best]
    return outs


def work(case):
    if case["kind"] == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (4 if case["type"] == "f32" else 2) + case["rows"] * (4 + 8 * case["given"] + 8 * case["top"]),
                "flops": 4 * n}
    if case["kind"] == "adapters":
        of, ranks = _requests(case)
        K, N = case["K"], case["N"]
        served = [a for a in of if a >= 0]
        return {"bytes": 2 * (len(served) * K + 2 * len(of) * N + sum(ranks[a] for a in set(served)) * (K + N)) + 4 * len(of),
                "flops": sum(2 * ranks[a] * (K + N) for a in served)}
    T = sum(_lengths(case)[0])
    moved = T * (2 * case["q_heads"] + 4 * case["kv_heads"]) * case["dim"] * 2
    return {"bytes": moved + 4 * case["rot"] + 4 * T * case["far"] + 12 * case["seqs"],
            "flops": T * (case["q_heads"] + case["kv_heads"]) * (case["rot"] * 3 + case["dim"] * 4)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"adapters": _exact_adapters, "normed": _exact_normed, "logprobs": _exact_logprobs}[case["kind"]](s)


def _exact_adapters(s):
    """Adapter by adapter: its rows alone, its own ranks alone."""
    out = s["y"].double()
    of, ranks, scales = s["adapter"].cpu().numpy(), s["ranks"].tolist(), s["scales"].double().tolist()
    for a in sorted(set(of[of >= 0].tolist())):
        rows = torch.from_numpy(np.flatnonzero(of == a)).to(DEV)
        r = ranks[a]
        out[rows] += scales[a] * ((s["x"][rows].double() @ s["a"][a, :r].double().T) @ s["b"][a, :, :r].double().T)
    return out


def _exact_normed(s):
    """Token by token on the host: a head divided by its root mean square, a pair as a complex number, turned by exp(i angle)."""
    case, page, rot = s["case"], s["case"]["page"], s["case"]["rot"]
    half = rot // 2
    first = np.arange(0, rot, 2) if case["interleaved"] else np.arange(half)
    second = first + (1 if case["interleaved"] else half)
    table = s["table"].cpu().numpy()
    places = np.concatenate([np.arange(m - n, m) for n, m in zip(s["new"], s["kv"])])
    seqs = np.concatenate([np.full(n, b) for b, n in enumerate(s["new"])])
    where = places if s["positions"] is None else s["positions"].cpu().numpy()
    freqs = np.array([THETA ** (-2.0 * i / rot) for i in range(half)], dtype=np.float64)
    turns = np.exp(1j * where[:, None].astype(np.float64) * freqs)

    def turned(x, weight):
        x = x.double().cpu().numpy()
        x = x / np.sqrt((x ** 2).sum(axis=2, keepdims=True) / x.shape[2] + EPS) * (weight.double().cpu().numpy() + case["offset"])
        z = (x[:, :, first] + 1j * x[:, :, second]) * turns[:, None, :]
        x[:, :, first], x[:, :, second] = z.real, z.imag
        return x

    q, k, v = turned(s["q"], s["q_weight"]), turned(s["k"], s["k_weight"]), s["v"].double().cpu().numpy()
    k_all, v_all = s["k_cache"].double().cpu().numpy(), s["v_cache"].double().cpu().numpy()
    k_all[table[seqs, places // page], :, places % page] = k
    v_all[table[seqs, places // page], :, places % page] = v
    return torch.from_numpy(q), torch.from_numpy(k_all), torch.from_numpy(v_all)


def _exact_logprobs(s):
    """Row by row: the likeliest by repeated search, the rest of the sum beside the largest's 1."""
    entropy, given, token, best = [], [], [], []
    V, n = s["logits"].shape[1], 0 if s["top_token"] is None else s["top_token"].shape[1]
    index = torch.arange(V, device=DEV)
    for r in range(s["logits"].shape[0]):
        x = s["logits"][r].double()
        top = int(torch.argmax(x))
        far = x - x[top]
        w = torch.exp(far)
        rest = w.sum() - 1.0 if float(w.sum()) > 1.5 else w[index != top].sum()
        logprob = far - torch.log1p(rest)
        entropy.append(torch.log1p(rest) - torch.where(w > 0, w * far, 0.0).sum() / (1.0 + rest))
        if s["given"] is not None:
            given.append(logprob[s["given"][r].long()])
        if n:
            # the n-th largest value splits the row; equal values by index
            m = min(n, V)
            edge = torch.topk(x, m).values[-1]
            above, at = index[x > edge], index[x == edge]
            kept = torch.cat((above, at[:m - above.numel()]))
            kept = kept[torch.sort(x[kept], descending=True, stable=True).indices]
            kept = kept[x[kept] > -math.inf]
            none = torch.full((n - kept.numel(),), -1, device=DEV)
            token.append(torch.cat((kept, none)).int())
            best.append(torch.cat((logprob[kept], torch.full((n - kept.numel(),), -math.inf, device=DEV, dtype=torch.float64))))
    outs = [torch.stack(entropy)]
    for part in (given, token, best):
        if part:
            outs.append(torch.stack(part))
    return outs
