"""What a decoder does between this library's linears, and after the output layer: its cases and plain forms.

Three operators: rotary positions with the append of keys and values to a paged cache (``append``),
attention over that cache, with a prefix that a batch may share (``attend``), and drawing the next token
from the logits (``sample``).  Head counts and widths are those of the 7B- and 70B-shaped stacks of
``synth`` (32 heads of 128; 64 query and 8 key heads of 128) and narrower heads; vocabularies are those
of the entropy workloads.

``run`` computes an operator in its plain form, elementary torch operations in 32 or 64 bits; with
``own`` set it makes the library's calls instead.  ``exact`` is a second writing in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
PLAIN, LINEAR, BASE, WAVELENGTH, RAMP = 0, 1, 2, 3, 4  # how rotary frequencies are scaled for long contexts


def listed():
    return [
        # one token of the 7B shapes goes into the cache: launch and latency
        dict(name="append_token_7b", kind="append", type="f16", seqs=1, new=1, kv=1000, q_heads=32, kv_heads=32,
             dim=128, rot=128, interleaved=False, scaling=PLAIN, page=16, token_major=False, fused=False, far=False),
        # a decode step of 32 sequences, grouped heads, frequencies scaled by wavelength for a long context
        dict(name="append_batch32_70b", kind="append", type="bf16", seqs=32, new=1, kv=1024, q_heads=64, kv_heads=8,
             dim=128, rot=128, interleaved=True, scaling=WAVELENGTH, page=16, token_major=False, fused=False, far=True),
        # chunks of nine prompts, narrow heads of which a quarter rotates, q, k and v in one row, pages token by token
        dict(name="append_chunks_80", kind="append", type="f16", seqs=9, new=300, kv=700, q_heads=32, kv_heads=32,
             dim=80, rot=20, interleaved=False, scaling=LINEAR, page=32, token_major=True, fused=True, far=False),
        # a long prompt of the 70B shapes
        dict(name="append_prompt_70b", kind="append", type="f16", seqs=1, new=2048, kv=2048, q_heads=64, kv_heads=8,
             dim=128, rot=128, interleaved=False, scaling=RAMP, page=64, token_major=False, fused=False, far=False),
        # one sequence decodes one token: launch and latency
        dict(name="attend_token_7b", kind="attend", type="f16", seqs=1, new=1, kv=777, prefix=0, q_heads=32,
             kv_heads=32, dim=128, page=16, token_major=False),
        # a batch of 16 sequences of all lengths, every head with keys of its own
        dict(name="attend_batch16_7b", kind="attend", type="f16", seqs=16, new=1, kv=4096, prefix=0, q_heads=32,
             kv_heads=32, dim=128, page=16, token_major=False),
        # 32 sequences with long histories, eight query heads to a key head
        dict(name="attend_batch32_70b", kind="attend", type="bf16", seqs=32, new=1, kv=16384, prefix=0, q_heads=64,
             kv_heads=8, dim=128, page=32, token_major=False),
        # 48 requests with one long system prompt and short histories of their own
        dict(name="attend_prefix_70b", kind="attend", type="f16", seqs=48, new=1, kv=512, prefix=8197, q_heads=64,
             kv_heads=8, dim=128, page=16, token_major=False),
        # a prompt's last chunk: 2048 new tokens behind 951 that are in the cache
        dict(name="attend_prompt_70b", kind="attend", type="f16", seqs=1, new=2048, kv=2999, prefix=0, q_heads=64,
             kv_heads=8, dim=128, page=64, token_major=False),
        # the next token of one sequence: launch and latency
        dict(name="sample_token", kind="sample", type="f32", rows=1, vocab=32000, mode="all"),
        # a batch whose requests bring settings of their own, logits as fq_linear leaves them
        dict(name="sample_batch32_f16", kind="sample", type="f16", rows=32, vocab=32000, mode="mixed"),
        # a large batch over a large vocabulary
        dict(name="sample_batch256", kind="sample", type="f32", rows=256, vocab=128256, mode="mixed"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "sample"])
    if kind == "sample":
        vocab = _log(rng, 100, 152064)
        return dict(kind="sample", type=rng.choice(["f32", "f16"]), rows=min(_log(rng, 1, 512), max(1, 30000000 // vocab)),
                    vocab=vocab, mode=rng.choice(["all", "mixed", "top_k", "top_p", "min_p", "temperature"]))
    dim = rng.choice([64, 80, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 32])
    q_heads = kv_heads * (rng.choice([1, 2]) if kv_heads == 32 else rng.choice([1, 2, 3, 4, 8]))
    case = dict(kind=kind, type=rng.choice(["f16", "bf16"]), q_heads=q_heads, kv_heads=kv_heads, dim=dim,
                page=rng.choice([8, 16, 32, 64, 128]), token_major=rng.random() < 0.3)
    if kind == "append":
        new = rng.choice([1, _log(rng, 1, 1500)])
        seqs = max(1, min(_log(rng, 1, 64), 4000 // new))
        kv = new + _log(rng, 1, 1000)
        rot = rng.choice([dim, dim, dim // 2, 20])
        case.update(seqs=seqs, new=new, kv=min(kv, new + 40000 * 8 // (seqs * kv_heads)), rot=rot,
                    interleaved=rng.random() < 0.5, scaling=rng.choice([PLAIN, LINEAR, BASE, WAVELENGTH, RAMP]),
                    fused=rng.random() < 0.4, far=rng.random() < 0.4)
    else:
        new = rng.choice([1, 1, rng.randint(2, 9), _log(rng, 10, 1500)])
        seqs = max(1, min(_log(rng, 1, 96), 3000 // new))
        prefix = rng.choice([0, 0, _log(rng, 1, 9000)])
        kv = new + _log(rng, 1, 16000)
        kv = max(new, min(kv, 1900000 // (seqs * kv_heads), 200000000 // (seqs * new * q_heads)))
        case.update(seqs=seqs, new=new, kv=kv, prefix=min(prefix, 300000000 // (seqs * new * q_heads)))
    return case


def _lengths(case):
    """(new tokens, length with them) of each sequence; the last one is the longest the case allows."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    new, kv = [], []
    for _ in range(case["seqs"] - 1):
        n = rng.randint(1, case["new"])
        new.append(n)
        kv.append(n + rng.randint(0, case["kv"] - case["new"]))
    return new + [case["new"]], kv + [case["kv"]]


def _scaling(case):
    return {PLAIN: {}, LINEAR: dict(factor=4.0), BASE: dict(factor=4.0),
            WAVELENGTH: dict(factor=8.0, low=1.0, high=4.0, original=8192),
            RAMP: dict(factor=16.0, low=1.0, high=32.0, original=4096)}[case["scaling"]]


def _amplitude(case):
    return 0.1 * math.log(16.0) + 1.0 if case["scaling"] == RAMP else 1.0


THETA = 10000.0


def _frequencies(case):
    """Radians per position of each rotating pair."""
    half, kind, s = case["rot"] // 2, case["scaling"], _scaling(case)
    base = THETA * s["factor"] ** (case["rot"] / (case["rot"] - 2)) if kind == BASE else THETA
    f = [base ** (-2.0 * i / case["rot"]) for i in range(half)]
    if kind == LINEAR:
        f = [v / s["factor"] for v in f]
    elif kind == WAVELENGTH:
        for i, v in enumerate(f):
            keep = (s["original"] * v / (2 * math.pi) - s["low"]) / (s["high"] - s["low"])
            keep = min(1.0, max(0.0, keep))
            f[i] = v * (keep + (1.0 - keep) / s["factor"])
    elif kind == RAMP:
        def pair(turns):  # the pair that makes so many turns over the original length
            return case["rot"] * math.log(s["original"] / (turns * 2 * math.pi)) / (2 * math.log(THETA))
        first, last = max(math.floor(pair(s["high"])), 0), min(math.ceil(pair(s["low"])), case["rot"] - 1)
        for i, v in enumerate(f):
            keep = 1.0 - min(1.0, max(0.0, (i - first) / max(last - first, 0.001)))
            f[i] = v * (keep + (1.0 - keep) / s["factor"])
    return f


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = random.Random(seed)
    if case["kind"] == "sample":
        return _prepare_sample(case, g, rng)
    dtype, page, heads, dim = TYPES[case["type"]], case["page"], case["kv_heads"], case["dim"]
    new, kv = _lengths(case)
    prefix = case.get("prefix", 0)
    held = [-(-n // page) for n in kv]
    prefix_pages = -(-prefix // page)
    pages = sum(held) + prefix_pages + 3
    order = list(range(pages))
    rng.shuffle(order)
    width = max(held) + 1
    table = torch.zeros((case["seqs"], width), dtype=torch.int32)
    for b, n in enumerate(held):
        table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    prefix_table = torch.tensor([order.pop() for _ in range(prefix_pages)], dtype=torch.int32)
    starts = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)

    def pool():
        shape = (pages, page, heads, dim) if case["token_major"] else (pages, heads, page, dim)
        t = torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, 1.0, generator=g)
        return t.permute(0, 2, 1, 3) if case["token_major"] else t  # [page][head][token][dim] either way

    s = dict(case=case, new=new, kv=kv, tokens=sum(new), max_q=max(new), max_kv=max(kv),
             q_start=starts.to(DEV), kv_len=torch.tensor(kv, dtype=torch.int32).to(DEV), table=table.to(DEV),
             prefix_table=prefix_table.to(DEV) if prefix else None, prefix=prefix, k_cache=pool(), v_cache=pool())
    T, Hq = s["tokens"], case["q_heads"]
    if case["kind"] == "append":
        if case["fused"]:
            row = torch.empty((T, Hq + 2 * heads, dim), dtype=dtype, device=DEV).normal_(0.0, 1.0, generator=g)
            s["q"], s["k"], s["v"] = row[:, :Hq], row[:, Hq:Hq + heads], row[:, Hq + heads:]
        else:
            s["q"], s["k"], s["v"] = (torch.empty((T, n, dim), dtype=dtype, device=DEV).normal_(0.0, 1.0, generator=g)
                                      for n in (Hq, heads, heads))
        s["q_out"] = torch.empty((T, Hq, dim), dtype=dtype, device=DEV)
        # positions of their own where the cache holds the end of a longer context
        s["positions"] = None
        if case["far"]:
            far = torch.tensor([rng.randint(10000, 120000) for _ in new], dtype=torch.int32)
            s["positions"] = torch.cat([torch.arange(n, dtype=torch.int32) + a for n, a in zip(new, far)]).to(DEV)
        s["freqs"] = torch.tensor(_frequencies(case), dtype=torch.float64).to(DEV)
    else:
        s["q"] = torch.empty((T, Hq, dim), dtype=dtype, device=DEV).normal_(0.0, 2.0, generator=g)
        s["out"] = torch.empty((T, Hq, dim), dtype=dtype, device=DEV)
        s["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=DEV)
    if own:
        import paper_2506_12024_amd as fq
        s["fq"] = fq
        s["cache"] = fq.KVCache(s["k_cache"], s["v_cache"])
        s["sequences"] = fq.Sequences(s["q_start"], s["kv_len"], s["table"], s["prefix_table"], prefix)
        if case["kind"] == "append":
            s["freqs"] = torch.tensor(fq.fq_rope_freqs(case["rot"], THETA, case["scaling"], **_scaling(case)),
                                      dtype=torch.float64).to(DEV)
        else:
            n = fq.fq_attend_workspace_bytes(s["cache"], s["sequences"], T, Hq, s["max_q"], s["max_kv"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return s


def _prepare_sample(case, g, rng):
    R, V = case["rows"], case["vocab"]
    logits = torch.empty((R, V), dtype=torch.float32, device=DEV).normal_(0.0, 3.0, generator=g)
    logits = logits.to(TYPES[case["type"]])

    def some(name, values, off):
        if case["mode"] not in ("all", "mixed", name):
            return off
        return rng.choice(values + ([off] if case["mode"] == "mixed" else []))

    rows = [(0.0 if case["mode"] == "mixed" and rng.random() < 0.1 else rng.choice([0.6, 0.8, 1.0, 1.2]),
             some("top_k", [1, 20, 50, 100, 1000], 0), some("top_p", [0.5, 0.8, 0.9, 0.95, 0.99], 1.0),
             some("min_p", [0.02, 0.05, 0.1], 0.0)) for _ in range(R)]
    t, k, p, m = zip(*rows)
    s = dict(case=case, logits=logits, temperature=torch.tensor(t, dtype=torch.float32).to(DEV),
             top_k=torch.tensor(k, dtype=torch.int32).to(DEV), top_p=torch.tensor(p, dtype=torch.float32).to(DEV),
             min_p=torch.tensor(m, dtype=torch.float32).to(DEV),
             u=torch.rand(R, dtype=torch.float32, device=DEV, generator=g),
             token=torch.empty(R, dtype=torch.int32, device=DEV),
             prob=torch.empty(R, dtype=torch.float32, device=DEV))
    if own:
        import paper_2506_12024_amd as fq
        s["fq"] = fq
        s["workspace"] = torch.empty(fq.fq_sample_workspace_bytes(R, V), dtype=torch.uint8, device=DEV)
    return s


def run(s):
    case = s["case"]
    if own:
        fq = s["fq"]
        if case["kind"] == "append":
            fq.fq_kv_append(s["cache"], s["sequences"], s["q"], s["k"], s["v"], s["q_out"], s["freqs"],
                            interleaved=case["interleaved"], amplitude=_amplitude(case), positions=s["positions"])
            return s["q_out"], s["k_cache"], s["v_cache"]
        if case["kind"] == "attend":
            fq.fq_attend(s["cache"], s["sequences"], s["q"], s["out"], 1.0 / math.sqrt(case["dim"]), s["max_q"],
                         s["max_kv"], s["workspace"], lse=s["lse"])
            return s["out"], s["lse"]
        call = fq.fq_sample if case["type"] == "f32" else fq.fq_sample_f16
        call(s["logits"], case["rows"], case["vocab"], s["u"], s["token"], s["workspace"], temperature=s["temperature"],
             top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], prob=s["prob"])
        return s["token"], s["prob"]
    return {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}[case["kind"]](s)


def _rotate(x, cos, sin, rot, interleaved):
    """x [tokens][heads][dim] in 32 bits; cos, sin [tokens][1][rot / 2]."""
    head, tail = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((turned, tail), dim=-1)


def _plain_append(s):
    case, page = s["case"], s["case"]["page"]
    t = torch.arange(s["tokens"], device=DEV)
    seq = torch.searchsorted(s["q_start"][1:].long(), t, right=True)
    place = s["kv_len"].long()[seq] - (s["q_start"].long()[seq + 1] - t)
    where = place if s["positions"] is None else s["positions"]
    angle = where.double()[:, None, None] * s["freqs"]
    cos, sin = (torch.cos(angle) * _amplitude(case)).float(), (torch.sin(angle) * _amplitude(case)).float()
    dtype = s["q"].dtype
    q = _rotate(s["q"].float(), cos, sin, case["rot"], case["interleaved"]).to(dtype)
    k = _rotate(s["k"].float(), cos, sin, case["rot"], case["interleaved"]).to(dtype)
    at = s["table"].long()[seq, place // page]
    s["k_cache"].permute(0, 2, 1, 3)[at, place % page] = k
    s["v_cache"].permute(0, 2, 1, 3)[at, place % page] = s["v"]
    return q, s["k_cache"], s["v_cache"]


def _plain_attend(s):
    case, page, dim, heads = s["case"], s["case"]["page"], s["case"]["dim"], s["case"]["kv_heads"]
    group = case["q_heads"] // heads
    outs, lses, at = [], [], 0
    for b, (n, m) in enumerate(zip(s["new"], s["kv"])):
        def states(cache):
            own_part = cache[s["table"][b, :-(-m // page)].long()].transpose(0, 1).reshape(heads, -1, dim)[:, :m]
            if not s["prefix"]:
                return own_part.float()
            shared = cache[s["prefix_table"].long()].transpose(0, 1).reshape(heads, -1, dim)[:, :s["prefix"]]
            return torch.cat((shared, own_part), dim=1).float()
        k, v = states(s["k_cache"]), states(s["v_cache"])
        q = s["q"][at:at + n].float().reshape(n, heads, group, dim).permute(1, 2, 0, 3).reshape(heads, group * n, dim)
        scores = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(dim))
        if n > 1:
            key, row = torch.arange(s["prefix"] + m, device=DEV), torch.arange(n, device=DEV)
            hidden = key[None, :] > (s["prefix"] + m - n + row)[:, None]
            scores = scores.view(heads, group, n, -1).masked_fill(hidden, -math.inf).view(heads, group * n, -1)
        top = scores.amax(dim=-1, keepdim=True)
        p = torch.exp(scores - top)
        total = p.sum(dim=-1, keepdim=True)
        o = torch.matmul(p, v) / total
        lse = (top + torch.log(total)).squeeze(-1)
        outs.append(o.view(heads, group, n, dim).permute(2, 0, 1, 3).reshape(n, heads * group, dim))
        lses.append(lse.view(heads, group, n).permute(2, 0, 1).reshape(n, heads * group))
        at += n
    return torch.cat(outs).to(s["q"].dtype), torch.cat(lses)


def _plain_sample(s):
    """Temperature, then the top_k largest, of these the fewest whose mass reaches top_p, of these the ones with
    min_p times the largest's; the first kept token, by index, where the running mass passes u times the whole."""
    V = s["case"]["vocab"]
    x, order = torch.sort(s["logits"].double(), dim=1, descending=True, stable=True)
    greedy = (s["temperature"] <= 0)[:, None]
    temperature = torch.where(greedy, 1.0, s["temperature"][:, None].double())
    w = torch.exp((x - x[:, :1]) / temperature)
    rank = torch.arange(V, device=DEV)[None, :]
    k = s["top_k"][:, None].long()
    keep = rank < torch.where(k > 0, k, V)
    mass = torch.cumsum(w * keep, dim=1)
    p = s["top_p"][:, None].double()
    keep &= (p >= 1.0) | (mass - w < p * mass[:, -1:]) | (rank == 0)
    keep &= w >= s["min_p"][:, None].double()
    keep = torch.where(greedy, rank == 0, keep)
    w = torch.zeros_like(w).scatter_(1, order, w * keep)  # by index again
    mass = torch.cumsum(w, dim=1)
    token = (mass <= s["u"][:, None].double() * mass[:, -1:]).sum(dim=1).clamp(max=V - 1)
    return token.int(), (w.gather(1, token[:, None]) / mass[:, -1:]).squeeze(1).float()


def work(case):
    if case["kind"] == "sample":
        size = 4 if case["type"] == "f32" else 2
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + case["rows"] * 28, "flops": 4 * n}
    new, kv = _lengths(case)
    T, dim = sum(new), case["dim"]
    if case["kind"] == "append":
        moved = T * (2 * case["q_heads"] + 4 * case["kv_heads"]) * dim * 2
        return {"bytes": moved + 8 * case["rot"] // 2 + 4 * T * case["far"] + 12 * case["seqs"],
                "flops": T * (case["q_heads"] + case["kv_heads"]) * case["rot"] * 3}
    keys = sum(kv) + case["prefix"]
    seen = sum(n * (m + case["prefix"]) - n * (n - 1) // 2 for n, m in zip(new, kv))
    return {"bytes": 4 * keys * case["kv_heads"] * dim + T * case["q_heads"] * (4 * dim + 4),
            "flops": 4 * seen * case["q_heads"] * dim}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["kind"]](s)


def _exact_append(s):
    """Token by token on the host: a pair as a complex number, turned by exp(i angle)."""
    case, page, rot = s["case"], s["case"]["page"], s["case"]["rot"]
    half = rot // 2
    freqs = np.array(_frequencies(case), dtype=np.float64)
    where = None if s["positions"] is None else s["positions"].cpu().numpy()
    table = s["table"].cpu().numpy()
    first = [2 * i for i in range(half)] if case["interleaved"] else list(range(half))
    second = [2 * i + 1 for i in range(half)] if case["interleaved"] else list(range(half, rot))

    def turned(x, turns):
        x = x.double().cpu().numpy()
        y = x.copy()
        z = (x[:, :, first] + 1j * x[:, :, second]) * turns[:, None, :]
        y[:, :, first], y[:, :, second] = z.real, z.imag
        return y

    places = np.concatenate([np.arange(m - n, m) for n, m in zip(s["new"], s["kv"])])
    seqs = np.concatenate([np.full(n, b) for b, n in enumerate(s["new"])])
    turns = _amplitude(case) * np.exp(1j * (places if where is None else where)[:, None].astype(np.float64) * freqs)
    q, k, v = turned(s["q"], turns), turned(s["k"], turns), s["v"].double().cpu().numpy()
    k_all, v_all = s["k_cache"].double().cpu().numpy(), s["v_cache"].double().cpu().numpy()
    for t, (b, at) in enumerate(zip(seqs, places)):
        k_all[table[b, at // page], :, at % page] = k[t]
        v_all[table[b, at // page], :, at % page] = v[t]
    return torch.from_numpy(q), torch.from_numpy(k_all), torch.from_numpy(v_all)


def _exact_attend(s):
    """Head by head: the weights are exp(score - log of the sum), the hidden keys are left out of the sum."""
    case, page, dim = s["case"], s["case"]["page"], s["case"]["dim"]
    group = case["q_heads"] // case["kv_heads"]
    out = torch.zeros((s["tokens"], case["q_heads"], dim), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["tokens"], case["q_heads"]), dtype=torch.float64, device=DEV)
    shared = torch.arange(s["prefix"], device=DEV)
    begin = 0
    for b, (n, m) in enumerate(zip(s["new"], s["kv"])):
        at = torch.arange(m, device=DEV)
        pages, slots = s["table"][b].long()[at // page], at % page
        if s["prefix"]:
            pages = torch.cat((s["prefix_table"].long()[shared // page], pages))
            slots = torch.cat((shared % page, slots))
        for h in range(case["q_heads"]):
            k = s["k_cache"][pages, h // group, slots].double()
            v = s["v_cache"][pages, h // group, slots].double()
            score = (s["q"][begin:begin + n, h].double() / math.sqrt(dim)) @ k.T
            if n > 1:
                score += torch.full_like(score, -math.inf).triu(s["prefix"] + m - n + 1)
            lse[begin:begin + n, h] = torch.logsumexp(score, dim=1)
            out[begin:begin + n, h] = torch.exp(score - lse[begin:begin + n, h, None]) @ v
        begin += n
    return out, lse


def _exact_sample(s):
    """Row by row on the host, keeping only what may be drawn."""
    V = s["case"]["vocab"]
    tokens, probs = [], []
    rows = zip(s["logits"].double().cpu().numpy(), s["temperature"].double().tolist(), s["top_k"].tolist(),
               s["top_p"].double().tolist(), s["min_p"].double().tolist(), s["u"].double().tolist())
    for x, temperature, k, p, m, u in rows:
        if temperature <= 0:
            tokens.append(int(np.argmax(x)))
            probs.append(1.0)
            continue
        order = np.lexsort((np.arange(V), -x))
        if k > 0:
            order = order[:k]
        w = np.exp((x[order] - x[order[0]]) / temperature)
        if p < 1.0:
            n = max(1, int(np.searchsorted(np.cumsum(w), p * np.cumsum(w)[-1], side="left")) + 1)
            order, w = order[:n], w[:n]
        order, w = order[w >= m], w[w >= m]
        by_index = np.argsort(order)
        order, w = order[by_index], w[by_index]
        mass = np.cumsum(w)
        i = min(int(np.searchsorted(mass, u * mass[-1], side="right")), len(order) - 1)
        tokens.append(int(order[i]))
        probs.append(float(w[i] / mass[-1]))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(probs, dtype=torch.float64)
