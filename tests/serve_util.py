"""What the tests of the paged cache, of attention over it and of sampling share: batches with shuffled pages, and plain
references in 64 bits (whole numbers for the weights of sampling)."""
import math

import numpy as np
import torch

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = {t: torch.finfo(t).eps for t in TYPES.values()}


class Batch:
    """Sequences with `new` tokens each, `kv` tokens in the cache with them, over a pool of shuffled pages."""

    def __init__(self, new, kv, page, prefix=0, spare=3, width=None, seed=0):
        rng = np.random.default_rng(seed)
        self.new, self.kv, self.page, self.prefix = list(new), list(kv), page, prefix
        held = [-(-n // page) for n in kv]
        pre = -(-prefix // page)
        self.pages = sum(held) + pre + spare
        order = list(rng.permutation(self.pages))
        self.width = width or max(max(held), 1)
        self.table = np.full((len(new), self.width), order[-1] if spare else 0, dtype=np.int32)
        for b, n in enumerate(held):
            self.table[b, :n] = [order.pop(0) for _ in range(n)]
        self.prefix_table = np.array([order.pop(0) for _ in range(pre)], dtype=np.int32)
        self.q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.tokens = int(self.q_start[-1])

    def places(self):
        """(sequence, place) of every row."""
        return [(b, m - n + j) for b, (n, m) in enumerate(zip(self.new, self.kv)) for j in range(n)]

    def slots(self, b):
        """(pages, tokens in them, whether it is a hole) of the keys that sequence b has, prefix first."""
        i = np.arange(self.prefix)
        pages = [self.prefix_table[i // self.page]] if self.prefix else []
        slots = [i % self.page] if self.prefix else []
        i = np.arange(self.kv[b])
        pages.append(self.table[b, i // self.page])
        slots.append(i % self.page)
        pages, slots = np.concatenate(pages), np.concatenate(slots)
        hole = (pages < 0) | (pages >= self.pages)
        return np.where(hole, 0, pages), slots, hole

    def sequences(self, dev="cuda:0"):
        import paper_2506_12024_amd as fq
        t = [torch.from_numpy(np.ascontiguousarray(a)).to(dev) for a in
             (self.q_start, np.array(self.kv, dtype=np.int32), self.table, self.prefix_table)]
        return fq.Sequences(t[0], t[1], t[2], t[3] if self.prefix else None, self.prefix)


def pool(gen, pages, heads, page, dim, dtype, token_major=False, dev="cuda:0"):
    """[page][head][token][dim] view of normal values."""
    shape = (pages, page, heads, dim) if token_major else (pages, heads, page, dim)
    t = torch.randn(shape, generator=gen).to(dtype).to(dev)
    return t.permute(0, 2, 1, 3) if token_major else t


def turn(x, positions, freqs, rot, interleaved, amplitude=1.0):
    """x float64 [tokens][heads][dim] -> (turned, sum of the magnitudes that went into each value)."""
    half = rot // 2
    ang = positions.astype(np.float64)[:, None, None] * np.asarray(freqs)[None, None, :]
    c, s = np.cos(ang) * amplitude, np.sin(ang) * amplitude
    lo = np.arange(0, rot, 2) if interleaved else np.arange(half)
    hi = lo + (1 if interleaved else half)
    y, size = x.copy(), np.zeros_like(x)
    a, b = x[:, :, lo], x[:, :, hi]
    y[:, :, lo], y[:, :, hi] = a * c - b * s, b * c + a * s
    size[:, :, lo] = size[:, :, hi] = (np.abs(a) + np.abs(b)) * abs(amplitude)
    return y, size


def attend(batch, q, k, v, scale, max_kv=None):
    """float64 q [tokens][q_heads][dim], k and v [page][head][token][dim] -> out, lse and, for the tolerance, the sum of p |v|,
    the largest scale * sum |q| |k| and the sum of |v| over the keys a row sees."""
    T, Hq, D = q.shape
    group = Hq // k.shape[1]
    out, lse = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf)
    size, steep, mass = np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.zeros((T, Hq, D))
    for b, (n, m) in enumerate(zip(batch.new, batch.kv)):
        pages, slots, hole = batch.slots(b)
        for h in range(Hq):
            kk, vv = k[pages, h // group, slots], v[pages, h // group, slots]
            for j in range(n):
                own = max(m - n + j + 1, 0)
                if max_kv is not None:
                    own = min(own, max_kv)
                seen = np.nonzero(~hole[:batch.prefix + own])[0]
                t = batch.q_start[b] + j
                if not len(seen):
                    continue
                score = scale * (kk[seen] @ q[t, h])
                top = score.max()
                p = np.exp(score - top)
                lse[t, h] = top + math.log(p.sum())
                p /= p.sum()
                out[t, h] = p @ vv[seen]
                size[t, h] = p @ np.abs(vv[seen])
                steep[t, h] = abs(scale) * (np.abs(kk[seen]) @ np.abs(q[t, h])).max()
                mass[t, h] = np.abs(vv[seen]).sum(axis=0)
    return out, lse, size, steep, mass


def attend_tolerance(dtype, out, size, steep, mass, dim):
    """p is rounded to the type (half a step) before it meets v, and so is the result; a score is a binary32 sum of `dim`
    products and takes a few more roundings on its way into the exponential, and an error of a score is one of p's and of the
    sum's; binary16 weights under 2^-25 of the largest (1) vanish."""
    half = EPS[dtype] / 2
    score = 2.0 * (dim + 8) * 2.0 ** -24 * steep[..., None] + 2.0 ** -20
    tiny = 2.0 ** -25 * mass if dtype == torch.float16 else 0.0
    return half * (1 + half) * (np.abs(out) + size) + score * size + tiny + 2.0 ** -25


def lse_tolerance(lse, steep, dim, keys):
    return (dim + 8) * 2.0 ** -24 * steep + (16 + math.log2(keys + 1)) * 2.0 ** -24 * (1 + np.abs(lse))


def weights(logits, temperature):
    """Whole weights of a row: multiples of 2^-min(51, 62 - ceil(log2 V)) of the largest."""
    x = logits.astype(np.float64).copy()
    x[np.isnan(x)] = -np.inf
    x = x + 0.0
    unit = min(51, 62 - (len(x) - 1).bit_length())
    top = x.max()
    if top == np.inf:
        w = np.where(x == np.inf, 1.0, 0.0)
    else:
        with np.errstate(under="ignore"):
            w = np.exp((x - top) * (1.0 / np.float64(temperature)))
        w[x == -np.inf] = 0.0
        w[x == top] = 1.0
    return x, w, [int(v) for v in np.rint(w * 2.0 ** unit).astype(np.uint64)]


def draw(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probability) of one row; the arguments are binary32 values."""
    from fractions import Fraction
    x = logits.astype(np.float64)
    V = len(x)
    x = np.where(np.isnan(x), -np.inf, x)
    if x.max() == -np.inf:
        return -1, 0.0
    if not temperature > 0:
        return int(np.argmax(x)), 1.0
    x, w, whole = weights(logits, temperature)
    order = np.lexsort((np.arange(V), -x))
    if 0 < top_k < V:
        order = order[:top_k]
    if not top_p >= 1:
        total = sum(whole[i] for i in order)
        need = Fraction(float(top_p)) * total if top_p > 0 else 0
        run, n = 0, 0
        for i in order:
            run += whole[i]
            n += 1
            if run >= need and run > 0:
                break
        order = order[:n]
    if min_p > 0:
        order = [i for i in order if w[i] >= min(float(min_p), 1.0) and x[i] > -np.inf]
    kept = sorted(i for i in order if whole[i])
    total = sum(whole[i] for i in kept)
    need = Fraction(float(u)) * total if u > 0 else 0
    run, token = 0, kept[-1]
    for i in kept:
        run += whole[i]
        if run > need:
            token = i
            break
    return int(token), whole[token] / total
