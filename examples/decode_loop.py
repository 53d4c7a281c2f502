"""A decoder's token loop on this library: a batch of requests behind one shared system prompt.

Random weights of the 7B shapes (as many layers as asked for), every linear resident as INT8 and INT4 copies.  The system
prompt is processed once and its pages are shared by all requests; each request's own prompt goes through in one chunk; then
every token takes, per layer, one plan for q, k and v, ``fq_kv_append`` (rotary positions, keys and values into the paged
cache), ``fq_attend`` (the shared prefix read once for the batch), and the linears after it; the output layer's logits
give the entropy for the precision scheduler and the token through ``fq_sample``.  Norms and the gate are torch's.
With ``--adapters`` requests bring low-rank adapters of the q and v projections (the system prompt goes without, so that its
pages stay shared), with ``--normed`` the heads of q and k are normed before they are turned, with ``--alternatives`` every
drawn token is reported with its log probability and the likeliest others.

    python examples/decode_loop.py --layers 4 --batch 8 --system 300 --prompt 20 --tokens 32
    python examples/decode_loop.py --layers 4 --batch 8 --adapters 3 --normed --alternatives 5
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_12024_amd as fq  # noqa: E402

DEV = "cuda:0"


class Linear:
    """A weight's resident copies (4 and 8 bits) and its entry in the bit-width array."""

    def __init__(self, N, K, gen):
        w = (torch.randn((N, K), generator=gen, device=DEV) / math.sqrt(K)).half()
        self.N, self.layer = N, fq.Layer(N, K)
        for bits in (4, 8):
            c, s, z = fq.fq_packed_sizes(N, K, bits)
            copy = (torch.empty(c, dtype=torch.uint8, device=DEV), torch.empty(s // 4, dtype=torch.float32, device=DEV),
                    torch.empty(z, dtype=torch.uint8, device=DEV))
            fq.fq_quantize(w, N, K, bits, fq.FQ_GROUP, *copy)
            self.layer.attach(bits, *copy)

    def __call__(self, x, bits=8):
        y = torch.empty((x.shape[0], self.N), dtype=torch.float16, device=DEV)
        fq.fq_linear(self.layer, bits, x.contiguous(), x.shape[0], y)
        return y


def norm(x):
    x = x.float()
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).half()


class Decoder:
    def __init__(self, layers, batch, pages, page=16, hidden=4096, ffn=11008, heads=32, kv_heads=32, vocab=32000, seed=0,
                 adapters=0, rank=8, normed=False):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.vocab, self.page = heads, kv_heads, hidden // heads, vocab, page
        kv = kv_heads * self.dim
        shapes = dict(q=(hidden, hidden), k=(kv, hidden), v=(kv, hidden), o=(hidden, hidden), gate=(ffn, hidden), up=(ffn, hidden),
                      down=(hidden, ffn))
        self.layers = [{n: Linear(N, K, gen) for n, (N, K) in shapes.items()} for _ in range(layers)]
        self.embed = torch.randn((vocab, hidden), generator=gen, device=DEV).half()
        self.out = fq.Layer(vocab, hidden)
        self.out_w = (torch.randn((vocab, hidden), generator=gen, device=DEV) * 3.0 / math.sqrt(hidden)).half()
        self.out.attach(16, self.out_w)
        shape = (pages, kv_heads, page, self.dim)
        self.cache = [fq.KVCache(torch.empty(shape, dtype=torch.float16, device=DEV), torch.empty(shape, dtype=torch.float16, device=DEV))
                      for _ in range(layers)]
        self.freqs = torch.tensor(fq.fq_rope_freqs(self.dim, 10000.0), dtype=torch.float64, device=DEV)
        # the bit-widths of every linear, which the scheduler lowers layer by layer
        names = list(shapes)
        self.entry = {(i, n): i * len(names) + j for i in range(layers) for j, n in enumerate(names)}
        self.bits = torch.full((len(self.entry),), 8, dtype=torch.int32, device=DEV)
        # q, k and v of a layer for a whole batch: one plan, its widths read from the array when it runs
        self.x = torch.empty((batch, hidden), dtype=torch.float16, device=DEV)
        self.qkv = [torch.empty((batch, n), dtype=torch.float16, device=DEV) for n in (hidden, kv, kv)]
        self.plans = []
        for layer in self.layers:
            ws = torch.empty(fq.Plan.workspace_bytes(3), dtype=torch.uint8, device=DEV)
            self.plans.append(fq.Plan([layer[n].layer for n in "qkv"], [self.x] * 3, self.qkv, batch, ws))
        self.workspace = {}
        # slots of adapters for q and v, the weights of the heads' norms
        more = torch.Generator(device=DEV).manual_seed(seed + 1)

        def slots(N):
            a = (torch.randn((adapters, rank, hidden), generator=more, device=DEV) / math.sqrt(hidden)).half()
            return fq.Adapters(a, torch.randn((adapters, N, rank), generator=more, device=DEV).half(),
                               scales=torch.full((adapters,), 0.5, device=DEV))
        self.adapters = [dict(q=slots(hidden), v=slots(kv)) if adapters else {} for _ in range(layers)]
        self.norms = [tuple((1.0 + 0.2 * torch.randn(self.dim, generator=more, device=DEV)).half() for _ in "qk") if normed else None
                      for _ in range(layers)]

    def step(self, tokens, seqs, max_q, max_kv, adapter=None):
        """Logits of the rows `tokens` (one int64 for each new token of the batch), through every layer.  adapter: int32, the
        slot of each row's request or -1; None: no row has one."""
        T = tokens.numel()
        h = self.embed[tokens]
        single = T == self.x.shape[0] and T <= fq.FQ_MAX_DECODE_M
        for i, layer in enumerate(self.layers):
            x = norm(h)
            if single:
                self.x.copy_(x)
                at = self.entry[i, "q"]
                self.plans[i].run(self.bits[at:at + 3])
                q, k, v = self.qkv
            else:
                q, k, v = (layer[n](x) for n in "qkv")
            if adapter is not None:
                for n, y in (("q", q), ("v", v)):
                    slots, key = self.adapters[i][n], (n, T)
                    if key not in self.workspace:
                        self.workspace[key] = torch.empty(fq.fq_adapters_workspace_bytes(slots, T), dtype=torch.uint8, device=DEV)
                    fq.fq_adapters_add(slots, x, adapter, y, y, self.workspace[key])
            q, k, v = q.view(T, self.heads, self.dim), k.view(T, self.kv_heads, self.dim), v.view(T, self.kv_heads, self.dim)
            turned, mixed = torch.empty_like(q), torch.empty_like(q)
            if self.norms[i]:
                fq.fq_kv_append_normed(self.cache[i], seqs, q, k, v, turned, self.freqs, *self.norms[i])
            else:
                fq.fq_kv_append(self.cache[i], seqs, q, k, v, turned, self.freqs)
            key = (seqs, T, max_q)
            need = fq.fq_attend_workspace_bytes(self.cache[i], seqs, T, self.heads, max_q, max_kv)
            if key not in self.workspace or self.workspace[key].numel() < need:
                self.workspace[key] = torch.empty(need, dtype=torch.uint8, device=DEV)
            fq.fq_attend(self.cache[i], seqs, turned, mixed, self.dim ** -0.5, max_q, max_kv, self.workspace[key])
            h = h + layer["o"](mixed.view(T, -1))
            x = norm(h)
            h = h + layer["down"](torch.nn.functional.silu(layer["gate"](x).float()).half() * layer["up"](x))
        logits = torch.empty((T, self.vocab), dtype=torch.float16, device=DEV)
        fq.fq_linear(self.out, 16, norm(h), T, logits)
        return logits


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def run(layers=2, batch=4, system=100, prompt=10, tokens=8, temperature=0.8, top_k=50, top_p=0.95, seed=0, quiet=False,
        adapters=0, rank=8, normed=False, alternatives=0, **shapes):
    page = 16
    own_pages = -(-(prompt + tokens) // page)
    shared_pages = -(-system // page)
    model = Decoder(layers, batch, shared_pages + batch * own_pages, page, seed=seed, adapters=adapters,
                    rank=rank, normed=normed, **shapes)
    slot = i32([b % (adapters + 1) - 1 for b in range(batch)]) if adapters else None  # every (adapters + 1)-th request has none
    host = torch.Generator().manual_seed(seed)
    text = torch.randint(0, model.vocab, (system + batch * prompt,), generator=host).to(DEV)

    # the system prompt once, as a sequence of its own in the shared pages
    prefix = i32(list(range(shared_pages)))
    model.step(text[:system], fq.Sequences(i32([0, system]), i32([system]), prefix.view(1, -1)), system, system)

    # every request's own prompt behind it, in one call
    table = i32([[shared_pages + b * own_pages + p for p in range(own_pages)] for b in range(batch)])
    lengths = i32([prompt] * batch)
    chunk = fq.Sequences(i32([b * prompt for b in range(batch + 1)]), lengths, table, prefix, system)
    logits = model.step(text[system:], chunk, prompt, prompt,
                        slot.repeat_interleave(prompt) if adapters else None)[prompt - 1::prompt].contiguous()

    # token by token; the scheduler sees the first request's entropy
    seqs = fq.Sequences(i32(list(range(batch + 1))), lengths, table, prefix, system)
    order = i32([model.entry[i, n] for i in range(layers) for n in "qkv"])
    state = torch.empty(fq.fq_sched_state_bytes(4), dtype=torch.uint8, device=DEV)
    lower = torch.full_like(order, 4)  # (the state reads both arrays as long as it is used)
    fq.fq_sched_init(state, 4, 1e9, 1, order, lower, order.numel(), model.bits)
    R, V = batch, model.vocab
    entropy, token = torch.empty(R, device=DEV), torch.empty(R, dtype=torch.int32, device=DEV)
    ws = torch.empty(fq.fq_sample_workspace_bytes(R, V), dtype=torch.uint8, device=DEV)
    settings = dict(temperature=torch.full((R,), temperature, device=DEV), top_k=i32([top_k] * R), top_p=torch.full((R,), top_p, device=DEV))
    gen = torch.Generator(device=DEV).manual_seed(seed)
    report = dict(logprob=[], top_token=[], top_logprob=[])
    ws_report = torch.empty(fq.fq_logprobs_workspace_bytes(R, V), dtype=torch.uint8, device=DEV)
    drawn, begin = [], time.time()
    for t in range(tokens):
        fq.fq_entropy_kl_f16(logits, None, R, V, entropy, None)
        fq.fq_sched_step(state, entropy)
        fq.fq_sample_f16(logits, R, V, torch.rand(R, generator=gen, device=DEV), token, ws, **settings)
        drawn.append(token.clone())
        if alternatives:
            logprob, best = torch.empty(R, device=DEV), torch.empty((R, alternatives), device=DEV)
            others = torch.empty((R, alternatives), dtype=torch.int32, device=DEV)
            fq.fq_logprobs_f16(logits, R, V, ws_report, given=token, given_logprob=logprob, top_token=others, top_logprob=best)
            for name, value in zip(report, (logprob, others, best)):
                report[name].append(value)
        if t + 1 < tokens:
            lengths.add_(1)
            logits = model.step(token.long(), seqs, 1, prompt + tokens, slot)
    drawn = torch.stack(drawn, 1).cpu()
    report = {name: torch.stack(v, 1).cpu() for name, v in report.items() if v}
    if not quiet:
        print("%d requests behind %d shared tokens, %d layers: %.2f ms a token; %d linears lowered to 4 bits" % (
            batch, system, layers, (time.time() - begin) * 1e3 / tokens, int((model.bits == 4).sum())))
        for b in range(batch):
            print("request %d: %s" % (b, drawn[b].tolist()))
            if alternatives:
                print("  ln p %s, likeliest %s" % (["%.2f" % v for v in report["logprob"][b].tolist()], report["top_token"][b].tolist()))
    return (model, text, drawn, report) if alternatives else (model, text, drawn)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("layers", 2), ("batch", 4), ("system", 100), ("prompt", 10), ("tokens", 8), ("top-k", 50), ("seed", 0),
                          ("adapters", 0), ("rank", 8), ("alternatives", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--normed", action="store_true")
    ap.add_argument("--temperature", type=float, default=0.8)
    ap.add_argument("--top-p", type=float, default=0.95)
    run(**{k.replace("-", "_"): v for k, v in vars(ap.parse_args()).items()})
