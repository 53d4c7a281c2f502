"""Adapters, normed append, attention, sampling and log probabilities together, as the example's loop uses them."""
import os
import sys

import pytest
import torch

import paper_2506_12024_amd as fq

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
SMALL = dict(hidden=512, ffn=1024, heads=8, kv_heads=2, vocab=1000)


def test_the_loop_reports_what_it_draws_and_repeats():
    import decode_loop as loop
    more = dict(adapters=2, rank=16, normed=True, alternatives=5)
    _, _, first, report = loop.run(layers=2, batch=5, system=37, prompt=5, tokens=6, quiet=True, **more, **SMALL)
    _, _, again, _ = loop.run(layers=2, batch=5, system=37, prompt=5, tokens=6, quiet=True, **more, **SMALL)
    assert torch.equal(first, again) and first.min() >= 0 and first.max() < 1000
    lp, best, token = report["logprob"], report["top_logprob"], report["top_token"]
    assert torch.all(lp <= best[..., 0]) and torch.all(best[..., :-1] >= best[..., 1:]) and torch.all(lp < 0)
    same = token == first[..., None]  # a drawn token that is among the alternatives has the same log probability there
    assert same.any() and torch.equal(best[same], lp[..., None].expand_as(best)[same])


def test_log_probabilities_are_those_of_the_logits():
    import decode_loop as loop
    model = loop.Decoder(1, 2, 8, **SMALL)
    text = torch.randint(0, 1000, (6,), generator=torch.Generator().manual_seed(3)).cuda()
    seqs = fq.Sequences(loop.i32([0, 6]), loop.i32([6]), loop.i32([[0]]))
    logits = model.step(text, seqs, 6, 6)
    given = text.roll(-1)[:, None].int()  # a prompt scored: every token behind those before it
    lp = torch.empty((6, 1), device="cuda")
    fq.fq_logprobs_f16(logits, 6, 1000, torch.empty(fq.fq_logprobs_workspace_bytes(6, 1000), dtype=torch.uint8, device="cuda"), given=given, given_logprob=lp)
    want = torch.log_softmax(logits.double(), 1).gather(1, given.long())
    assert (lp - want).abs().max() < 1e-5


def test_steps_give_the_logits_of_one_chunk_and_requests_do_not_mix():
    """Four requests with adapters 1, none, 0 and 1, token by token and in one call: the same logits up to the roundings of two routes; a
    request without an adapter has the bits of a batch without adapters."""
    import decode_loop as loop
    system, n, batch = 37, 12, 4
    model = loop.Decoder(2, batch, 16, adapters=2, rank=8, normed=True, **SMALL)
    text = torch.randint(0, 1000, (system + batch * n,), generator=torch.Generator().manual_seed(3)).cuda()
    prefix = loop.i32([0, 1, 2])
    model.step(text[:system], fq.Sequences(loop.i32([0, system]), loop.i32([system]), prefix.view(1, -1)), system, system)
    slot, own = loop.i32([1, -1, 0, 1]), text[system:].view(batch, n)
    length, table = loop.i32([0] * batch), loop.i32([[3 + b] for b in range(batch)])
    one = fq.Sequences(loop.i32(list(range(batch + 1))), length, table, prefix, system)

    def by_token(which):
        rows = []
        for t in range(n):
            length.fill_(t + 1)
            rows.append(model.step(own[:, t], one, 1, n, which).clone())
        return torch.stack(rows, 1)
    steps, without = by_token(slot), by_token(None)
    assert torch.equal(steps[1], without[1])
    assert all(not torch.equal(steps[b], without[b]) for b in (0, 2, 3))
    length.fill_(n)
    chunks = fq.Sequences(loop.i32([b * n for b in range(batch + 1)]), length, table, prefix, system)
    chunk = model.step(text[system:], chunks, n, n, slot.repeat_interleave(n)).view(batch, n, -1).float()
    # 16-bit roundings along two layers: a few 2^-11 of the largest logit
    assert (steps.float() - chunk).abs().max() < 0.02 * chunk.abs().max()
