"""A long prompt with adapters through the example's decoder: every linear with an adapter takes several launches, in place."""
import os
import sys

import pytest
import torch

import paper_2506_12024_amd as fq

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
SMALL = dict(hidden=512, ffn=1024, heads=8, kv_heads=2, vocab=1000)


def test_long_prompts_have_the_logits_of_their_chunks():
    """Two prompts of 330 tokens with adapters 1 and 0 and one of 40 without, in one call and in chunks of 10: the same logits up to the
    roundings of the routes."""
    import decode_loop as loop
    model = loop.Decoder(2, 3, 80, adapters=2, rank=16, normed=True, **SMALL)
    lengths, slots = [330, 330, 40], [1, 0, -1]
    text = [torch.randint(0, 1000, (n,), generator=torch.Generator().manual_seed(n + i)).cuda() for i, n in enumerate(lengths)]
    table = loop.i32([[25 * b + p for p in range(25)] for b in range(3)])
    starts = [0, 330, 660, 700]
    whole = model.step(torch.cat(text), fq.Sequences(loop.i32(starts), loop.i32(lengths), table), 330, 330,
                       torch.cat([loop.i32([s] * n) for s, n in zip(slots, lengths)])).float()
    plain = model.step(torch.cat(text), fq.Sequences(loop.i32(starts), loop.i32(lengths), table), 330, 330).float()
    assert torch.equal(whole[660:], plain[660:]) and not torch.any(torch.all(whole[:660] == plain[:660], dim=1))
    for b in range(3):
        rows = []
        for t in range(0, lengths[b], 10):
            one = fq.Sequences(loop.i32([0, 10]), loop.i32([t + 10]), table[b:b + 1].contiguous())
            rows.append(model.step(text[b][t:t + 10], one, 10, 340, loop.i32([slots[b]] * 10)).clone())
        part = torch.cat(rows).float()
        # 16-bit roundings along two layers: a few 2^-11 of the largest logit
        assert (part - whole[starts[b]:starts[b + 1]]).abs().max() < 0.02 * part.abs().max()
