"""The example's token loop: what it draws is what the same text gives in one chunk without a cache of its own steps."""
import os
import sys

import pytest
import torch

import paper_2506_12024_amd as fq

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
SMALL = dict(hidden=512, ffn=1024, heads=8, kv_heads=2, vocab=1000)


def test_the_loop_runs_and_repeats():
    import decode_loop as loop
    model, _, first = loop.run(layers=2, batch=3, system=37, prompt=5, tokens=6, quiet=True, **SMALL)
    _, _, again = loop.run(layers=2, batch=3, system=37, prompt=5, tokens=6, quiet=True, **SMALL)
    assert int((model.bits == 4).sum()) == 1  # six tokens, a window of four: one linear was lowered
    assert torch.equal(first, again) and first.min() >= 0 and first.max() < 1000


def test_steps_give_the_logits_of_one_chunk():
    """A text behind a shared prefix, token by token and in one call: the same logits up to the roundings of two routes."""
    import decode_loop as loop
    system, n = 37, 20
    model = loop.Decoder(2, 1, 8, **SMALL)
    text = torch.randint(0, 1000, (system + n,), generator=torch.Generator().manual_seed(3)).cuda()
    prefix = loop.i32([0, 1, 2])
    model.step(text[:system], fq.Sequences(loop.i32([0, system]), loop.i32([system]), prefix.view(1, -1)), system, system)
    length = loop.i32([0])
    table = loop.i32([[3, 4]])
    one = fq.Sequences(loop.i32([0, 1]), length, table, prefix, system)
    steps = []
    for t in range(n):
        length.fill_(t + 1)
        steps.append(model.step(text[system + t:system + t + 1], one, 1, n))
    steps = torch.cat(steps).float()
    length.fill_(n)
    chunk = model.step(text[system:], fq.Sequences(loop.i32([0, n]), length, table, prefix, system), n, n).float()
    whole = fq.Sequences(loop.i32([0, system + n]), loop.i32([system + n]), loop.i32([[5, 6, 7, 3]]))
    plain = model.step(text, whole, system + n, system + n).float()[system:]
    # 16-bit roundings along two layers: a few 2^-11 of the largest logit
    top = chunk.abs().max()
    assert (steps - chunk).abs().max() < 0.02 * top and (plain - chunk).abs().max() < 0.02 * top
