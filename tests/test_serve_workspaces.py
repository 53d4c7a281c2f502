"""What fq_attend needs at a length against what the size call answered for a longer one, without a GPU: a refusal names what
the call needs."""
import random
import re

import paper_2506_12024_amd as fq
from paper_2506_12024_amd import binding as B
from test_serve_pins import FAKE, attend, kv, seqs


def need(c, s, T, heads, dim, max_q, max_kv):
    rc = attend(c, s, T=T, q=1 << 32, o=1 << 44, qs=heads * dim, os=heads * dim, heads=heads, max_q=max_q, max_kv=max_kv, n=255)
    assert rc == B.FQ_ERR_SHAPE
    has, needs = re.search(r"the workspace has (\d+) bytes, the call needs (\d+)", fq.fq_last_error()).groups()
    assert int(has) == 255
    return int(needs)


def test_a_size_is_enough_for_every_smaller_length():
    rng = random.Random(11)
    more = 0
    for _ in range(1500):
        dim, kv_heads = rng.choice([8, 64, 80, 96, 128, 136, 256]), rng.choice([1, 2, 4, 8, 32])
        heads = kv_heads * rng.choice([1, 2, 4, 8])
        n = rng.choice([1, 1, 2, 5, 40, 300])
        max_q = rng.choice([1, 1, 2, 7, 40, 700])
        T = max(max_q, rng.randint(n, n * max_q))
        prefix = rng.choice([0, 0, 30, 999, 9000])
        _, c = kv(heads=kv_heads, dim=dim, ps=1 << 16, hs=4096, ts=256)
        _, s = seqs(n=n, width=20000, prefix_table=FAKE if prefix else None, prefix=prefix)
        try:
            last = 0
            asked = sorted(rng.randint(1, 300000 if rng.random() < 0.5 else 3000) for _ in range(4))
            needed = []
            for m in asked:
                size = fq.lib.fq_attend_workspace_bytes(c, s, T, heads, max_q, m)
                assert size >= last, "a longer one asks for less"
                last = size
                needed += [need(c, s, T, heads, dim, max_q, k) for k in {m, m - m // 7, m // 2 + 1, rng.randint(1, m)}]
                assert 256 <= max(needed) <= size, (dim, heads, kv_heads, n, max_q, T, prefix, m)
            more += max(needed) > need(c, s, T, heads, dim, max_q, asked[-1])
        finally:
            fq.lib.fq_kv_destroy(c), fq.lib.fq_seqs_destroy(s)
    assert more > 50  # (a shorter length may need more: that is what the size has to cover)
