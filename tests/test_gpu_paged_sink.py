"""Attention over a paged cache behind tokens that take nearly all of the sum and have no value of their own (attention sinks): the output
is that of the tail, whose probabilities lie far below the largest."""
import math

import pytest

pytestmark = pytest.mark.gpu

# tokens, how far the tail's scores lie below the sinks', their spread (powers of two)
EVERY = 80                                     # a sink every so many tokens, so that every warp and every part of a context meets them
TAILS = [(4096, 20.45, 0.0), (32768, 24.45, 0.3), (32768, 25.5, 1.0)]


@pytest.mark.parametrize("n,below,spread", TAILS)
@pytest.mark.parametrize("rows", [1, 3, 20])
@pytest.mark.parametrize("dtype,bits,group", [("fp16", 16, 0), ("fp16", 8, 64), ("fp16", 4, 32), ("bf16", 16, 0)])
def test_tail_behind_sinks(n, below, spread, rows, dtype, bits, group):
    import torch
    from paper_2403_05527_b200 import binding as G
    from tests import paged_harness as H
    d, q_heads = 128, 2
    pool = H.Pool(G, [n], [rows], dtype, bits, group, 64, 1, d, seed=rows)
    # queries of ones: a score is the sum of a key's channels over sqrt(d)
    k = torch.randn((n, 1, d), generator=pool.gen) * (spread * math.log(2))
    v = torch.randn((n, 1, d), generator=pool.gen) * 0.5 + 0.5
    k[::EVERY], v[::EVERY] = below * math.log(2) / math.sqrt(d), 0.0
    sides = [[x.to(pool.dtype)] for x in (k, v)]
    pool.fill(sides)
    q = torch.ones((rows, q_heads, d), dtype=pool.dtype, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.zeros((rows, q_heads), device="cuda")
    scratch = pool.scratch(G, q_heads)
    G.gear_paged_attn(pool.cache, q, out, pool.d_starts, scratch, max_rows=rows, lse=lse)
    assert G.gear_paged_status(scratch) == 0
    e = H.attention_errors(pool, sides, q, out, lse, True, 0, rows=[0, rows - 1])
    assert max(e) <= 1.0, e
