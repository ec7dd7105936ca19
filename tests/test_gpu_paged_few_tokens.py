"""Probabilities in two parts: with few rows over rows as they are, and over codes where a sequence's rows see few tokens, whatever the
table has room for."""
import math

import pytest

pytestmark = pytest.mark.gpu
FORMATS = [("fp16", 16, 0), ("bf16", 16, 0), ("fp16", 8, 64), ("bf16", 8, 128), ("fp16", 4, 32), ("bf16", 4, 64)]


def _fine_errors(pool, sides, q, out, window=0):
    """Largest error over a bound that leaves no room for a probability rounded once.

    As attention_errors derives, h half a step of the type, but a probability p is its rounded value and the rest (at most h p) rounded
    again: off by h^2 p.  Parts of fp16 below its normal numbers are off by 2^-25 each instead, beside a largest probability of at least
    2^7: 2 n 2^-32 of the largest |v| in a sum over n tokens."""
    import torch
    from oracle import paged_oracle as O
    half = torch.finfo(pool.dtype).eps / 2
    tiny = torch.finfo(pool.dtype).smallest_normal * torch.finfo(pool.dtype).eps
    worst = 0.0
    for s, n in enumerate(pool.lengths):
        lo, hi = int(pool.starts[s]), int(pool.starts[s + 1])
        k, v = (pool.stands_for(side[s]) for side in sides)
        ref, _, mag, big = O.attend(q[lo:hi].cpu(), k, v, [n - (hi - r) for r in range(lo, hi)], True, window, 1 / math.sqrt(pool.d))
        e = ((pool.d + 1) * 2.0 ** -23 * big + 2.0 ** -21)[..., None]
        bound = half * ref.abs() + half * half * mag + (2 * e + 2 * n * 2.0 ** -23) * mag + 2 * n * 2.0 ** -32 * float(v.abs().max()) + tiny
        worst = max(worst, float(((out[lo:hi].cpu().double() - ref).abs() / bound).max()))
    return worst


def _contexts(pool):
    """Values that take turns in sign, so that what is left of them is far smaller than they are."""
    import torch
    sides = [[], []]
    for n in pool.lengths:
        sides[0].append(pool.draw(n, 0.5))
        v = torch.randn((n, pool.heads, pool.d), generator=pool.gen).abs() + 2
        sides[1].append((v * (1 - 2 * (torch.arange(n) % 2))[:, None, None]).to(pool.dtype))
    return sides


@pytest.mark.parametrize("dtype,bits,group", FORMATS)
@pytest.mark.parametrize("d,q_heads,rows", [(128, 2, 1), (128, 8, 4), (64, 4, 3)])
@pytest.mark.parametrize("room", [0, 40000])
def test_few_tokens_are_not_rounded_once(dtype, bits, group, d, q_heads, rows, room):
    import torch
    from paper_2403_05527_b200 import binding as G
    from tests import paged_harness as H
    group = min(group, d)
    lengths = [5, 40, 200]
    pool = H.Pool(G, lengths, [rows] * 3, dtype, bits, group, 16, 2, d, seed=rows, room=room)
    sides = _contexts(pool)
    pool.fill(sides)
    q = (torch.randn((pool.n_rows, q_heads, d), generator=pool.gen) * 0.2).to(pool.dtype).cuda()
    out = torch.full_like(q, 7.0)
    scratch = pool.scratch(G, q_heads)
    G.gear_paged_attn(pool.cache, q, out, pool.d_starts, scratch, max_rows=rows)
    assert G.gear_paged_status(scratch) == 0
    e = _fine_errors(pool, sides, q, out)
    assert e <= 1.0, e


@pytest.mark.parametrize("dtype,bits,group", FORMATS[2:])
def test_a_window_of_few_tokens_in_a_long_context(dtype, bits, group):
    import torch
    from paper_2403_05527_b200 import binding as G
    from tests import paged_harness as H
    pool = H.Pool(G, [3000], [2], dtype, bits, group, 16, 2, 128, seed=3)
    sides = _contexts(pool)
    pool.fill(sides)
    q = (torch.randn((2, 4, 128), generator=pool.gen) * 0.2).to(pool.dtype).cuda()
    out = torch.full_like(q, 7.0)
    scratch = pool.scratch(G, 4)
    G.gear_paged_attn(pool.cache, q, out, pool.d_starts, scratch, max_rows=2, window=30)
    assert G.gear_paged_status(scratch) == 0
    e = _fine_errors(pool, sides, q, out, 30)
    assert e <= 1.0, e


@pytest.mark.parametrize("dtype,bits,group", FORMATS)
@pytest.mark.parametrize("rows", [1, 4])
def test_a_wider_table_gives_the_same_bits(dtype, bits, group, rows):
    import torch
    from paper_2403_05527_b200 import binding as G
    from tests import paged_harness as H
    runs = []
    for room in (0, 2000, 40000):
        pool = H.Pool(G, [50], [rows], dtype, bits, group, 16, 2, 128, seed=7, room=room)
        sides = _contexts(pool)
        pool.fill(sides)
        q = (torch.randn((rows, 4, 128), generator=pool.gen) * 0.2).to(pool.dtype).cuda()
        out, lse = torch.full_like(q, 7.0), torch.zeros((rows, 4), device="cuda")
        scratch = pool.scratch(G, 4)
        G.gear_paged_attn(pool.cache, q, out, pool.d_starts, scratch, max_rows=rows, lse=lse)
        assert G.gear_paged_status(scratch) == 0
        runs.append((out, lse))
    for out, lse in runs[1:]:
        assert H.same_bits(out, runs[0][0]) and H.same_bits(lse, runs[0][1])
