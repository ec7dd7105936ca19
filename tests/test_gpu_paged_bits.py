"""What the bits of an attention over a paged cache may depend on: the sequence's own rows, not on whose rows lie beside them, on rows of
nobody, or on what ran before."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,group", [(16, 0), (8, 64)])
@pytest.mark.parametrize("heads,q_heads", [(1, 3), (2, 10), (1, 33)])
def test_many_rows_do_not_depend_on_neighbours(heads, q_heads, bits, group):
    """Head ratios that do not divide a tile of 128 query rows, a sequence that ends inside a tile: the rest of the tile holds the next
    sequence's rows, rows of nobody, and rows of a call before."""
    import torch
    from paper_2403_05527_b200 import binding as G
    from tests import paged_harness as H
    lengths, rows, pad = [1500, 700], [50, 30], 90
    pool = H.Pool(G, lengths, rows, "bf16", bits, group, 16, heads, 128, seed=q_heads)
    sides = [[pool.draw(n) for n in lengths] for _ in range(2)]
    pool.fill(sides)
    n = pool.n_rows
    base = (torch.randn((n + pad, q_heads, 128), generator=pool.gen) * 0.3).to(pool.dtype)
    scratch = pool.scratch(G, q_heads, n + pad)
    runs = []
    for neighbour, nobody, before in ((1.0, 1.0, 1.0), (20.0, 1.0, 1.0), (1.0, 40.0, 1.0), (1.0, 1.0, 40.0), (40.0, float("nan"), 20.0)):
        other = (base * before).cuda()
        out = torch.full((n + pad, q_heads, 128), 7.0, dtype=pool.dtype, device="cuda")
        lse = torch.zeros((n + pad, q_heads), device="cuda")
        G.gear_paged_attn(pool.cache, other, out, pool.d_starts, scratch, max_rows=50, lse=lse)
        q = base.clone()
        q[rows[0]:n] *= neighbour
        q[n:] *= nobody
        G.gear_paged_attn(pool.cache, q.cuda(), out, pool.d_starts, scratch, max_rows=50, lse=lse)
        assert G.gear_paged_status(scratch) == 0
        runs.append((out[:rows[0]].cpu(), lse[:rows[0]].cpu()))
        e = H.attention_errors(pool, sides, q, out[:n], lse, True, 0, rows=[0, 20, 49])
        assert max(e) <= 1.0, e
    for out, lse in runs[1:]:
        assert H.same_bits(out, runs[0][0]) and H.same_bits(lse, runs[0][1])


@pytest.mark.parametrize("bits,group", [(16, 0), (8, 64), (4, 32)])
def test_few_rows_do_not_depend_on_neighbours(bits, group):
    import torch
    from paper_2403_05527_b200 import binding as G
    from tests import paged_harness as H
    lengths, rows, pad = [1500, 700, 90], [2, 3, 1], 5
    pool = H.Pool(G, lengths, rows, "fp16", bits, group, 16, 2, 128, seed=bits)
    sides = [[pool.draw(n) for n in lengths] for _ in range(2)]
    pool.fill(sides)
    n = pool.n_rows
    base = (torch.randn((n + pad, 6, 128), generator=pool.gen) * 0.3).to(pool.dtype)
    scratch = pool.scratch(G, 6, n + pad)
    runs = []
    for neighbour, nobody in ((1.0, 1.0), (30.0, 1.0), (30.0, float("nan"))):
        q = base.clone()
        q[rows[0]:n] *= neighbour
        q[n:] *= nobody
        out, lse = torch.full_like(q, 7.0).cuda(), torch.zeros((n + pad, 6), device="cuda")
        G.gear_paged_attn(pool.cache, q.cuda(), out, pool.d_starts, scratch, max_rows=3, lse=lse)
        assert G.gear_paged_status(scratch) == 0
        assert (out[n:] == 7.0).all() and (lse[n:] == 0.0).all()
        runs.append((out[:rows[0]].cpu(), lse[:rows[0]].cpu()))
    for out, lse in runs[1:]:
        assert H.same_bits(out, runs[0][0]) and H.same_bits(lse, runs[0][1])
