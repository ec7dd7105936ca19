"""Waits of the paged attention that run out: a test switch lets a warp wait, with a limit of a few dozen polls, on a barrier that nothing
completes, while its copies are under way.  The kernel returns by itself, the status word says so, and the next call is right."""
import pytest

pytestmark = pytest.mark.gpu


def _calls_around_a_dead_wait(which, rows, bits, group, d, q_heads=8):
    import torch
    from paper_2403_05527_b200 import binding as G
    from tests import paged_harness as H
    lengths = [900, 40, 0, 300]
    rows = [min(n, rows) for n in lengths]
    pool = H.Pool(G, lengths, rows, "fp16", bits, group, 16, 2, d, seed=bits)
    sides = [[pool.draw(n) for n in lengths] for _ in range(2)]
    pool.fill(sides)
    q = (torch.randn((pool.n_rows, q_heads, d), generator=pool.gen) * 0.3).half().cuda()
    scratch, want = pool.scratch(G, q_heads), torch.full_like(q, 7.0)
    G.gear_paged_attn(pool.cache, q, want, pool.d_starts, scratch, max_rows=max(rows))
    assert G.gear_paged_status(scratch) == 0
    e = H.attention_errors(pool, sides, q, want, None, True, 0, rows=list(range(0, pool.n_rows, 17)))
    assert max(e) <= 1.0, e
    got = torch.zeros_like(q)
    G.gear_paged_test_dead_wait(which)
    try:
        G.gear_paged_attn(pool.cache, q, got, pool.d_starts, scratch, max_rows=max(rows))
        assert G.gear_paged_status(scratch) == G.GEAR_ERR_TIMEOUT
        assert G.gear_paged_status(scratch) == 0                       # reading clears the word
    finally:
        G.gear_paged_test_dead_wait(0)
    G.gear_paged_scratch_init(scratch)
    for _ in range(2):
        got.fill_(7.0)
        G.gear_paged_attn(pool.cache, q, got, pool.d_starts, scratch, max_rows=max(rows))
        assert G.gear_paged_status(scratch) == 0 and H.same_bits(got, want)


@pytest.mark.parametrize("rows", [1, 4])
@pytest.mark.parametrize("bits,group,d", [(16, 0, 128), (16, 0, 64), (8, 64, 128), (4, 32, 128)])
def test_few_rows(rows, bits, group, d):
    _calls_around_a_dead_wait(1, rows, bits, group, d)


FORMS = [(16, 0, 128), (16, 0, 64), (8, 64, 128), (4, 32, 64)]


@pytest.mark.parametrize("which,bits,group,d", [(which, *form) for which in (2, 3, 4, 5, 6) for form in FORMS if which < 6 or form[0] < 16])
def test_many_rows(which, bits, group, d):
    """Warps of rows, copies of keys and values, copies of queries, products, conversion (of codes alone)."""
    _calls_around_a_dead_wait(which, 290, bits, group, d)
