"""Tables that are wrong where no row's look-up sees it: the append says so too."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,group", [(16, 0), (8, 64), (4, 32)])
def test_append_finds_what_is_wrong_with_tables(bits, group):
    import torch
    from paper_2403_05527_b200 import binding as G
    from tests import paged_harness as H
    lengths, rows = [60, 60, 60, 20] + [0] * 400, [20, 20, 20, 0] + [0] * 400
    pool = H.Pool(G, lengths, rows, "fp16", bits, group, 16, 2, 128, seed=4)
    sides = [[pool.draw(n) for n in lengths] for _ in range(2)]
    new = [torch.cat([x[n - r:] for x, n, r in zip(side, lengths, rows)]).cuda() for side in sides]
    scratch = pool.scratch(G, 2)

    def status(starts=None, changed=None):
        pool.d_starts.copy_(pool.starts if starts is None else torch.tensor(starts, dtype=torch.int32))
        pool.d_lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        for s, n in (changed or {}).items():
            pool.d_lengths[s] = n
        G.gear_paged_append(pool.cache, new[0], new[1], pool.d_starts, scratch)
        return G.gear_paged_status(scratch)

    assert status() == 0
    for side, (codes, par) in enumerate(pool.expected([[x[n - r:] for x, n, r in zip(side, lengths, rows)] for side in sides], only_rows=True)):
        assert H.same_bits(pool.codes[side], codes)
        assert par is None or H.same_bits(pool.params[side], par)
    rest = [60] * 401
    assert status([0, 40, 20, 60] + rest) == G.GEAR_ERR_STATE          # falls: the rows that fall back have another owner each
    assert status([0, 20, 40, 60, 61] + rest[1:]) == G.GEAR_ERR_STATE  # falls and stays
    assert status([5, 20, 40, 60] + rest) == G.GEAR_ERR_STATE          # does not begin at 0
    # sequences without rows
    assert status(changed={3: -1}) == status(changed={3: 65}) == status(changed={403: 2 ** 30}) == G.GEAR_ERR_STATE
    assert status(changed={403: -2 ** 31}) == G.GEAR_ERR_STATE
    assert status(changed={2: 19}) == G.GEAR_ERR_STATE                 # more rows than tokens
    assert status() == 0
