"""Which pools the binding of the paged cache takes, without a GPU: tensors of the host that say they are on a device."""
import pytest
import torch

from paper_2403_05527_b200 import binding as G

PAGES, HEADS, PAGE, D = 8, 2, 16, 128


class OnDevice(torch.Tensor):
    """A tensor whose address nobody reads."""
    is_cuda = property(lambda self: True)


def _on_device(*shape, dtype=torch.float16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


def _make(k, v, **more):
    table = _on_device(1, 4, dtype=torch.int32)
    lengths = _on_device(1, dtype=torch.int32)
    return G.make_paged(k, v, table, lengths, dtype=more.pop("dtype", torch.float16), page_size=PAGE, n_kv_heads=HEADS, head_dim=D, **more)


def test_pools_and_their_distances():
    page = HEADS * PAGE * D * 2
    k, v = (_on_device(PAGES, HEADS, PAGE, D) for _ in range(2))
    assert _make(k, v).struct.page_bytes == page
    both = _on_device(PAGES, 2, HEADS, PAGE, D)
    halves = _make(both[:, 0], both[:, 1]).struct
    assert (halves.n_pages, halves.page_bytes) == (PAGES, 2 * page)
    assert _make(k[:1], v[:1].expand(1, HEADS, PAGE, D)).struct.n_pages == 1


@pytest.mark.parametrize("side", [0, 1])
def test_pools_of_fewer_pages_than_they_count_are_refused(side):
    """Expanded pools, and pages that overlap."""
    whole = _on_device(PAGES, HEADS, PAGE, D)
    one = _on_device(1, HEADS, PAGE, D).expand(PAGES, HEADS, PAGE, D)
    over = _on_device(PAGES * HEADS * PAGE * D).as_strided((PAGES, HEADS, PAGE, D), (PAGE * D, PAGE * D, D, 1))
    for bad in (one, over):
        for pair in ((bad, bad), (bad, whole) if side == 0 else (whole, bad)):
            with pytest.raises(ValueError):
                _make(*pair)
    codes = [_on_device(PAGES, HEADS, PAGE, D, dtype=torch.uint8) for _ in range(2)]
    params = [_on_device(PAGES, HEADS, PAGE, D // 64, 2) for _ in range(2)]
    assert _make(*codes, bits=8, group=64, k_params=params[0], v_params=params[1]).struct.param_bytes == HEADS * PAGE * D // 64 * 4
    one = _on_device(1, HEADS, PAGE, D // 64, 2).expand(PAGES, HEADS, PAGE, D // 64, 2)
    with pytest.raises(ValueError):
        _make(*codes, bits=8, group=64, k_params=one, v_params=one)


def test_pools_of_another_type_are_refused():
    """Rows as they are in a pool of the other type of 16 bits would be read as numbers that they are not.  Bytes are taken for either."""
    k, v = (_on_device(PAGES, HEADS, PAGE, D, dtype=torch.bfloat16) for _ in range(2))
    assert _make(k, v, dtype=torch.bfloat16).struct.dtype == G.GEAR_BF16
    raw = [_on_device(PAGES, HEADS, PAGE, D * 2, dtype=torch.uint8) for _ in range(2)]
    assert _make(*raw, dtype=torch.bfloat16).struct.dtype == G.GEAR_BF16
    for pair in ((k, v), (k, raw[1]), (raw[0], v)):
        with pytest.raises(ValueError):
            _make(*pair, dtype=torch.float16)
