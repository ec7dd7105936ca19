"""Scratch of the paged cache on another device than the current one, without a GPU: the calls that clear it and read its status word refuse
it, as the others do (the word would be read while its own device still works on it)."""
import pytest

from paper_2403_05527_b200 import binding as G


class Scratch:
    """What the binding asks a tensor for; its address is never read."""
    nbytes = 1 << 20

    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device

    def data_ptr(self):
        return 1 << 20

    def is_contiguous(self):
        return True


class Library:
    def __init__(self):
        self.calls = 0

    def gear_paged_scratch_init(self, *args):
        self.calls += 1
        return 0

    def gear_paged_status(self, *args):
        self.calls += 1
        return 0


@pytest.fixture
def library(monkeypatch):
    fake = Library()
    monkeypatch.setattr(G, "lib", lambda: fake)
    monkeypatch.setattr(G, "_current_device", lambda: 0)
    return fake


@pytest.mark.parametrize("device", [1, -1])
def test_other_devices_are_refused(library, device):
    with pytest.raises(ValueError):
        G.gear_paged_scratch_init(Scratch(device), stream=0)
    with pytest.raises(ValueError):
        G.gear_paged_status(Scratch(device))
    assert library.calls == 0


def test_the_current_device_is_taken(library):
    G.gear_paged_scratch_init(Scratch(0), stream=0)
    assert G.gear_paged_status(Scratch(0)) == 0 and library.calls == 2
