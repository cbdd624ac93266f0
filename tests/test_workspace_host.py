"""What the wrappers take as a workspace: its address goes to the kernels (no GPU needed)."""
import pytest
import torch

from paper_1907_01729_amd import _binding

DEV = torch.device("cuda", 0)


@pytest.mark.parametrize("bad", [torch.empty(256, dtype=torch.uint8), torch.empty(64), torch.empty(0), 4096, "none"])
def test_memory_of_the_host_is_refused(bad):
    with pytest.raises(TypeError):
        _binding._scratch(bad, 64, DEV)


class Elsewhere(torch.Tensor):
    """A tensor on the CPU that says that it lies on a GPU."""
    place = DEV

    @property
    def is_cuda(self):
        return True

    @property
    def device(self):
        return self.place


def as_if(t, place=DEV):
    t = t.as_subclass(Elsewhere)
    t.place = place
    return t


def test_other_devices_and_views_are_refused():
    with pytest.raises(ValueError):
        _binding._scratch(as_if(torch.empty(64, dtype=torch.uint8), torch.device("cuda", 1)), 64, DEV)
    with pytest.raises(ValueError):
        _binding._scratch(as_if(torch.empty(1, dtype=torch.uint8).expand(64)), 64, DEV)
    with pytest.raises(ValueError):
        _binding._scratch(as_if(torch.empty(16, 16, dtype=torch.uint8)[:, :8]), 64, DEV)


def test_what_fits_is_taken(monkeypatch):
    """By its bytes, whatever its type; what is too small or lies askew is replaced."""
    made = []
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda shape, device, dtype: made.append((shape, device, dtype)))
    for t in (empty(64, dtype=torch.uint8), empty(16), empty(4, 4), empty(1 << 12, dtype=torch.uint8)):
        assert t.data_ptr() % 16 == 0
        t = as_if(t)
        assert _binding._scratch(t, 64, DEV) is t
    assert not made
    for t in (empty(63, dtype=torch.uint8), empty(80, dtype=torch.uint8)[8:], empty(80, dtype=torch.uint8)[1:], None):
        assert _binding._scratch(None if t is None else as_if(t), 64, DEV) is None
    assert made == [((64,), DEV, torch.uint8)] * 4
