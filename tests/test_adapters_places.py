"""Places of a set of adapters that there are not, also numbers that a C int would take for others."""
import pytest
import torch

from paper_2406_02629_amd import Adapters, SSNet, SSNetError, binding


class Calls:
    """the library, with the packing noted instead of launched"""

    def __init__(self, lib):
        self._lib, self.packed = lib, []

    def __getattr__(self, name):
        return getattr(self._lib, name)

    def ssnet_pack_adapter(self, *args):
        self.packed.append(args)
        return 0


@pytest.mark.parametrize("index", [-1, 4, 1 << 31, 1 << 32, (1 << 32) + 1, -(1 << 32)])
def test_a_place_that_is_none_is_refused(index, monkeypatch):
    ss = SSNet(3, 1, device=None)
    held = Adapters(ss, 4, 16, 4, 10)
    monkeypatch.setattr(binding, "_device_tensor", lambda t, *args: t)
    ss.lib = Calls(ss.lib)
    a, b = torch.zeros((3, 16, 4), dtype=torch.int64), torch.zeros((3, 4, 10), dtype=torch.int64)
    with pytest.raises(SSNetError) as e:
        held.load(index, a, b)
    assert e.value.code == binding.EINVAL and not ss.lib.packed
    held.load(3, a, b)
    assert [call[2] for call in ss.lib.packed] == [3]
