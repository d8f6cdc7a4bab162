"""CPU: which addresses a set of caches has."""
import pytest

from paper_2505_02351_amd.pages import _places


def test_each_address_once_in_order():
    assert _places([4096, 64, 1 << 40, 64, 4096], 1024) == [4096, 64, 1 << 40]
    assert _places([0, 1024, 2048], 1024) == [0, 1024, 2048] and _places([16], 1 << 30) == [16] and _places([0, 0], 0) == [0]


@pytest.mark.parametrize("addresses,size", [([0, 1008], 1024), ([2048, 0, 1040, 1 << 20], 1040), ([5000, 4999, 5000], 1024)])
def test_overlaps_are_refused(addresses, size):
    with pytest.raises(ValueError, match="overlap"):
        _places(addresses, size)
