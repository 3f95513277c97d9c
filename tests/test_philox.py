"""The tests' Philox 4x32-10 against the values published with it."""

import pytest

from tests.philox import keep_mask, philox


@pytest.mark.parametrize("counter,key,want", [
    ((0,) * 4, (0,) * 2, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_published_values(counter, key, want):
    assert tuple(int(v) for v in philox(counter, key)) == want


def test_a_mask_goes_by_place_alone():
    wide, narrow = keep_mask(5, 6, 1, 2, 9, 40, 20000), keep_mask(5, 6, 1, 2, 4, 40, 20000)
    assert (wide[:4] == narrow).all() and not (keep_mask(5, 6, 2, 2, 9, 40, 20000) == wide).all()
