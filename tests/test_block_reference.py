"""The dropout's reference generator against the published test vectors of Philox 4x32-10, and the layout of the numbers drawn from it."""
import numpy as np
import pytest

from block_reference import numbers16, philox

ONES = 0xFFFFFFFF


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((ONES,) * 4, (ONES,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_published_vectors(counter, key, words):
    assert philox([counter], key) == [words]


def test_layout():
    got = numbers16(3, 11, 0, 0)
    first = (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)
    assert got.shape == (3, 11) and got[0, :8].tolist() == [w >> s & 0xFFFF for w in first for s in (0, 16)]
    assert got[2, 8:].tolist() == numbers16(6, 8, 0, 0)[5, :3].tolist()
    assert np.array_equal(numbers16(2, 8, -1, -1), numbers16(2, 8, 2 ** 64 - 1, 2 ** 64 - 1))
