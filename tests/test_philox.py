"""The tests' own generator against the known answers that its authors publish."""
import numpy as np
import pytest

from philox import kept, philox


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_known_answers(counter, key, words):
    assert tuple(int(w) for w in philox(counter, key)) == words


def test_share_of_kept_elements():
    """2^20 elements: within five standard deviations of 1 - p, in every column and for every p."""
    for p in (0.1, 0.5, 0.9):
        m = kept(np.arange(4096), 256, p, 12345, 6, 7).double()
        assert abs(float(m.mean()) - (1 - p)) < 5 * (p * (1 - p) / m.numel()) ** 0.5
        assert float((m.mean(0) - (1 - p)).abs().max()) < 6 * (p * (1 - p) / 4096) ** 0.5
