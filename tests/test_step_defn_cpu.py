"""The generator against its authors' published answers, and what the mask's definition promises."""
import numpy as np

import step_defn as defn


def test_philox_gives_the_published_numbers():
    """Known answers of philox4x32-10 that its authors distribute with the paper."""
    f = 0xFFFFFFFF
    for counter, key, want in [
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((f, f, f, f), (f, f), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]:
        assert tuple(defn.philox(counter, key)) == want


def test_all_places_at_once_are_the_counters_one_by_one():
    seed, offset = 0x123456789ABCDEF0, 0xFEDCBA9876543210
    got = defn.numbers(3, 21, seed, offset, first_row=7)
    for r in range(3):
        for c in range(21):
            word = defn.philox((c // 8, 7 + r, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))[c % 8 // 2]
            assert got[r, c] == (word >> 16 if c % 2 else word & 0xFFFF)


def test_the_mask_keeps_what_it_should():
    m = defn.mask(200, 1000, 0.1, 1, 2).numpy()
    cut = 6554
    assert set(np.unique(m)) == {0.0, 65536 / (65536 - cut)}
    # 200000 places: the share kept is within five standard deviations, and so is the mean of what is left of ones
    assert abs((m > 0).mean() - (1 - cut / 65536)) < 5 * (0.09 / 200000) ** 0.5
    assert (defn.mask(4, 16, 0.0, 1, 2) == 1).all()
