"""The two writings of the generator that the dropout tests rely on agree, and its bits are spread as they should be."""
import numpy as np

import philox


def test_matrix_of_bits_is_that_of_single_counters():
    seed, offset = 0x0123456789ABCDEF, 0xFEDCBA9876543210
    got = philox.bits(3, 21, seed, offset, first_row=7)
    for r in range(3):
        for k in range(21):
            w = philox.words((k // 8, 7 + r, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))[k % 8 // 2]
            assert got[r, k] == (w >> 16 if k % 2 else w & 0xFFFF)


def test_share_of_kept_elements():
    """Of n elements the kept ones are off by six standard deviations, sqrt(n p (1 - p)), once in 10^8 draws; the seeds are fixed."""
    n = 512 * 4096
    for seed, p in ((1, 0.1), (2, 0.5), (3, 0.9)):
        q = philox.threshold(p) / 65536
        kept = philox.keep(512, 4096, p, seed, 5).sum()
        assert abs(kept - n * (1 - q)) < 6 * (n * q * (1 - q)) ** 0.5
    a, b = philox.keep(512, 4096, 0.5, 1, 5), philox.keep(512, 4096, 0.5, 1, 6)
    assert abs((a == b).sum() - n / 2) < 6 * (n / 4) ** 0.5                  # another offset: other elements
    assert np.array_equal(philox.keep(4, 64, 0.0, 1, 5), np.ones((4, 64), dtype=bool)) and not philox.keep(4, 64, 1.0, 1, 5).any()
