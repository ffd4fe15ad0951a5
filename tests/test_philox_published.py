"""The generator against the words that its authors publish for seven rounds (the known answers beside Salmon et al., 2011), for counters and keys of zeros, of ones and of pi's digits."""
import numpy as np
import pytest

import philox

ONES = 0xFFFFFFFF
PI = (0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344, 0xA4093822, 0x299F31D0)


@pytest.mark.parametrize("counter,key,words", [((0,) * 4, (0,) * 2, (0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48)),
                                               ((ONES,) * 4, (ONES,) * 2, (0x5207DDC2, 0x45165E59, 0x4D8EE751, 0x8C52F662)),
                                               (PI[:4], PI[4:], (0x4DFCCABA, 0x190A87F0, 0xC47362BA, 0xB6B5242A))])
def test_published_words(counter, key, words):
    assert tuple(philox.words(counter, key)) == words
    if counter[0] == 0:                                                      # the whole rows' writing, whose counter's first word is the place over 8, its second the row
        got = philox.bits(1, 8, key[0] | key[1] << 32, counter[2] | counter[3] << 32, first_row=counter[1])
        assert np.array_equal(got[0], [w >> s & 0xFFFF for w in words for s in (0, 16)])
