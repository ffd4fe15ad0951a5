"""The counter-based generator behind dropout, in Python's own whole numbers and, for whole matrices, in numpy's: what the kernels are held to."""
import numpy as np


def words(counter, key):
    """Philox4x32 of seven rounds (Salmon et al., 2011): four words from four words of a counter and two of a key."""
    x, k = list(counter), list(key)
    for _ in range(7):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(b >> 32) ^ x[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ x[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return x


def bits(M, K, seed, offset, first_row=0):
    """The 16 bits of every element of M rows of K."""
    mask = np.uint64(0xFFFFFFFF)
    units = (K + 7) // 8
    x = [np.broadcast_to(np.arange(units, dtype=np.uint64)[None, :], (M, units)),
         np.broadcast_to(np.arange(first_row, first_row + M, dtype=np.uint64)[:, None], (M, units)),
         np.full((M, units), offset & 0xFFFFFFFF, dtype=np.uint64), np.full((M, units), offset >> 32, dtype=np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(7):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)    # below 2^64: nothing is lost
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), b & mask, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k1), a & mask]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    halves = [h for v in x for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))]
    return np.stack(halves, axis=2).reshape(M, units * 8)[:, :K].astype(np.int64)


def threshold(p):
    return round(p * 65536)


def keep(M, K, p, seed, offset, first_row=0):
    return bits(M, K, seed, offset, first_row) >= threshold(p)


def kept_factor(p):
    return 65536 / (65536 - threshold(p)) if threshold(p) < 65536 else 0.0
