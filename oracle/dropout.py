"""The mask of include/tahq_dropout.h: Philox 4x32 in NumPy's 64-bit integers."""
import numpy as np

M = np.uint64(0xFFFFFFFF)
SHIFT = np.uint64(32)


def philox(counter, key, rounds=10):
    """counter: four arrays of 32-bit numbers, key: two numbers; four arrays."""
    c = [np.asarray(v, np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> SHIFT) ^ c[1] ^ np.uint64(k[0]), b & M, (a >> SHIFT) ^ c[3] ^ np.uint64(k[1]), a & M]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(p):
    return int(np.floor(np.float64(np.float32(p)) * 65536 + 0.5))


def kept(first, count, p, seed, offset):
    """Whether elements first .. first + count - 1 are kept."""
    e = np.arange(first, first + count, dtype=np.uint64)
    block = e // np.uint64(8)
    same = np.full_like(block, offset % (1 << 32)), np.full_like(block, offset >> 32)
    words = np.stack(philox((block & M, block >> SHIFT, *same), (seed % (1 << 32), seed >> 32)))
    place = (e % np.uint64(8)).astype(np.int64)
    word = words[place // 2, np.arange(count)]
    return np.where(place % 2 == 1, word >> np.uint64(16), word & np.uint64(0xFFFF)).astype(np.int64) >= threshold(p)


def scale(p):
    t = threshold(p)
    return np.float32(65536 / (65536 - t)) if t < 65536 else np.float32(0)
