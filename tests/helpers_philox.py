"""Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011) in numpy's 64-bit whole numbers, and the mask that dropout documents."""
import numpy as np

LOW = np.uint64(0xffffffff)


def philox_4x32_10(counter, key):
    """counter: four arrays of words (uint64 holding 32 bits); key: two numbers.  Returns the block's four arrays of words."""
    a, b, c, d = counter
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(10):
        u, v = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b, c, d = (v >> np.uint64(32)) ^ b ^ np.uint64(k0), v & LOW, (u >> np.uint64(32)) ^ d ^ np.uint64(k1), u & LOW
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return a, b, c, d


def kept(first, count, p, seed, step, site):
    """Which of the elements first .. first + count - 1 dropout keeps, and the scale."""
    lo, hi = first // 8, -(-(first + count) // 8)
    group = np.arange(lo, hi, dtype=np.uint64)
    words = philox_4x32_10([group & LOW, group >> np.uint64(32), np.full_like(group, step & 0xffffffff), np.full_like(group, site)],
                           (seed & 0xffffffff, (seed >> 32) & 0xffffffff))
    halves = np.stack([h for w in words for h in (w & np.uint64(0xffff), w >> np.uint64(16))], 1).reshape(-1)
    limit = int(np.floor(float(np.float32(p)) * 65536 + 0.5))
    return halves[first - 8 * lo:][:count] >= limit, 65536.0 / (65536 - limit)
