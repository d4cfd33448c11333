"""The dropout mask from its definition: Philox 4x32 with 7 rounds, in NumPy's 64-bit
integers (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011)."""
import numpy as np

_M = (np.uint64(0xD2511F53), np.uint64(0xCD9E8D57))
_W = (0x9E3779B9, 0xBB67AE85)
_LOW = np.uint64(0xFFFFFFFF)


def philox(counter, key, rounds):
    """counter: four arrays of 32-bit values (uint64); key: two numbers."""
    c = [np.asarray(v, np.uint64) for v in counter]
    for r in range(rounds):
        k = [np.uint64((key[i] + r * _W[i]) & 0xFFFFFFFF) for i in range(2)]
        p = [c[0] * _M[0], c[2] * _M[1]]
        hi = [v >> np.uint64(32) for v in p]
        lo = [v & _LOW for v in p]
        c = [hi[1] ^ c[1] ^ k[0], lo[1], hi[0] ^ c[3] ^ k[1], lo[0]]
    return c


def threshold(p):
    """16-bit numbers below it keep an element."""
    return int(np.floor((1.0 - p) * 65536 + 0.5))


def keep(n, seed, step, site, p, first=0):
    """Truth value for each of n elements from `first` (a multiple of 8) on."""
    assert first % 8 == 0
    b = np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64)
    full = lambda v: np.full_like(b, v & 0xFFFFFFFF)
    w = philox((b & _LOW, b >> np.uint64(32), full(step), full(site)),
               (seed & 0xFFFFFFFF, seed >> 32), 7)
    half = np.stack([np.stack([v & np.uint64(0xFFFF), v >> np.uint64(16)], -1) for v in w], 1)
    return (half < threshold(p)).reshape(-1)[:n]
