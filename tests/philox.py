"""Dropout's mask in plain numpy, for tests: ten rounds of Philox-4x32 as published (Salmon, Moraes, Dror, Shaw, 2011)."""
import numpy as np

LOW = np.uint64(0xFFFFFFFF)


def philox(counter, seed):
    """Four words (uint64 arrays below 2^32) for four counter words, under a seed of 64 bits."""
    x, y, z, w = counter
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = x * np.uint64(0xD2511F53), z * np.uint64(0xCD9E8D57)
        x, y, z, w = (b >> np.uint64(32)) ^ y ^ np.uint64(k0), b & LOW, (a >> np.uint64(32)) ^ w ^ np.uint64(k1), a & LOW
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return x, y, z, w


def kept(m, c, p, seed, offset, row0=0):
    """Which of m x c values are kept: 16 bits each, against p in 65536ths."""
    n = -(-c // 8)
    col, row = np.meshgrid(np.arange(n, dtype=np.uint64), np.arange(row0, row0 + m, dtype=np.uint64))
    words = philox([col, row, np.full_like(row, offset & 0xFFFFFFFF), np.full_like(row, offset >> 32)], seed)
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2)
    return (halves.reshape(m, n * 8)[:, :c] >= np.uint64(int(p * 65536 + 0.5)))
