"""The generator of dropout by its definition, in Python's whole numbers and numpy's words."""
import numpy as np

WORD = 0xFFFFFFFF


def philox(counter, key, rounds):
    """One block, in whole numbers."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & WORD, (a >> 32) ^ c[3] ^ k[1], a & WORD]
        k = [(k[0] + 0x9E3779B9) & WORD, (k[1] + 0xBB67AE85) & WORD]
    return c


def border(p):
    return int(round(p * 65536))


def kept(n, p, seed, site, first=0):
    """Which of n elements from 8 * first on are kept, and the scale of those."""
    seed &= (1 << 64) - 1
    low, word = np.uint64(WORD), np.uint64(32)
    block = np.arange(first, first + -(-n // 8), dtype=np.uint64)
    c = [block & low, block >> word, np.full_like(block, site), np.zeros_like(block)]
    k0, k1 = seed & WORD, seed >> 32
    for _ in range(7):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> word) ^ c[1] ^ np.uint64(k0), b & low, (a >> word) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & WORD, (k1 + 0xBB67AE85) & WORD
    words = np.stack(c, 1)
    u = np.stack((words & np.uint64(0xFFFF), words >> np.uint64(16)), 2).reshape(-1)[:n]
    t = border(p)
    return u >= t, (65536.0 / (65536 - t) if t < 65536 else 0.0)
