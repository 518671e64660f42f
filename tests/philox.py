"""The generator of dropout's masks in whole numbers: Philox-4x32 with ten rounds."""

import numpy as np


def philox(block, offset, seed):
    """The four words of one block."""
    c = [block & 0xFFFFFFFF, block >> 32, offset & 0xFFFFFFFF, offset >> 32]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return tuple(c)


def kept(first, n, p, seed, offset):
    """Whether the values first .. first + n - 1 are kept, and the scale of those that are."""
    limit = int(np.floor(p * 65536 + 0.5))
    if p < 1:
        limit = min(limit, 65535)
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    keep, b = [], None
    for e in range(first, first + n):
        if e >> 3 != b:
            b = e >> 3
            words = philox(b, offset, seed)
        w = words[(e & 7) >> 1]
        keep.append((w >> 16 if e & 1 else w & 0xFFFF) >= limit)
    return np.array(keep, dtype=bool), 65536 / (65536 - limit) if limit < 65536 else 0.0
