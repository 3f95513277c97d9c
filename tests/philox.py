"""Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random
numbers: as easy as 1, 2, 3", 2011) in numpy, and the masks made of it."""

import numpy as np

M32 = np.uint64(0xFFFFFFFF)


def philox(counter, key):
    """counter: four arrays (or numbers) of 32-bit words, key: two; the four words of the result."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)  # 32 x 32 bits: no overflow
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & M32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & M32]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def keep_mask(seed, step, worker, site, rows, cols, threshold):
    """Where worker's rows are kept: columns 8j .. 8j+7 of row i have the halves of the words of one counter."""
    seed, step, per = seed % 2 ** 64, step % 2 ** 64, -(-cols // 8)
    q = np.arange(rows * per, dtype=np.uint64)
    full = np.ones_like(q)
    words = philox((q & M32, (q >> np.uint64(32)) + np.uint64(worker << 16), full * np.uint64(step % 2 ** 32),
                    full * np.uint64(((step >> 32) % 2 ** 16 << 16) | site)), (seed % 2 ** 32, seed >> 32))
    u = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1)
    return u.reshape(rows, per * 8)[:, :cols] >= threshold
