"""Philox4x32-10 on the host (Salmon, Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3, 2011), in numpy."""
import numpy as np

MASK = np.uint64(0xffffffff)


def philox(counter, key):
    """counter: four, key: two arrays of 32-bit numbers; four arrays."""
    c0, c1, c2, c3 = (np.asarray(v, dtype=np.uint64) for v in counter)
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = (b >> np.uint64(32)) ^ c1 ^ np.uint64(k0), b & MASK, (a >> np.uint64(32)) ^ c3 ^ np.uint64(k1), a & MASK
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return c0, c1, c2, c3


def pieces(seed, step, rows, cols, first_row=0):
    """[rows x cols] pieces of 16 bits, as tl_dropout numbers them."""
    blocks = -(-cols // 8)
    c = np.broadcast_to(np.arange(blocks), (rows, blocks))
    r = np.broadcast_to(np.arange(first_row, first_row + rows)[:, None], (rows, blocks))
    full = lambda v: np.full((rows, blocks), v, dtype=np.uint64)
    words = philox((c, r, full(step & 0xffffffff), full(step >> 32)), (seed & 0xffffffff, seed >> 32))
    out = np.stack([part for w in words for part in (w & np.uint64(0xffff), w >> np.uint64(16))], axis=2)
    return out.reshape(rows, 8 * blocks)[:, :cols]
