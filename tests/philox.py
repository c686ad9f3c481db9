"""The masks of dropout in numpy, from the definition: Philox 4x32 with ten rounds (Salmon et al., SC 2011), 16 bits for each of eight
columns of a row."""
import numpy as np

M32 = (1 << 32) - 1


def philox(counter, key):
    """counter: four arrays of 32-bit values in uint64; key: two numbers."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & np.uint64(M32), (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & np.uint64(M32)]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return c


def border(p):
    return int(np.rint(p * 65536))


def factor(p):
    t = border(p)
    return 65536 / (65536 - t) if t < 65536 else 0.0


def kept(p, seed, number, rows, cols, first_row=0):
    """True where an element of rows first_row .. is kept."""
    blocks = -(-cols // 8)
    i = np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None]
    j = np.arange(blocks, dtype=np.uint64)[None]
    number %= 1 << 64
    seed %= 1 << 64
    w = philox([j + 0 * i, i + 0 * j, np.uint64(number & M32) + 0 * (i + j), np.uint64(number >> 32) + 0 * (i + j)], (seed & M32, seed >> 32))
    halves = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], -1).reshape(rows, 8 * blocks)
    return halves[:, :cols] >= border(p)
