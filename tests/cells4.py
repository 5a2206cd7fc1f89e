"""Plain definitions of the cell layers' operators in 64 bits, on numpy arrays:
values that 4-bit blocks stand for, the codes' place in memory, and the draws of
a dropout."""
import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def block_scale(block):
    """Exponent of the scale of one block (1-D, fp64), or None for a block of NaN."""
    if not np.isfinite(block).all():
        return None
    top = np.abs(block).max(initial=0.0)
    e = -127
    while 6.0 * 2.0 ** e < top:
        e += 1
    return e


def nearest_code(mag):
    """Code 0 .. 7 of a magnitude: the nearest level, the even code of two."""
    gap = np.abs(LEVELS - mag)
    best = np.flatnonzero(gap == gap.min())
    return int(best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1])


def quantise(x):
    """(values, codes [rows][blocks][32], scale bytes [rows][blocks]) of x [rows][cols]."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    blocks = -(-cols // 32)
    values = np.empty_like(x)
    codes = np.zeros((rows, blocks, 32), np.uint8)
    scales = np.zeros((rows, blocks), np.uint8)
    for r in range(rows):
        for b in range(blocks):
            part = x[r, 32 * b:32 * b + 32]
            e = block_scale(part)
            if e is None:
                scales[r, b] = 255
                values[r, 32 * b:32 * b + 32] = np.nan
                continue
            scales[r, b] = e + 127
            for k, v in enumerate(part):
                c = nearest_code(abs(v) * 2.0 ** -e)
                codes[r, b, k] = c | (8 if np.signbit(v) else 0)
                values[r, 32 * b + k] = np.copysign(LEVELS[c] * 2.0 ** e, v)
    return values, codes, scales


def packed(codes, scales):
    """The bytes of codes [groups][blocks][16][16] and scales [groups][blocks][16]
    as the library lays them out; rows past the last are 0."""
    rows, blocks, _ = codes.shape
    groups = -(-rows // 16)
    c = np.zeros((groups, blocks, 16, 16), np.uint8)
    s = np.zeros((groups, blocks, 16), np.uint8)
    for r in range(rows):
        c[r // 16, :, r % 16] = codes[r, :, 0::2] | codes[r, :, 1::2] << 4
        s[r // 16, :, r % 16] = scales[r]
    return c, s


def philox4x32(counter, key):
    """Philox4x32-10 by Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def draws(elements, seed, index):
    """32-bit draws of the element numbers `elements` (iterable of int)."""
    index %= 2 ** 64
    out = []
    for e in elements:
        c = (e // 4 % 2 ** 32, e // 4 >> 32, index % 2 ** 32, index >> 32)
        out.append(philox4x32(c, (seed % 2 ** 32, seed >> 32))[e % 4])
    return np.array(out, dtype=np.uint64)


def threshold(rate):
    return min(2 ** 32, int(np.floor(float(np.float32(rate)) * 2.0 ** 32)))
