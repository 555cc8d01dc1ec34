"""OCP MXFP4 by definition, in float64: blocks of 32 elements share a power of two (E8M0), each element
an E2M1 code (sign, two exponent bits of bias 1, one mantissa bit; no infinity, no NaN).

A block with largest magnitude a gets the exponent floor(log2 a) - 2 (2: that of E2M1's largest
binade), here not below -125, and its elements the nearest E2M1 value of x / 2^e (ties to the even
code, at most 6).  Byte b of a scale is 2^(b - 127), 255 NaN; a block with a NaN or an infinity is NaN.

Layout of the library's pages: a (page, kv head) is a run of 16 rows of 64 bytes (element 2 i in the
low half of byte i), then of 16 rows of 4 scale bytes."""
import numpy as np

BLOCK, ROWS, DIM = 32, 16, 128
CODE_BYTES, SCALE_BYTES = DIM // 2, DIM // BLOCK
RUN = ROWS * (CODE_BYTES + SCALE_BYTES)


def e2m1_decode(codes):
    """Codes 0..15 -> float64, from their bit fields."""
    c = np.asarray(codes).astype(np.int64)
    sign, e, m = c >> 3, (c >> 1) & 3, c & 1
    mag = np.where(e == 0, m * 0.5, (1 + 0.5 * m) * 2.0 ** (e - 1))
    return np.where(sign == 1, -mag, mag)


def e2m1_encode(y):
    """float64 -> codes: the nearest magnitude, ties to the even code, saturating."""
    y = np.asarray(y, np.float64)
    a = np.minimum(np.abs(y), 6.0)
    grid = e2m1_decode(np.arange(8))
    best = np.zeros(a.shape, np.int64)
    dist = np.abs(a - grid[0])
    for c in range(1, 8):
        d = np.abs(a - grid[c])
        closer = (d < dist) | ((d == dist) & (c % 2 == 0))
        best, dist = np.where(closer, c, best), np.where(closer, d, dist)
    return (best + 8 * np.signbit(y)).astype(np.uint8)


def quantise(x):
    """x [..., 128] (float64) -> (codes uint8 [..., 128], scale bytes uint8 [..., 4])."""
    x = np.asarray(x, np.float64)
    b = x.reshape(x.shape[:-1] + (SCALE_BYTES, BLOCK))
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    _, e = np.frexp(np.abs(b).max(-1))                    # a = m 2^e with m in [1/2, 1): floor(log2 a) = e - 1
    e = np.where(np.abs(b).max(-1) == 0, -125, np.maximum(e - 3, -125))
    codes = np.where(bad[..., None], 0, e2m1_encode(np.ldexp(b, -e[..., None])))
    return codes.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def dequantise(codes, scales):
    """float64 values of codes [..., 128] and scale bytes [..., 4]."""
    scales = np.asarray(scales).astype(np.int64)
    power = np.where(scales == 255, np.nan, np.ldexp(1.0, scales - 127))
    v = e2m1_decode(codes).reshape(codes.shape[:-1] + (SCALE_BYTES, BLOCK)) * power[..., None]
    return v.reshape(codes.shape)


def pack(codes):
    """[..., 128] codes -> [..., 64] bytes."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(data):
    return np.stack([data & 15, data >> 4], -1).reshape(data.shape[:-1] + (DIM,))


def store(pool, page, slot, x):
    """Rows x [n][Hkv][128] into slots (page[i], slot[i]) of a pool [pages][Hkv][RUN], in place."""
    codes, scales = quantise(x)
    data = pack(codes)
    for i, (p, s) in enumerate(zip(page, slot)):
        pool[p, :, CODE_BYTES * s:CODE_BYTES * (s + 1)] = data[i]
        at = ROWS * CODE_BYTES + SCALE_BYTES * s
        pool[p, :, at:at + SCALE_BYTES] = scales[i]


def load(pool, page, slot):
    """(bytes [n][Hkv][68] of the slots, codes then scales; their values [n][Hkv][128])."""
    data = np.stack([pool[p, :, CODE_BYTES * s:CODE_BYTES * (s + 1)] for p, s in zip(page, slot)])
    scales = np.stack([pool[p, :, ROWS * CODE_BYTES + SCALE_BYTES * s:ROWS * CODE_BYTES + SCALE_BYTES * (s + 1)]
                       for p, s in zip(page, slot)])
    return np.concatenate([data, scales], -1), dequantise(unpack(data), scales)


def from_rows(pages):
    """A pool of values [pages][Hkv][16][128] -> [pages][Hkv][RUN] bytes."""
    codes, scales = quantise(pages)
    flat = pages.shape[:2]
    return np.concatenate([pack(codes).reshape(flat + (-1,)), scales.reshape(flat + (-1,))], -1)
