"""Microscaled 4-bit floating point in numpy binary64: the definition the CUDA quantizer and products are held to.

Shares no code with the GPU path.  Every decision is taken by comparing |x| with (midpoint of two levels) * scale:
with at most 24 significant bits in x, 4 in a scale and 3 in a midpoint, and powers of two besides, both sides are
exact in binary64.
"""
import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = {"mx": 32, "nv": 16}


def e4m3_values():
    """Values of the 127 non-negative finite E4M3 bytes 0x00 .. 0x7e."""
    v = []
    for b in range(127):
        e, f = b >> 3, b & 7
        v.append(f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10))
    return np.array(v)


E4M3 = e4m3_values()


def nearest(a, table, scale):
    """Index of the entry of the rising `table` whose product with `scale` is nearest to a >= 0; a tie goes to the
    even index, anything beyond the last entry to the last."""
    mids = (table[1:] + table[:-1]) / 2.0
    idx = np.zeros(np.shape(a), dtype=np.int64)
    for k, m in enumerate(mids):                    # passes midpoint k: at least entry k + 1
        edge = m * scale
        idx += (a >= edge) if (k + 1) % 2 == 0 else (a > edge)
    return idx


def tensor_scale(amax):
    """2^max(ceil(log2(amax / 2688)), -100); 1 where amax is None, 0, infinite or NaN."""
    if amax is None or not (amax > 0.0) or not math.isfinite(amax):
        return 1.0
    e = math.frexp(amax)[1] - 12
    while 2688.0 * 2.0 ** e < amax:
        e += 1
    while 2688.0 * 2.0 ** (e - 1) >= amax:
        e -= 1
    return 2.0 ** max(e, -100)


def quantize(x, fmt, amax=None):
    """codes uint8 [rows, blocks * B] (sign in bit 3), scale bytes uint8 [rows, blocks], values float64 [rows, cols]."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    B = BLOCK[fmt]
    nb = -(-cols // B)
    z = np.zeros((rows, nb * B))
    z[:, :cols] = x
    z = z.reshape(rows, nb, B)
    bad = ~np.isfinite(z).all(axis=2)
    z = np.where(bad[..., None], 0.0, z)
    m = np.abs(z).max(axis=2)
    if fmt == "mx":
        e = np.frexp(m)[1] - 1                       # floor(log2 m) for m > 0
        byte = np.clip(np.where(m > 0, e - 2 + 127, 0), 0, 254)
        scale = 2.0 ** (byte - 127.0)
        byte = np.where(bad, 0xFF, byte)
    else:
        t = tensor_scale(amax)
        byte = nearest(m, E4M3, 6.0 * t)
        scale = E4M3[byte] * t
        byte = np.where(bad, 0x7F, byte)
    code = nearest(np.abs(z), LEVELS, scale[..., None])
    code = np.where(scale[..., None] == 0.0, 0, code)
    sign = (z < 0) | ((z == 0) & np.signbit(z))
    values = LEVELS[code] * np.where(sign, -1.0, 1.0) * scale[..., None]
    values = np.where(bad[..., None], np.nan, values)
    code = code + 8 * sign
    return (code.reshape(rows, nb * B).astype(np.uint8), byte.astype(np.uint8), values.reshape(rows, nb * B)[:, :cols])


def tile_rows(rows, offsets=None):
    """Scale tile row and row inside it for each row; the number of tile rows."""
    if offsets is None:
        r = np.arange(rows)
        return r // 128, r % 128, -(-rows // 128)
    tr, ir = np.full(rows, -1), np.full(rows, -1)
    for e in range(len(offsets) - 1):
        for r in range(offsets[e], offsets[e + 1]):
            tr[r], ir[r] = offsets[e] // 128 + e + (r - offsets[e]) // 128, (r - offsets[e]) % 128
    return tr, ir, rows // 128 + len(offsets) - 1


def untile_scales(buf, rows, nblk, offsets=None):
    """Scale bytes [rows, nblk] from the tiled buffer, by the layout's formula (rows of no group: 0)."""
    n4 = -(-nblk // 4)
    tr, ir, _ = tile_rows(rows, offsets)
    b = np.arange(nblk)
    at = ((tr[:, None] * n4 + b[None, :] // 4) * 512 + (ir[:, None] % 32) * 16 + (ir[:, None] // 32) * 4 + b[None, :] % 4)
    return np.where(tr[:, None] >= 0, np.asarray(buf)[np.where(tr[:, None] >= 0, at, 0)], 0)


def unpack(codes, cols):
    """Codes [rows, cols] from packed bytes [rows, ld]: even column in the low half."""
    c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(codes.shape[0], -1)
    return c[:, :cols]
