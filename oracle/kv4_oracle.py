"""The 4-bit key-value cache in numpy binary64: block tables, rotary positions, the append and the attention that the
CUDA kernels are held to.  Shares no code with the GPU path; a block's scale and codes are those of fp4_oracle."""
import numpy as np

from oracle import fp4_oracle as F


def held(dim):
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def page_tables(past, new, table, free, page, rows, cursor=0):
    """(table, lengths, offsets, requests, positions, slots, next) token by token; -1 for what cannot be had."""
    table = np.array(table)
    lengths = [p + n for p, n in zip(past, new)]
    offsets = np.minimum(np.concatenate(([0], np.cumsum(new))), rows)
    requests, positions, slots = np.full(rows, -1), np.zeros(rows, dtype=np.int64), np.full(rows, -1)
    at, row = cursor, 0
    for i, (p, n) in enumerate(zip(past, new)):
        for q in range(-(-p // page), -(-(p + n) // page)):
            if q < table.shape[1]:
                table[i, q] = free[at] if at < len(free) else -1
            at += 1
        for t in range(p, p + n):
            if row < rows:
                entry = table[i, t // page] if t // page < table.shape[1] else -1
                requests[row], positions[row] = i, t
                slots[row] = entry * page + t % page if entry >= 0 else -1
            row += 1
    return table, np.array(lengths), offsets, requests, positions, slots, at


def rotate(x, positions, freq, axis=None, adjacent=False):
    """x [tokens, heads, dim], positions [axes, tokens], freq [pairs]; channels from 2 * pairs on stay."""
    x = np.array(x, dtype=np.float64)
    half = len(freq)
    for j in range(half):
        angle = np.asarray(positions, dtype=np.float64)[0 if axis is None else axis[j]] * freq[j]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        a, b = (2 * j, 2 * j + 1) if adjacent else (j, j + half)
        x[..., a], x[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return x


def quantize(x, amax=None):
    """codes uint8 [tokens, heads, dim], scale bytes [tokens, heads, dim / 16], values float64."""
    x = np.asarray(x, dtype=np.float64)
    n, h, d = x.shape
    code, byte, value = F.quantize(x.reshape(n * h, d), "nv", amax)
    return code.reshape(n, h, d), byte.reshape(n, h, d // 16), value.reshape(n, h, d)


def unpack(codes, scales, dim):
    """Codes [pages, 2, heads, page, dim] and scale bytes from the cache's buffers; what lies behind dim is returned too."""
    c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(*codes.shape[:-1], -1)
    return c[..., :dim], scales[..., :dim // 16], c[..., dim:], scales[..., dim // 16:]


def seen(length, n, causal=True, window=0):
    """[n, length] truth values: which positions the new tokens see."""
    own = length - n + np.arange(n)[:, None]
    place = np.arange(length)[None]
    see = place <= own if causal else np.ones((n, length), dtype=bool)
    return see & (place > own - window) if window else see


def attend(q, k, v, scale, causal=True, window=0):
    """q [n, heads, dim], k and v [length, kv_heads, dim].  Returns (o, spread): spread = sum of weight * |v|, what relative errors
    of the weights and of the sums are relative to.  What a row does not see has no part in it, NaN included."""
    n, heads, dim = q.shape
    length, kv_heads, _ = k.shape
    o, spread = np.zeros((n, heads, dim)), np.zeros((n, heads, dim))
    see = seen(length, n, causal, window)
    for j in range(n):
        at = np.flatnonzero(see[j])
        if not len(at):
            continue
        for h in range(heads):
            kh, vh = k[at, h // (heads // kv_heads)], v[at, h // (heads // kv_heads)]
            with np.errstate(invalid="ignore"):
                s = kh @ np.asarray(q[j, h], dtype=np.float64) * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                o[j, h], spread[j, h] = w @ vh, w @ np.abs(vh)
    return o, spread
