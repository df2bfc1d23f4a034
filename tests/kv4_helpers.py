"""Shared by the tests of the 4-bit key-value cache: batches with their pages, and the bound their results are held to."""
import numpy as np
import torch

from oracle import kv4_oracle as K
from paper_2309_15531_b200 import binding as B

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half a step, relative


class Batch:
    """Requests with `lengths` tokens in a cache, of which the last `new` are queries.  Pages in random order, some pages
    of nobody, memory that nothing was written to full of NaN scales."""
    more_tokens = 0                                      # that tables have room for: a longer reach takes small calls to other kernels

    def __init__(self, lengths, new, heads, kv_heads, dim, page=16, dtype=torch.bfloat16, seed=0, amax=True, loud=4.0, gap=0,
                 width_more=1, k=None, v=None):
        g = torch.Generator().manual_seed(seed)
        self.lengths_, self.new_, self.heads, self.kv_heads, self.dim, self.page = list(lengths), list(new), heads, kv_heads, dim, page
        counts = [-(-n // page) for n in lengths]
        self.n_pages, width = sum(counts) + 3, max(counts + [0]) + width_more
        if len(lengths) <= 300:
            width += self.more_tokens // page
        order = torch.randperm(self.n_pages, generator=g).tolist()
        table, at = torch.full((len(lengths), width), -7, dtype=torch.int32), 0
        for i, c in enumerate(counts):
            table[i, :c] = torch.tensor(order[at:at + c], dtype=torch.int32)
            at += c
        total, rows = sum(lengths), sum(new)
        x = torch.randn(2, total, kv_heads, dim, generator=g)
        x[0] *= torch.where(torch.rand(kv_heads, dim, generator=g) < 0.05, loud, 1.0)
        self.k = (x[0] if k is None else k).to(dtype).cuda()
        self.v = (x[1] if v is None else v).to(dtype).cuda()
        self.q = torch.randn(rows, heads + gap, dim, generator=g).to(dtype).cuda()[:, :heads]
        self.table = table.cuda()
        self.lengths = torch.tensor(lengths, dtype=torch.int32).cuda()
        self.offsets = torch.tensor(np.concatenate(([0], np.cumsum(new))), dtype=torch.int32).cuda()
        slots = [table[i, t // page].item() * page + t % page for i, n in enumerate(lengths) for t in range(n)]
        self.slots = torch.tensor(slots, dtype=torch.int32).cuda()
        self.amax = (B.absmax(self.k.reshape(total, -1)), B.absmax(self.v.reshape(total, -1))) if amax and total else (None, None)
        self.cache = B.Kv4Cache(self.n_pages, page, kv_heads, dim, *self.amax)
        self.cache.scales.fill_(0x7F)
        if total:
            B.kv4_append(self.k, self.v, self.cache, self.slots)

    def values(self):
        """Keys and values of the cache by the oracle, float64 [tokens, kv_heads, dim]."""
        return [K.quantize(x.double().cpu().numpy(), None if a is None else float(a.item()))[2]
                for x, a in zip((self.k, self.v), self.amax)]

    def want(self, scale=None, causal=True, window=0):
        """(o, bound) of all query rows.

        The bound, with u half a step of the result's type: u |o| for the one rounding; weights are rounded to fp16, 2^-11 relative
        (below 2^-14 of the largest 2^-25 absolute); a score is a binary32 sum of dim exact products whose terms the
        tensor core cuts off at 2^-22 of the sum of magnitudes for every 16 of them, then two roundings and an
        exponential within 2^-22, and it enters the weight and the sum of weights; the sum over tokens is cut off the same way for every
        16 tokens, with a few roundings where parts are joined."""
        kq, vq = self.values()
        q = self.q.double().cpu().numpy()
        scale = self.dim ** -0.5 if scale is None else scale
        o, bound = np.zeros(q.shape), np.zeros(q.shape)
        at = row = 0
        for n, m in zip(self.lengths_, self.new_):
            k, v = kq[at:at + n], vq[at:at + n]
            o[row:row + m], spread = K.attend(q[row:row + m], k, v, scale, causal, window)
            if n and m:
                most = np.nanmax(np.abs(v), initial=0.0)
                magnitude = np.abs(q[row:row + m]).max() * np.abs(np.nan_to_num(k)).sum(2).max() * abs(scale)
                score = (self.dim / 16 + 4) * 2.0 ** -22 * magnitude + 2.0 ** -21
                weight = 2.0 ** -11 + 2.0 * np.expm1(score)
                bound[row:row + m] = (HALF[self.q.dtype] * np.abs(o[row:row + m]) + (weight + (n / 16 + 32) * 2.0 ** -22) * spread
                                      + n * 2.0 ** -25 * most + 2.0 ** -24 * most)
            at, row = at + n, row + m
        return o, bound

    def run(self, **more):
        return B.kv4_attention(self.q, self.cache, self.table, self.lengths, self.offsets, **more)


def check(got, want, bound):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    off = np.abs(got - want) - bound
    worst = np.nanmax(off, initial=-1.0)
    assert worst <= 0, f"{worst} beyond the bound at {np.unravel_index(np.nanargmax(off), off.shape)}"
