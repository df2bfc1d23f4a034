"""Small weights of the attention over the 4-bit cache: tokens with nearly all the weight and values of zero, so that the result is what
the many others have."""
import math

import numpy as np
import pytest
import torch

from kv4_helpers import HALF, Batch
from oracle import kv4_oracle as K

pytestmark = pytest.mark.gpu

EVERY = 32                                               # so that every part of the work has one of the large ones


@pytest.mark.parametrize("tail", [23.51, 26.5])
@pytest.mark.parametrize("n,new,heads,kv_heads,dim,dtype,more_tokens", [
    # a cluster of CTAs; the line of few rows; the kernel for many rows, both tiles the same rows and a tile each
    (8000, 1, 4, 2, 64, torch.float16, 0), (9000, 1, 2, 1, 64, torch.float16, 0), (9000, 2, 6, 1, 128, torch.bfloat16, 0),
    (9000, 1, 2, 1, 256, torch.float16, 0), (9000, 40, 2, 1, 64, torch.float16, 1 << 20), (5000, 33, 1, 1, 128, torch.float16, 1 << 20),
    (5000, 33, 5, 1, 128, torch.bfloat16, 1 << 20)])
def test_many_small_weights_beside_large_ones(monkeypatch, n, new, heads, kv_heads, dim, dtype, more_tokens, tail):
    """Every 32nd token has the keys' only numbers: the others' weights are 2^-tail of its own.

    The bound, with u half a step of the result's type: u |o|; a weight is rounded to fp16 as 2^7 times what it is to the row's reference,
    which is some score of the row: 2^-11 relative, and where that is below 2^-14 half of fp16's least step, 2^-25.  The sum of weights is
    2^7 at least for every 32 tokens, so that this is 32 * 2^-32 of the largest value; a score's error as in kv4_helpers; sums 2^-22
    for every 16 tokens; results below 2^-14 have fp16's least step."""
    monkeypatch.setattr(Batch, "more_tokens", more_tokens)
    g = torch.Generator().manual_seed(n + dim)
    k, v = torch.zeros(n, kv_heads, dim), 1000.0 + 250.0 * torch.randn(n, kv_heads, dim, generator=g)
    k[::EVERY] = 1.0
    v[::EVERY] = 0.0
    b = Batch([n], [new], heads, kv_heads, dim, 64, dtype, k=k, v=v, amax=False)
    b.q = torch.ones_like(b.q)
    k, v = b.values()
    scale = tail * math.log(2.0) / float(np.abs(k[0, 0]).sum())
    got = b.run(scale=scale).double().cpu().numpy()
    want, spread = K.attend(b.q.double().cpu().numpy(), k, v, scale)
    score = (dim / 16 + 4) * 2.0 ** -22 * tail * math.log(2.0) + 2.0 ** -21
    bound = (HALF[dtype] * np.abs(want) + (2.0 ** -11 + 2.0 * np.expm1(score) + (n / 16 + 32) * 2.0 ** -22) * spread
             + EVERY * 2.0 ** -32 * np.abs(v).max() + (2.0 ** -25 if dtype == torch.float16 else 0.0))
    assert np.all(np.abs(got - want) <= bound), float((np.abs(got - want) / bound).max())
