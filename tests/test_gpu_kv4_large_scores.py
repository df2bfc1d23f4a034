"""Attention over the 4-bit cache with scores far beyond the exponential's range, where binary32 holds them in steps of ones and tens: weights stay
finite, and some token has one."""
import numpy as np
import pytest
import torch

from kv4_helpers import HALF, Batch

pytestmark = pytest.mark.gpu

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("more_tokens", [0, 1 << 20], ids=["narrow", "wide"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n_new", [1, 40, 130])
@pytest.mark.parametrize("power", range(20, 33))
def test_results_lie_among_the_values(monkeypatch, power, n_new, dtype, more_tokens, up):
    """Scores of 2^power and -2^power (in powers of two) that grow or fall along the cache by 0 to 48 steps of one.  A weight is only known
    to within the score's own rounding, so that any mean of the values may come out, and nothing else: values lie from 1 to 2, and one that
    has the largest score by far is taken alone: its weight, rounded to fp16 (2^-11), by itself, and a rounding of the result."""
    monkeypatch.setattr(Batch, "more_tokens", more_tokens)
    g = torch.Generator().manual_seed(power)
    levels = sorted(LEVELS * 2, reverse=not up)
    n = 100 * len(levels)
    k, v = torch.zeros(n, 1, 64), 1.0 + torch.rand(n, 1, 64, generator=g)
    k[..., :16], k[:, 0, 16], k[..., 17] = 6.0, torch.tensor(levels).repeat_interleave(100), 6.0
    for sign in (1.0, -1.0):
        b = Batch([n], [n_new], 2, 1, 64, 64, dtype, k=k, v=v, amax=False)
        b.q = torch.zeros_like(b.q)
        b.q[..., :16] = sign * 2.0 ** 13                 # 16 * 6 * 2^13: 0.75 * 2^20
        for small in (1.0, 0.25, 0.0625):
            b.q[..., 16] = small * 2.0 ** (20 - power) * 8.0
            values = b.values()[1]
            lo, hi = values.min(), values.max()
            got = b.run(scale=2.0 ** (power - 20) * float(np.log(2.0))).double().cpu().numpy()
            step = HALF[dtype]
            assert np.all((got >= lo * (1 - 2.0 ** -8 - step)) & (got <= hi * (1 + 2.0 ** -8 + step))), (sign, small, got.min(), got.max())
    alone = n - n_new - 50
    k[:, 0, 16], k[:, 0, 17], k[:, 0, 18] = 0.0, 6.0, 0.0
    k[alone, 0, :16] = -6.0
    b = Batch([n], [n_new], 2, 1, 64, 64, dtype, k=k, v=v, amax=False)
    b.q = torch.zeros_like(b.q)
    b.q[..., :16] = -2.0 ** 13
    got = b.run(scale=2.0 ** (power - 20)).double().cpu().numpy()
    want = np.broadcast_to(b.values()[1][alone], got.shape)
    assert np.all(np.abs(got - want) <= (2.0 ** -11 + HALF[dtype]) * 1.001 * want)
