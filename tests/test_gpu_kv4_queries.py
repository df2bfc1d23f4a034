"""Queries that kv4_append rotates, in binary32: formed in binary64 and rounded once."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as K
from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,turned", [(1, 3, 64, 64), (200, 5, 80, 48), (3000, 2, 128, 128)])
def test_binary32_queries_are_rounded_once(tokens, heads, dim, turned, adjacent):
    """Half a step, 2^-24 of the result; in binary64 a cosine or sine of an angle up to 2^20 (2^-33 off, by the product's rounding, on both
    sides), two products and a sum."""
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn(tokens, heads + 2, dim, generator=g).cuda()
    positions = torch.randint(0, 1 << 20, (tokens,), generator=g).int().cuda()
    turn, slots = B.Rotary.of(turned, adjacent=adjacent), torch.full((tokens,), -1, dtype=torch.int32, device="cuda")
    got = B.kv4_append(x[:, :1], x[:, 1:2], B.Kv4Cache(1, 16, 1, dim), slots, q=x[:, 2:], rotary=turn, positions=positions).double().cpu().numpy()
    q = x[:, 2:].double().cpu().numpy()
    want = K.rotate(q, positions.cpu().numpy()[None], turn.freq.cpu().numpy(), adjacent=adjacent)
    pair = np.abs(K.rotate(q, np.zeros((1, tokens)), np.zeros(turned // 2), adjacent=adjacent)).max(-1, keepdims=True)
    assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -31 * pair)
