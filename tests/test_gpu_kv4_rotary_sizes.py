"""kv4_append with a rotated part of 8, 24, 40, .. channels, whose halves end inside eight channels (a half of a head of 48, 80 or 208, say):
codes, scales and values equal to the oracle's, queries within their roundings."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as K
from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.mark.parametrize("dtype", list(U))
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("tokens,heads,kv_heads,dim,turned,sections", [
    (1, 3, 2, 16, 8, None), (40, 5, 1, 48, 24, (3, 5, 4)), (33, 2, 2, 80, 40, None), (17, 4, 3, 208, 104, (20, 16, 16)), (9, 1, 1, 128, 120, None),
    (20, 2, 1, 256, 248, (100, 24)), (7107, 1, 1, 48, 24, None)])
def test_against_the_oracle(tokens, heads, kv_heads, dim, turned, sections, adjacent, dtype):
    g = torch.Generator().manual_seed(turned)
    x = (2.0 * torch.randn(tokens, heads + 2 * kv_heads, dim, generator=g)).to(dtype).cuda()
    q, k, v = x.split((heads, kv_heads, kv_heads), dim=1)
    turn = B.Rotary.of(turned, sections=sections, adjacent=adjacent)
    positions = torch.randint(0, 100000, (turn.axes, tokens), generator=g).int()
    page = 32
    cache = B.Kv4Cache(-(-tokens // page), page, kv_heads, dim, torch.tensor([9.0]).cuda())
    slots = torch.randperm(cache.n_pages * page, generator=g)[:tokens].int()
    k_values, v_values = (torch.empty(tokens, kv_heads, dim, device="cuda") for _ in range(2))
    out = B.kv4_append(k, v, cache, slots.cuda(), q=q, rotary=turn, positions=positions.cuda(), k_values=k_values, v_values=v_values)
    freq, axis = turn.freq.cpu().numpy(), None if turn.axis is None else turn.axis.cpu().numpy()
    rotate = lambda t: K.rotate(t.double().cpu().numpy(), positions.numpy(), freq, axis, adjacent)
    codes, scales, more, more_s = K.unpack(cache.codes.cpu().numpy(), cache.scales.cpu().numpy(), dim)
    p, o = slots.numpy() // page, slots.numpy() % page
    for which, (t, amax, values) in enumerate(((rotate(k), 9.0, k_values), (v.double().cpu().numpy(), None, v_values))):
        code, byte, value = K.quantize(t, amax)
        got = codes[p, which, :, o]
        assert np.array_equal(np.where(got & 7, got, 0), np.where(code & 7, code, 0)) and np.array_equal(scales[p, which, :, o], byte)
        assert np.array_equal(values.double().cpu().numpy(), value)
    assert not more.any() and not more_s.any()
    # as in the other sizes: the result's rounding, and binary32 products with rounded cosines where the type has 16 bits
    want, top = rotate(q), float(q.double().abs().max())
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= U[dtype] * np.abs(want) + 6 * 2.0 ** -24 * top + 2.0 ** -25)
    assert torch.equal(out[..., turned:], q[..., turned:])
    odd = torch.zeros(tokens, heads, dim + 3, dtype=dtype, device="cuda")[..., 1:dim + 1]
    odd.copy_(q)
    assert torch.equal(B.kv4_append(k, v, cache, slots.cuda(), q=odd, rotary=turn, positions=positions.cuda(), q_out=odd), out)


def test_sizes_that_are_refused():
    for pairs in (2, 6, 130):
        with pytest.raises(ValueError):
            B.Rotary(torch.ones(pairs, device="cuda"))
