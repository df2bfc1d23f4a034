"""Rotary positions and the quantizing append: codes, scales and values equal to the oracle's (decisions are those of the
rotation in binary64), rotated queries within their type's rounding."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as K
from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _case(tokens, heads, kv_heads, dim, rotary, adjacent, sections, dtype, page, seed=0, far=100000):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(tokens, heads + 2 * kv_heads, dim, generator=g) * 3
    qkv = qkv.to(DT[dtype]).cuda()
    axes = 1 if sections is None else len(sections)
    pos = torch.randint(0, far, (axes, tokens), generator=g, dtype=torch.int32)
    n_pages = -(-tokens // page) + 1
    slots = torch.randperm(n_pages * page, generator=g)[:tokens].int()
    return qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], pos, slots, n_pages


def _check_cache(cache, slots, k, v, amax, dim, same):
    """Codes and scales at the tokens' slots; everything else in the cache as it was."""
    codes, scales, more, more_s = K.unpack(cache.codes.cpu().numpy(), cache.scales.cpu().numpy(), dim)
    page = cache.page_size
    touched = np.zeros((cache.n_pages, page), dtype=bool)
    at = np.asarray(slots)
    inside = (at >= 0) & (at < cache.n_pages * page)
    p, o = at[inside] // page, at[inside] % page
    touched[p, o] = True
    for which, (x, a) in enumerate(((k, amax[0]), (v, amax[1]))):
        code, byte, _ = K.quantize(x[inside], a)
        got = codes[p, which, :, o]
        zero = (got & 7) == 0
        assert np.array_equal(np.where(zero, 0, got), np.where((code & 7) == 0, 0, code)), ("codes", which)
        assert np.array_equal(scales[p, which, :, o], byte), ("scales", which)
        assert not more[p, which, :, o].any() and not more_s[p, which, :, o].any()
    rest = ~touched
    assert bool((cache.codes.cpu().numpy().transpose(0, 3, 1, 2, 4)[rest] == same).all())
    assert bool((cache.scales.cpu().numpy().transpose(0, 3, 1, 2, 4)[rest] == same).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("tokens,heads,kv_heads,dim,rotary,adjacent,sections,page", [
    (1, 32, 32, 128, 128, False, None, 16),
    (7, 8, 1, 64, 64, False, None, 16),
    (50, 6, 3, 80, 48, True, None, 32),
    (33, 4, 2, 96, 96, False, (8, 20, 20), 16),
    (21, 5, 5, 16, 16, False, None, 1024),
    (40, 16, 2, 128, 64, True, (8, 12, 12), 64),
    (12, 3, 1, 256, 256, False, (32, 48, 48), 16),
    (9, 2, 2, 144, 112, False, (10, 20, 26), 16),
    (300, 12, 4, 128, 128, False, (16, 24, 24), 128)])
def test_against_the_oracle(tokens, heads, kv_heads, dim, rotary, adjacent, sections, page, dtype):
    q, k, v, pos, slots, n_pages = _case(tokens, heads, kv_heads, dim, rotary, adjacent, sections, dtype, page, seed=tokens)
    rot = B.Rotary.of(rotary, sections=sections, adjacent=adjacent)
    cache = B.Kv4Cache(n_pages, page, kv_heads, dim, k_amax=torch.tensor([14.0]).cuda(), v_amax=torch.tensor([2000.0]).cuda())
    cache.codes.fill_(0x5A)
    cache.scales.fill_(0x5A)
    vdt = torch.float32 if dtype == "f32" else torch.bfloat16
    kv, vv = (torch.full((tokens, kv_heads, dim), 7.0, dtype=vdt, device="cuda") for _ in range(2))
    out = B.kv4_append(k, v, cache, slots.cuda(), q=q, rotary=rot, positions=pos.cuda(), k_values=kv, v_values=vv)
    freq = 10000.0 ** (-np.arange(rotary // 2) / (rotary // 2))
    axis = None if sections is None else np.repeat(np.arange(len(sections)), sections)
    turned = K.rotate(k.double().cpu().numpy(), pos.numpy(), freq, axis, adjacent)
    _check_cache(cache, slots.numpy(), turned, v.double().cpu().numpy(), (14.0, 2000.0), dim, 0x5A)
    assert np.array_equal(kv.double().cpu().numpy(), K.quantize(turned, 14.0)[2])
    assert np.array_equal(vv.double().cpu().numpy(), K.quantize(v.double().cpu().numpy(), 2000.0)[2])
    # two products of a cosine or sine that was rounded, rounded, and a sum rounded: 3 halves of a step and a half of a b
    # each; then the result's rounding
    x = q.double().cpu().numpy()
    want = K.rotate(x, pos.numpy(), freq, axis, adjacent)
    top = np.abs(x).max()
    u = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= u * np.abs(want) + 6 * 2.0 ** -24 * top + 2.0 ** -25)
    assert np.array_equal(out.cpu()[..., rotary:].float().numpy(), q.cpu()[..., rotary:].float().numpy())


def test_without_rotation_and_without_an_amax():
    _, k, v, _, slots, n_pages = _case(37, 1, 3, 128, 0, False, None, "bf16", 16)
    cache = B.Kv4Cache(n_pages, 16, 3, 128)
    assert B.kv4_append(k, v, cache, slots.cuda()) is None
    _check_cache(cache, slots.numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(), (None, None), 128, 0)


def test_positions_of_zero_give_ties_and_far_ones_lose_nothing():
    """At position 0 the values stay on the grid of their type, where ties are frequent."""
    for far in (1, 2 ** 31 - 1):
        q, k, v, pos, slots, n_pages = _case(64, 2, 2, 64, 64, False, None, "bf16", 16, far=far)
        cache = B.Kv4Cache(n_pages, 16, 2, 64, k_amax=torch.tensor([2688.0]).cuda())
        B.kv4_append(k, v, cache, slots.cuda(), q=q, rotary=B.Rotary.of(64), positions=pos.cuda())
        turned = K.rotate(k.double().cpu().numpy(), pos.numpy(), 10000.0 ** (-np.arange(32) / 32))
        _check_cache(cache, slots.numpy(), turned, v.double().cpu().numpy(), (2688.0, None), 64, 0)


@pytest.mark.parametrize("turned", [False, True])
def test_every_decision_at_its_middle(turned):
    """Blocks whose largest value and whose elements lie on, just above and just below the middles of scales and levels (the
    rotation is by 0, so that they stay where they are)."""
    from oracle import fp4_oracle as F
    rows = []
    for b in range(1, 126, 3):
        for edge in (6 * F.E4M3[b], 3 * (F.E4M3[b] + F.E4M3[b + 1])):
            for top in (edge, np.nextafter(np.float32(edge), np.float32(0)), np.nextafter(np.float32(edge), np.float32(1e9))):
                s = F.E4M3[F.nearest(np.array([float(top)]), F.E4M3, 6.0)[0]]
                mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) * s
                below, above = np.nextafter(mids.astype(np.float32), np.float32(0)), np.nextafter(mids.astype(np.float32), np.float32(1e9))
                rows.append(np.concatenate(([top], mids, -below, [0.0])))
                rows.append(np.concatenate(([-top], -mids, above, [-0.0])))
    x = np.array(rows, dtype=np.float32)
    n = len(x) // 4
    k = torch.tensor(x[:4 * n].reshape(n, 1, 64)).cuda()
    cache = B.Kv4Cache(-(-n // 16), 16, 1, 64)
    slots = torch.arange(n, dtype=torch.int32)
    more = dict(rotary=B.Rotary.of(64), positions=torch.zeros(n, dtype=torch.int32).cuda()) if turned else {}
    B.kv4_append(k, k, cache, slots.cuda(), **more)
    _check_cache(cache, slots.numpy(), k.double().cpu().numpy(), k.double().cpu().numpy(), (None, None), 64, 0)


@pytest.mark.parametrize("turned", [False, True])
def test_extremes(turned):
    """Zeros, subnormal numbers, what saturates, infinities and NaN."""
    k = torch.zeros(8, 1, 64)
    k[1] = 1e-40
    k[2] = 3e38
    k[3, 0, :16] = 1e5
    k[4, 0, 5], k[4, 0, 40] = float("inf"), 1.0
    k[5, 0, 50] = float("nan")
    k[6] = 2.0 ** -12
    k[7, 0, ::2], k[7, 0, 1::2] = 448 * 6, -448 * 6
    k = k.cuda()
    cache, slots = B.Kv4Cache(1, 16, 1, 64), torch.arange(8, dtype=torch.int32)
    kv = torch.empty(8, 1, 64, device="cuda")
    more = dict(rotary=B.Rotary.of(32), positions=torch.zeros(8, dtype=torch.int32).cuda()) if turned else {}
    B.kv4_append(k, k, cache, slots.cuda(), k_values=kv, **more)
    x = k.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        y = K.rotate(x, np.zeros((1, 8)), 10000.0 ** (-np.arange(16) / 16)) if turned else x
    _check_cache(cache, slots.numpy(), y, x, (None, None), 64, 0)
    want, got = K.quantize(y)[2], kv.double().cpu().numpy()
    assert np.array_equal(np.isnan(want), np.isnan(got)) and np.array_equal(np.nan_to_num(want), np.nan_to_num(got))


def test_tokens_without_a_slot_are_not_stored():
    q, k, v, pos, slots, n_pages = _case(30, 2, 2, 64, 64, False, None, "bf16", 16)
    slots[3], slots[9], slots[20] = -1, n_pages * 16, 2 ** 31 - 1
    cache = B.Kv4Cache(n_pages, 16, 2, 64)
    cache.codes.fill_(0x33)
    cache.scales.fill_(0x33)
    out = B.kv4_append(k, v, cache, slots.cuda(), q=q, rotary=B.Rotary.of(64), positions=pos.cuda())
    turned = K.rotate(k.double().cpu().numpy(), pos.numpy(), 10000.0 ** (-np.arange(32) / 32))
    _check_cache(cache, slots.numpy(), turned, v.double().cpu().numpy(), (None, None), 64, 0x33)
    assert bool(out.any(-1).all())


def test_unaligned_and_strided_tensors_and_rotation_in_place():
    """Views that start at an odd element and have odd strides; q turned in place gives what a copy gives."""
    g = torch.Generator().manual_seed(4)
    flat = torch.randn(25 * 1001 + 1, generator=g).half().cuda()[1:]
    all_heads = flat.view(25, 1001)[:, :14 * 71].as_strided((25, 14, 64), (1001, 71, 1))
    q, k, v = all_heads[:, :8], all_heads[:, 8:11], all_heads[:, 11:]
    pos, slots = torch.arange(25, dtype=torch.int32).cuda() * 3, torch.arange(25, dtype=torch.int32).cuda()
    a, b = (B.Kv4Cache(2, 16, 3, 64) for _ in range(2))
    rot = B.Rotary.of(64, adjacent=False)
    one = B.kv4_append(k, v, a, slots, q=q, rotary=rot, positions=pos)
    two = B.kv4_append(k.contiguous(), v.contiguous(), b, slots, q=q.contiguous(), rotary=rot, positions=pos)
    assert torch.equal(one, two) and torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    wide = torch.empty(25, 9, 64, dtype=torch.float16, device="cuda").fill_(5)
    B.kv4_append(k, v, a, slots, q=q, rotary=rot, positions=pos, q_out=wide[:, :8])
    assert torch.equal(wide[:, :8], one) and bool((wide[:, 8] == 5).all())
    for adjacent in (False, True):
        rot = B.Rotary.of(48, adjacent=adjacent)
        want = B.kv4_append(k, v, a, slots, q=q, rotary=rot, positions=pos)
        mine = q.clone()
        assert B.kv4_append(k, v, a, slots, q=mine, rotary=rot, positions=pos, q_out=mine) is mine and torch.equal(mine, want)


def test_graph_replays_and_no_tokens():
    q, k, v, pos, slots, n_pages = _case(20, 4, 2, 128, 128, False, (16, 24, 24), "bf16", 16)
    k, pos, slots = k.clone(), pos.cuda(), slots.cuda()
    cache, rot = B.Kv4Cache(n_pages, 16, 2, 128), B.Rotary.of(128, sections=(16, 24, 24))
    out = torch.empty(20, 4, 128, dtype=torch.bfloat16, device="cuda")
    B.kv4_append(k[:0], v[:0], cache, slots[:0], q=q[:0], rotary=rot, positions=pos[:, :0])
    assert not bool(cache.codes.any())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.kv4_append(k, v, cache, slots, q=q, rotary=rot, positions=pos, q_out=out)
    k.mul_(0.5)
    pos.add_(17)
    graph.replay()
    other = B.Kv4Cache(n_pages, 16, 2, 128)
    want = B.kv4_append(k, v, other, slots, q=q, rotary=rot, positions=pos)
    assert torch.equal(out, want) and torch.equal(cache.codes, other.codes) and torch.equal(cache.scales, other.scales)


def test_refusals_of_the_binding():
    q, k, v, pos, slots, n_pages = _case(5, 2, 2, 64, 64, False, None, "bf16", 16)
    cache, rot, pos, slots = B.Kv4Cache(n_pages, 16, 2, 64), B.Rotary.of(64), pos.cuda(), slots.cuda()
    for bad in (dict(q=q), dict(q=q, rotary=rot), dict(positions=pos), dict(q=q, rotary=B.Rotary.of(64, sections=(8, 24)), positions=pos),
                dict(rotary=rot, positions=pos[:, :4]), dict(rotary=B.Rotary.of(128), positions=pos)):
        with pytest.raises(ValueError):
            B.kv4_append(k, v, cache, slots, **bad)
    with pytest.raises(ValueError):
        B.kv4_append(k, v, cache, slots[:4])
    with pytest.raises(ValueError):
        B.kv4_append(k[:, :1], v[:, :1], cache, slots)
    for bad in (dict(v=v.float()), dict(slots=slots.long())):
        with pytest.raises(AssertionError):
            B.kv4_append(**{**dict(k=k, v=v, cache=cache, slots=slots), **bad})
    for bad in ((0, 16, 2, 64), (4, 20, 2, 64), (4, 16, 2, 60), (4, 16, 0, 64)):
        with pytest.raises(ValueError):
            B.Kv4Cache(*bad)
    with pytest.raises(ValueError):
        B.Rotary(torch.ones(8, device="cuda"), torch.full((8,), -1, device="cuda"))
