"""Buffers of a Kv4Cache, of PageTables and of a Rotary that are replaced (loaded from a file, moved): calls take the new ones.  No GPU."""
import copy

import pytest
import torch

from paper_2309_15531_b200 import binding as B

TABLES = ("lengths", "offsets", "requests", "positions", "slots", "cursor")


def _cache(amax=None):
    return B.Kv4Cache(3, 16, 2, 80, amax, amax, device="cpu")


def _pointers(cache):
    c = cache._ref._obj
    return c.codes, c.scales, c.amax


def _own(cache):
    return cache.codes.data_ptr(), cache.scales.data_ptr(), None if cache.amax is None else cache.amax.data_ptr()


def test_a_cache_whose_buffers_are_replaced():
    cache = _cache(torch.ones(1))
    assert _pointers(cache) == _own(cache)
    old = cache.codes, cache.scales, cache.amax          # kept, so that no new buffer gets an old address
    cache.codes, cache.scales, cache.amax = (t.clone() for t in old)
    assert _pointers(cache) == _own(cache)
    assert all(a != b.data_ptr() for a, b in zip(_pointers(cache), old))
    cache.amax = None
    assert _pointers(cache) == _own(cache) and cache.amax is None
    cache = _cache()
    cache.amax = torch.ones(2)
    assert _pointers(cache) == _own(cache)


def test_a_copy_of_a_cache_that_gets_buffers_of_its_own():
    cache = _cache()
    other = copy.copy(cache)
    other.codes = cache.codes.clone()
    assert _pointers(other) == _own(other) and _pointers(cache) == _own(cache)
    assert _pointers(other)[0] != _pointers(cache)[0] and _pointers(other)[1] == _pointers(cache)[1]


def test_buffers_of_a_cache_that_do_not_fit():
    cache = _cache(torch.ones(1))
    codes, scales, amax = cache.codes, cache.scales, cache.amax
    before = _pointers(cache)
    for wrong in (codes[:2], codes.int(), codes.reshape(-1), codes.transpose(2, 3).contiguous().transpose(2, 3), codes.to("meta")):
        with pytest.raises(ValueError):
            cache.codes = wrong
    for wrong in (scales[1:], scales.to(torch.int8), scales[..., :4], scales.reshape(-1)):
        with pytest.raises(ValueError):
            cache.scales = wrong
    for wrong in (torch.ones(1), torch.ones(3), torch.ones(2, dtype=torch.float64), torch.ones(4)[::2]):
        with pytest.raises(ValueError):
            cache.amax = wrong
    assert cache.codes is codes and cache.scales is scales and cache.amax is amax and _pointers(cache) == before


@pytest.mark.parametrize("name", TABLES)
def test_tables_whose_buffers_are_replaced(name):
    tables = B.PageTables(3, 5, device="cpu")
    other = copy.copy(tables)
    at = lambda t: [getattr(t, n).data_ptr() for n in TABLES]
    assert tables._p == at(tables)
    old = getattr(tables, name)
    setattr(tables, name, old.clone())
    assert tables._p == at(tables) and getattr(tables, name).data_ptr() != old.data_ptr()
    assert other._p == at(other) and other._p != tables._p
    for wrong in (old[:-1], old.long(), torch.zeros(2 * old.numel(), dtype=torch.int32)[::2] if old.numel() > 1 else old[:0]):
        with pytest.raises(ValueError):
            setattr(tables, name, wrong)
    assert tables._p == at(tables)


def _rotary():
    """Its constructor wants a device; the setters are what is looked at."""
    turn = object.__new__(B.Rotary)
    turn.dim, turn.adjacent, turn.axes, turn.dev = 32, False, 1, -1
    turn.freq, turn.axis = torch.ones(16), None
    return turn


def test_a_rotary_whose_numbers_are_replaced():
    turn = _rotary()
    assert turn._freq_p == turn.freq.data_ptr() and turn.freq.dtype == torch.float64 and turn._axis_p == 0
    other, kept = copy.copy(turn), turn.freq
    turn.freq = turn.freq * 0.5
    assert turn._freq_p == turn.freq.data_ptr() != kept.data_ptr() and float(turn.freq[3]) == 0.5
    assert other._freq_p == other.freq.data_ptr() == kept.data_ptr()
    turn.axis = torch.arange(16) % 3
    assert turn._axis_p == turn.axis.data_ptr() and turn.axes == 3 and turn.axis.dtype == torch.uint8
    turn.axis = None
    assert turn._axis_p == 0 and turn.axes == 1
    for wrong in (torch.ones(8), torch.ones(2, 8)):
        with pytest.raises(ValueError):
            turn.freq = wrong
    for wrong in (torch.zeros(8, dtype=torch.int32), torch.ones(16), torch.full((16,), -1), torch.full((16,), 256)):
        with pytest.raises(ValueError):
            turn.axis = wrong
    assert turn._freq_p == turn.freq.data_ptr() and turn._axis_p == 0
