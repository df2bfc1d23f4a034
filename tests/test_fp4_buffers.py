"""Buffers of an Fp4Tensor that are replaced (loaded from a file, moved): calls take the new ones.  No GPU."""
import pytest
import torch

from paper_2309_15531_b200 import binding as B


def _pointers(t):
    c = t._operand()._obj
    return c.codes, c.scales, c.ld


@pytest.mark.parametrize("experts", [0, 3])
def test_replaced_buffers_are_the_ones_that_calls_take(experts):
    t = B.Fp4Tensor(40, 96, B.MXFP4, experts=experts, device="cpu")
    assert _pointers(t) == (t.codes.data_ptr(), t.scales.data_ptr(), 48)
    t.codes, t.scales = t.codes.clone(), t.scales.clone()
    assert _pointers(t) == (t.codes.data_ptr(), t.scales.data_ptr(), 48)
    wide = torch.zeros(t.codes.shape[0], 64, dtype=torch.uint8)[:, :48]
    t.codes = wide
    assert _pointers(t) == (wide.data_ptr(), t.scales.data_ptr(), 64)


def test_buffers_that_do_not_fit_are_refused():
    t = B.Fp4Tensor(40, 96, B.NVFP4, device="cpu")
    codes, scales, before = t.codes, t.scales, _pointers(t)
    for wrong in (codes[:39], codes[:, :32], codes.int(), torch.zeros(48, 40, dtype=torch.uint8).t(), codes.reshape(-1)):
        with pytest.raises(ValueError):
            t.codes = wrong
    for wrong in (scales[1:], scales.int(), scales.reshape(2, -1), torch.zeros(2 * scales.numel(), dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            t.scales = wrong
    assert t.codes is codes and t.scales is scales and _pointers(t) == before


def test_views_follow_the_buffers_of_their_stack():
    t = B.Fp4Tensor(40, 96, B.NVFP4, experts=3, device="cpu")
    one = t.expert(2)
    before = _pointers(one)
    t.codes = torch.zeros_like(t.codes)
    t.scales = torch.zeros_like(t.scales)
    assert _pointers(one) != before
    assert _pointers(one) == (t.codes.data_ptr() + 2 * 40 * 48, t.scales.data_ptr() + 2 * t.scale_bytes, 48)
    assert one.codes.shape == (40, 48) and one.scales.shape == (t.scale_bytes,)
    with pytest.raises(ValueError):
        one.codes = one.codes.clone()
    with pytest.raises(ValueError):
        one.scales = one.scales.clone()
