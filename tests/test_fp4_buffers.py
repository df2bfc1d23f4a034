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


def test_the_quantizer_that_keeps_the_amax_checks_its_arguments():
    import ctypes as C
    L = B.lib()

    def call(amax, kept, fmt=B.NVFP4):
        q = B.Fp4TensorC(256, 256, kept, 48)
        return L.adadim_quantize_fp4_amax(256, B.BF16, 0 if amax == 0 else 40, 96, 96, 40, fmt, None, None, 0, C.byref(q), None,
                                          B.BF16, 0, amax or None, None)

    assert call(256, None) == 1                           # nowhere to keep it
    assert call(258, 256) == 5 and call(256, 258) == 5    # alignment
    assert call(0, None) == 0                             # an empty matrix
