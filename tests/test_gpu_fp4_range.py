"""NVFP4 products whose two tensor scales multiply to less than 2^-149 or to 2^128 and more, while the results are ordinary
binary32 numbers.

The bar is the other products' (exact products, binary32 accumulation of 64-deep steps, one rounding to the result's type):
    |y - y_ref| <= u |y_ref| + (steps + 2) 2^-22 S,   S = sum_k |a_k b_k|,  steps = ceil(in / 64),  u = 2^-8, 2^-23
(multiplying by powers of two loses nothing as long as the result is a normal number, which the inputs see to).  A row of
zeros gives zeros exactly."""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -23}
# few tokens quantized inside the product with one CTA to a tile and with a cluster; behind the quantizer the same; many
# tokens with results that leave as bulk stores and directly
SHAPES = [(3, 320, 300, torch.bfloat16), (8, 4096, 300, torch.float32), (40, 320, 300, torch.float32),
          (40, 4096, 300, torch.bfloat16), (3000, 320, 2000, torch.bfloat16), (1500, 1000, 3000, torch.float32)]


def _check(y, qx, qw, inp):
    ref, S = qx @ qw.T, np.abs(qx) @ np.abs(qw).T
    assert np.abs(ref[1:]).min() > 0.0 and np.abs(ref).max() < 2.0 ** 127
    tol = U[y.dtype] * np.abs(ref) + (-(-inp // 64) + 2) * 2.0 ** -22 * S
    err = np.abs(y.double().cpu().numpy() - ref)
    assert np.all(err <= tol), f"max err / tol {float(np.nanmax(err / np.maximum(tol, 1e-300)))}, NaN: {bool(np.isnan(err).any())}"
    assert not bool(y[0].any().item())


@pytest.mark.parametrize("tokens,inp,out,dtype", SHAPES)
def test_tensor_scales_whose_product_is_below_binary32(tokens, inp, out, dtype):
    """|x|, |w| in [2^-65, 2^-64): tensor scales 2^-75, their product 2^-150; results 2^-124 and more, all of one sign."""
    g = torch.Generator().manual_seed(tokens)
    x = ((1.0 + 0.99 * torch.rand(tokens, inp, generator=g)) * 2.0 ** -65).to(dtype)
    w = (1.0 + 0.99 * torch.rand(out, inp, generator=g)) * 2.0 ** -65
    x[0] = 0.0
    amax = torch.tensor([2.0 ** -64], device="cuda")
    W = B.quantize_fp4(w.cuda(), B.NVFP4, amax=amax)
    y = B.fp4_linear(x.cuda(), W, x_amax=amax)
    assert y.dtype == dtype
    _check(y, F.quantize(x.float().numpy(), "nv", 2.0 ** -64)[2], F.quantize(w.numpy(), "nv", 2.0 ** -64)[2], inp)


@pytest.mark.parametrize("tokens,inp,out,dtype", SHAPES)
def test_tensor_scales_whose_product_is_beyond_binary32(tokens, inp, out, dtype):
    """Expected magnitudes of 2^76 (tensor scales 2^65, their product 2^130), one element in eight of X near 2^58 and the
    others 0: results below 2^127."""
    g = torch.Generator().manual_seed(tokens + 1)
    x = ((1.0 + torch.rand(tokens, inp, generator=g)) * 2.0 ** 58).to(dtype)
    x[torch.rand(tokens, inp, generator=g) < 0.875] = 0.0
    w = (1.0 + torch.rand(out, inp, generator=g)) * 2.0 ** 58
    x[0] = 0.0
    amax = torch.tensor([2.0 ** 76], device="cuda")
    W = B.quantize_fp4(w.cuda(), B.NVFP4, amax=amax)
    y = B.fp4_linear(x.cuda(), W, x_amax=amax)
    assert y.dtype == dtype
    _check(y, F.quantize(x.float().numpy(), "nv", 2.0 ** 76)[2], F.quantize(w.numpy(), "nv", 2.0 ** 76)[2], inp)


def test_a_scale_pair_that_only_overflows_together_with_small_sums():
    """Rows of an expert stack that a router points outside the tokens are rows of zeros, whatever the scales."""
    x = torch.full((4, 64), 2.0 ** 58, device="cuda")
    amax = torch.tensor([2.0 ** 76], device="cuda")
    W = B.Fp4Tensor(48, 64, B.NVFP4, experts=2)
    for e in range(2):
        B.quantize_fp4(torch.full((48, 64), 2.0 ** 58, device="cuda"), B.NVFP4, amax=amax, q=W.expert(e))
    idx = torch.tensor([0, -1, 9, 3], dtype=torch.int32, device="cuda")
    y = B.fp4_linear_grouped(x, torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda"), W, row_index=idx, x_amax=amax)
    q = F.quantize(np.full((1, 64), 2.0 ** 58), "nv", 2.0 ** 76)[2]
    want = float((q * q).sum())                           # one product repeated: exact in binary32
    assert y[0].tolist() == [want] * 48 and y[3].tolist() == [want] * 48
    assert not bool(y[1:3].any().item())
