"""Pins of the 4-bit floating-point oracle to the formats' definitions, and of the library's host-side rules."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import fp4_oracle as F


def test_e4m3_table():
    assert F.E4M3[0x7E] == 448.0 and F.E4M3[1] == 2.0 ** -9 and F.E4M3[8] == 2.0 ** -6 and F.E4M3[0x38] == 1.0
    assert np.all(np.diff(F.E4M3) > 0)


def test_ties_go_to_the_even_code():
    x = np.zeros((1, 32))
    x[0, :9] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -2.5]
    codes, byte, values = F.quantize(x, "mx")
    assert byte[0, 0] == 127
    assert values[0, :9].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -2.0]
    assert codes[0, 8] == 8 + 4


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_nearest_level_by_brute_force(fmt):
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((8, 96)) * np.exp(rng.uniform(-8, 8, (8, 1)))).astype(np.float32)
    amax = float(np.abs(x).max()) if fmt == "nv" else None
    codes, byte, values = F.quantize(x, fmt, amax)
    B, t = F.BLOCK[fmt], F.tensor_scale(amax)
    for r in range(8):
        for b in range(96 // B):
            m = float(np.abs(x[r, b * B:(b + 1) * B]).max())
            if fmt == "mx":
                s = 2.0 ** (int(byte[r, b]) - 127)
                assert 4.0 * s <= m < 8.0 * s
            else:
                s = F.E4M3[byte[r, b]] * t
                assert abs(F.E4M3[byte[r, b]] - m / (6 * t)) == np.abs(F.E4M3 - m / (6 * t)).min()
            if s == 0.0:
                continue
            for c in range(b * B, (b + 1) * B):
                best = np.abs(F.LEVELS - min(abs(float(x[r, c])) / s, 6.0)).min()
                assert abs(abs(values[r, c]) / s - min(abs(float(x[r, c])) / s, 6.0)) <= best * (1 + 1e-12)


def test_tensor_scale_covers_amax_and_no_more():
    for a in (2688.0, 2688.0 * (1 + 2.0 ** -23), 1344.0, 1.0, 448.0, 1e-6, 3e38):
        t = F.tensor_scale(a)
        assert t == 2.0 ** round(math.log2(t)) and 2688.0 * t >= a > 1344.0 * t
    assert F.tensor_scale(None) == F.tensor_scale(0.0) == F.tensor_scale(math.inf) == F.tensor_scale(math.nan) == 1.0
    assert F.tensor_scale(1e-38) == 2.0 ** -100


def test_groups_never_share_a_tile_row():
    rng = np.random.default_rng(5)
    for _ in range(50):
        counts = rng.integers(0, 300, rng.integers(1, 12)) * (rng.random() < 0.9)
        off = np.concatenate(([0], np.cumsum(counts)))
        tr, ir, n = F.tile_rows(int(off[-1]), off)
        assert len(set(zip(tr.tolist(), ir.tolist()))) == len(tr) and (len(tr) == 0 or tr.max() < n)
        for e in range(len(counts)):
            assert np.all(ir[off[e]:off[e + 1]] == np.arange(counts[e]) % 128)


@pytest.fixture(scope="module")
def lib():
    from paper_2309_15531_b200 import build
    build.build()
    from paper_2309_15531_b200 import binding as B
    return B, B.lib()


def test_sizes_of_the_layout(lib):
    B, L = lib
    assert L.adadim_fp4_scale_bytes(B.NVFP4, 128, 64, 0) == 512 and L.adadim_fp4_scale_bytes(B.MXFP4, 128, 128, 0) == 512
    assert L.adadim_fp4_scale_bytes(B.NVFP4, 129, 65, 0) == 4 * 512
    assert L.adadim_fp4_scale_bytes(B.MXFP4, 300, 1, 5) == (300 // 128 + 5) * 512
    assert L.adadim_fp4_scale_bytes(7, 128, 64, 0) == 0 and L.adadim_fp4_scale_bytes(B.NVFP4, -1, 64, 0) == 0
    assert B.workspace_bytes(B.WS_FP4, 16, 4096, 4, 0) >= 16 * 2048 + 64 * 512
    assert B.workspace_bytes(B.WS_FP4, 0, 4096, 4, 0) == 0


def test_refusals_need_no_gpu(lib):
    B, L = lib
    q = B.Fp4TensorC(256, 256, None, 64)
    bad_ld, bad_codes, bad_scales = B.Fp4TensorC(256, 256, None, 56), B.Fp4TensorC(264, 256, None, 64), B.Fp4TensorC(256, 272, None, 64)

    def quant(X=256, dt=B.F16, rows=8, cols=128, ldx=128, x_rows=8, fmt=B.NVFP4, idx=None, off=None, n=0, t=q, v=None,
              vdt=B.BF16, ldv=128):
        return L.adadim_quantize_fp4(X, dt, rows, cols, ldx, x_rows, fmt, idx, off, n, C.byref(t) if t is not None else None,
                                     v, vdt, ldv, None)
    assert quant(fmt=2) == 4 and quant(dt=9) == 3 and quant(v=256, vdt=B.F16) == 3
    assert quant(rows=-1) == 2 and quant(cols=(1 << 20) + 1) == 2 and quant(ldx=127) == 2 and quant(x_rows=7) == 2
    assert quant(n=2) == 1 and quant(off=256, n=0) == 4 and quant(off=256, n=1025) == 4 and quant(off=258, n=2) == 5
    assert quant(X=None) == 1 and quant(t=None) == 1 and quant(X=257) == 5 and quant(idx=258) == 5
    assert quant(t=bad_ld) == 2 and quant(t=bad_codes) == 5 and quant(t=bad_scales) == 5
    assert quant(v=256, ldv=100) == 2 and quant(v=257) == 5
    assert quant(rows=0, X=None, t=None) == 0 and quant(cols=0, X=None, t=None) == 0

    def lin(X=256, dt=B.BF16, rows=8, inp=128, ldx=128, t=q, out=128, fmt=B.MXFP4, Y=256, ydt=B.BF16, ldy=128, ws=256,
            wsb=1 << 20):
        return L.adadim_fp4_linear(X, dt, rows, inp, ldx, None, C.byref(t) if t is not None else None, out, fmt, Y, ydt,
                                   ldy, None, ws, wsb, None)
    assert lin(fmt=5) == 4 and lin(dt=4) == 3 and lin(ydt=4) == 3 and lin(inp=0) == 2 and lin(out=-1) == 2
    assert lin(ldy=100) == 2 and lin(ldx=100) == 2 and lin(X=None) == 1 and lin(Y=None) == 1 and lin(t=None) == 1
    assert lin(ws=None) == 1 and lin(ws=128) == 5 and lin(wsb=512) == 6 and lin(Y=257) == 5
    assert lin(rows=0) == 0 and lin(out=0) == 0

    def grp(n=2, off=256, rows=8, x_rows=8, idx=None, out=128):
        return L.adadim_fp4_linear_grouped(256, B.BF16, x_rows, 128, 128, None, idx, off, n, rows, C.byref(q), out, B.MXFP4,
                                           256, B.BF16, 128, None, 256, 1 << 20, None)
    assert grp(n=0) == 4 and grp(n=-1) == 4 and grp(off=None) == 1 and grp(x_rows=7) == 2 and grp(idx=258) == 5
    assert grp(n=1024, out=1 << 22) == 2 and grp(rows=0) == 0
    assert L.adadim_fp4_matmul(None, 8, C.byref(q), 128, 128, 0, 256, B.F32, 128, None, None) == 1
    assert L.adadim_fp4_matmul_grouped(C.byref(q), 8, None, 0, C.byref(q), 128, 128, 0, 256, B.F32, 128, None, None) == 4
    assert L.adadim_absmax(256, B.F32, 8, 8, 4, 256, None) == 2 and L.adadim_absmax(None, B.F32, 8, 8, 8, 256, None) == 1
    assert L.adadim_absmax(256, B.F32, 8, 8, 8, None, None) == 1 and L.adadim_absmax(None, B.F32, 0, 8, 8, None, None) == 0
