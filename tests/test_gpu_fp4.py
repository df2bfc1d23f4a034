"""The 4-bit floating-point operators on the GPU against the binary64 oracle (through the C ABI).

Quantizer: codes, scale bytes and values are exact (the sign of a zero is not specified).  Products: every product of two quantized numbers is
exact, so what is left is the binary32 accumulation and one rounding to the result's type.  Bar:
    |y - y_ref| <= u |y_ref| + (steps + 2) 2^-22 S + tiny,   S = sum_k |a_k b_k|,  steps = ceil(in / 64)
with u = 2^-8, 2^-11, 2^-23 for bf16, fp16, fp32 results (half an ulp, rounded up for fp32), each 64-deep
accumulation losing at most 2^-22 of what it adds up, and tiny = 2^-24 for the smallest fp16 numbers."""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from paper_2309_15531_b200 import binding as B
from paper_2309_15531_b200 import flows

pytestmark = pytest.mark.gpu

FMT = {"mx": B.MXFP4, "nv": B.NVFP4}
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -23}


def _x(rows, cols, dtype, seed, scale=1.0, gap=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols + gap, generator=g) * scale
    x[:, torch.rand(cols + gap, generator=g) < 0.02] *= 60.0
    x[torch.rand(rows, cols + gap, generator=g) < 0.05] = 0.0
    return x.to(DT[dtype]).cuda()[:, :cols]


def _np(t):
    return t.detach().float().cpu().numpy()


def _unsigned_zero(codes):
    return np.where(codes == 8, 0, codes).astype(np.uint8)           # the sign of a zero code is not specified


def _check_quantized(q, x_np, fmt, amax, offsets=None, values=None):
    codes, byte, ref = F.quantize(x_np, fmt, amax)
    codes = _unsigned_zero(codes)
    rows, cols = x_np.shape
    live = np.ones(rows, bool) if offsets is None else (np.arange(rows) >= offsets[0]) & (np.arange(rows) < offsets[-1])
    got = q.codes.cpu().numpy()
    assert np.array_equal(_unsigned_zero(F.unpack(got, cols))[live], codes[live, :cols])
    wide = -(-((cols + 1) // 2) // 8) * 8                            # what is behind the last column is zero
    assert not F.unpack(got, wide * 2)[live, cols:].any()
    sc = F.untile_scales(q.scales.cpu().numpy(), rows, byte.shape[1], offsets)
    assert np.array_equal(sc[live], byte[live])
    if values is not None:
        want = torch.as_tensor(ref).to(values.dtype)
        assert np.array_equal(_np(values)[live], want.float().numpy()[live], equal_nan=True)
    return ref


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,gap", [(1, 1, 0), (1, 16, 0), (3, 17, 0), (2, 33, 7), (127, 64, 8), (129, 255, 1),
                                           (130, 257, 0), (257, 1003, 0), (64, 2048, 16), (300, 640, 3)])
def test_quantize(fmt, dtype, rows, cols, gap):
    x = _x(rows, cols, dtype, rows + cols, 0.3, gap)
    amax = B.absmax(x)
    a = float(np.abs(_np(x)).max())
    assert float(amax.item()) == a
    v = torch.empty(rows, cols + gap, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")[:, :cols]
    q = B.quantize_fp4(x, FMT[fmt], amax=amax, values=v)
    _check_quantized(q, _np(x), fmt, a, values=v)
    n4 = -(-cols // (4 * F.BLOCK[fmt]))                              # what the tiles hold beyond the matrix is zero
    nb = -(-cols // F.BLOCK[fmt])
    buf = F.untile_scales(q.scales.cpu().numpy(), -(-rows // 128) * 128, n4 * 4)
    assert not buf[rows:].any() and not buf[:, nb:].any()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_quantize_special_values(fmt):
    nan, inf, top = float("nan"), float("inf"), 3.4028234663852886e38
    rows = [
        [0.0] * 32, [-0.0] * 32, [1e-45, 2e-45] * 16, [1.1754944e-38, -5e-39] * 16, [top, -top] * 16,
        [inf] + [1.0] * 31, [1.0] * 31 + [nan], [-inf, 2.0] * 16, [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0] * 4,
        [5.0, 0.2500001, 0.7499999, 1.2500001, 1.7499999, 2.5000002, 3.4999998, 4.9999995] * 4,
        [7.9999995, -7.5, 4.0, 2.0] * 8, [8.0, 1.0, 0.5, -0.25] * 8, [448.0 * 6, 1.0, 300.0, -2000.0] * 8, [1e-3] * 31 + [100.0],
    ]
    x = torch.tensor(rows, dtype=torch.float32, device="cuda")
    for amax in (None, 0.0, inf, nan, 1.0, 2688.0, 1e-38, top, 1e-30):
        a = torch.tensor([amax], device="cuda") if amax is not None else None
        v = torch.empty_like(x)
        q = B.quantize_fp4(x, FMT[fmt], amax=a, values=v)
        a32 = None if amax is None else float(np.float32(amax))
        _check_quantized(q, x.cpu().numpy(), fmt, a32, values=v)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_quantize_every_bf16_pattern(fmt):
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16).reshape(256, 256)
    x = x[:, torch.randperm(256, generator=torch.Generator().manual_seed(1))].cuda().contiguous()
    q = B.quantize_fp4(x, FMT[fmt])
    _check_quantized(q, _np(x), fmt, None)


def test_quantize_ties_of_nvfp4_block_scales():
    """Blocks whose m / 6 is a midpoint of two E4M3 numbers, and its binary32 neighbours."""
    mids = (F.E4M3[1:] + F.E4M3[:-1]) / 2 * 6.0
    m = np.concatenate([np.nextafter(mids.astype(np.float32), np.float32(0)), mids.astype(np.float32),
                        np.nextafter(mids.astype(np.float32), np.float32(1e9))])
    x = np.zeros((len(m), 16), np.float32)
    x[:, 3] = m
    x[:, 7] = m * np.float32(0.3)
    q = B.quantize_fp4(torch.as_tensor(x).cuda(), B.NVFP4)
    _check_quantized(q, x, "nv", None)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("counts,cap", [((5,), 0), ((0, 130, 0, 1, 127, 128, 129, 0), 0), ((0, 0, 0), 3), ((1, 1, 1, 1), 9),
                                        ((256, 0, 300), 40)])
def test_quantize_groups_and_gather(fmt, counts, cap):
    off = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    rows, cols = int(off[-1]) + cap, 200
    x = _x(57, cols, "bf16", 11)
    idx = torch.randint(0, 57, (rows,), generator=torch.Generator().manual_seed(2)).int()
    if rows > 4:
        idx[3], idx[4] = -1, 57                                      # outside: rows of zeros
    gathered = np.zeros((rows, cols), np.float32)
    ok = (idx.numpy() >= 0) & (idx.numpy() < 57)
    gathered[ok] = _np(x)[idx.numpy()[ok]]
    q = B.Fp4Tensor(rows, cols, FMT[fmt], groups=len(counts))
    q.codes.fill_(0x55)
    B.quantize_fp4(x, FMT[fmt], q=q, row_index=idx.cuda(), offsets=torch.as_tensor(off).cuda())
    _check_quantized(q, gathered, fmt, None, offsets=off)
    assert bool((q.codes[int(off[-1]):] == 0x55).all().item())       # rows of no group are left alone


def test_absmax_over_chunks_and_nan():
    x = _x(100, 333, "f16", 4, gap=5)
    a = B.absmax(x[:40])
    B.absmax(x[40:], a)
    assert float(a.item()) == float(x.abs().max().item())
    assert float(B.absmax(-x[:1, :1].abs() - 2).item()) == float((x[:1, :1].abs() + 2).max().item())
    x[7, 9] = float("nan")
    assert np.isnan(float(B.absmax(x).item()))
    assert float(B.absmax(x[:0]).item()) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,gap", [(1, 1, 0), (1, 8191, 0), (3, 8193, 0), (5, 20000, 8), (7, 9001, 3), (300, 129, 0)])
def test_absmax_finds_the_largest_wherever_it_is(dtype, rows, cols, gap):
    g = torch.Generator().manual_seed(rows + cols)
    x = torch.rand(rows, cols + gap, generator=g).to(DT[dtype]).cuda()[:, :cols]
    if gap:
        x.as_strided((rows, cols + gap), (cols + gap, 1))[:, cols:] = 100.0          # what lies between rows is not read
    for at in (0, cols - 1, cols // 2, cols // 3):
        r = at % rows
        old = x[r, at].item()
        x[r, at] = -9.0
        assert float(B.absmax(x).item()) == 9.0
        x[r, at] = old
    assert float(B.absmax(x).item()) == float(x.abs().max().float().item())


def _assert_product(y, xa, wb, inp, what=""):
    """xa, wb: quantized values float64 of the rows of y and of the weight."""
    ref = xa @ wb.T
    S = np.abs(xa) @ np.abs(wb).T
    steps = -(-inp // 64)
    tol = U[y.dtype] * np.abs(ref) + (steps + 2) * 2.0 ** -22 * S + (2.0 ** -24 if y.dtype == torch.float16 else 0.0)
    err = np.abs(y.double().cpu().numpy() - ref)
    assert np.all(err <= tol), f"{what}: max err / tol {float(np.max(err / np.maximum(tol, 1e-300)))}"


SHAPES = [(1, 1, 1), (1, 64, 16), (1, 4096, 1024), (2, 63, 127), (5, 65, 129), (16, 256, 128), (17, 255, 130), (33, 257, 96),
          (64, 1000, 257), (65, 512, 128), (127, 320, 300), (128, 128, 128), (129, 1344, 129), (300, 700, 513), (700, 384, 640)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("tokens,inp,out", SHAPES)
def test_linear(fmt, tokens, inp, out):
    for k, dtype in enumerate(("bf16", "f16", "f32")):
        if k != (tokens + inp) % 3 and tokens * inp > 4096 * 16:
            continue
        x = _x(tokens, inp, dtype, 7 * tokens + inp, 1.0, gap=k * 3)
        w = _x(out, inp, "f16", out + inp, 0.02)
        xa, wa = B.absmax(x), B.absmax(w)
        W = B.quantize_fp4(w, FMT[fmt], amax=wa)
        y = torch.full((tokens, out + k), -7.0, dtype=x.dtype, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.fp4_linear(x, W, x_amax=xa, y=y[:, :out], status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and bool((y[:, out:] == -7.0).all().item())
        qx = F.quantize(_np(x), fmt, float(xa.item()))[2]
        qw = F.quantize(_np(w), fmt, float(wa.item()))[2]
        _assert_product(y[:, :out], qx, qw, inp, dtype)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_quantized_activations_give_the_same_bits(fmt):
    x, w = _x(40, 520, "bf16", 1), _x(200, 520, "f16", 2, 0.02)
    W = B.quantize_fp4(w, FMT[fmt], amax=B.absmax(w))
    y = B.fp4_linear(x, W)
    q = B.quantize_fp4(x, FMT[fmt])
    assert torch.equal(B.fp4_linear(q, W), y) and y.dtype == torch.bfloat16
    y32 = B.fp4_linear(q, W, y=torch.empty(40, 200, device="cuda"))
    assert torch.equal(y32.bfloat16(), y)
    assert torch.equal(B.fp4_linear(x, W), y)                        # no order of sums depends on chance


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("tokens", [3, 200])
def test_nan_and_infinity_stay_in_their_rows(fmt, tokens):
    x, w = _x(tokens, 320, "bf16", 1), _x(150, 320, "f16", 2, 0.02)
    x[1, 300], x[2, 0] = float("nan"), float("inf")
    w[5, 7] = float("nan")
    y = B.fp4_linear(x, B.quantize_fp4(w, FMT[fmt]), y=torch.zeros(tokens, 150, device="cuda"))
    bad = torch.isnan(y)
    want = torch.zeros_like(bad)
    want[1], want[2], want[:, 5] = True, True, True
    assert torch.equal(bad, want) and not bool(torch.isinf(y).any().item())


GROUPS = [((1,), 64, 16), ((0, 3, 0), 130, 100), ((5, 0, 17, 1), 256, 129), ((130, 1, 0, 0, 260), 320, 257),
          ((0, 0), 64, 64), ((40,) * 9, 128, 64), ((2, 0, 1, 0, 3, 1, 1, 5), 1000, 300), ((300, 0, 129, 128), 96, 384),
          ((1,) * 33, 70, 48)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("counts,inp,out", GROUPS)
def test_linear_grouped(fmt, counts, inp, out):
    off = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    E, rows, x_rows = len(counts), int(off[-1]) + 2, 23                # two rows of capacity beyond the groups
    x = _x(x_rows, inp, "bf16", inp)
    idx = torch.randint(0, x_rows, (rows,), generator=torch.Generator().manual_seed(3)).int().cuda()
    xa = B.absmax(x)
    ws = [_x(out, inp, "f16", 100 + e, 0.02) for e in range(E)]
    wa = torch.zeros(1, device="cuda")
    for w in ws:
        B.absmax(w, wa)
    W = B.Fp4Tensor(out, inp, FMT[fmt], experts=E)
    for e, w in enumerate(ws):
        B.quantize_fp4(w, FMT[fmt], amax=wa, q=W.expert(e))
    y = torch.full((rows, out), -7.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = torch.as_tensor(off).cuda()
    B.fp4_linear_grouped(x, o, W, row_index=idx, x_amax=xa, y=y, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and bool((y[int(off[-1]):] == -7.0).all().item())
    qx = F.quantize(_np(x), fmt, float(xa.item()))[2][idx.cpu().numpy()]
    for e in range(E):
        a, z = off[e], off[e + 1]
        if z > a:
            _assert_product(y[a:z], qx[a:z], F.quantize(_np(ws[e]), fmt, float(wa.item()))[2], inp, f"expert {e}")
    q = B.quantize_fp4(x, FMT[fmt], amax=xa, row_index=idx, offsets=o)
    y2 = torch.full_like(y, -7.0)
    B.fp4_linear_grouped(q, o, W, y=y2)
    assert torch.equal(y2, y)


# Shapes that the many-token kernel takes, with token tiles of different heights, results that can and cannot leave as
# bulk stores (rows that are not 16-byte aligned), edges inside a tile in both directions, and short last stages.
MANY = [(3000, 320, 2000, "bf16", 0), (600, 1344, 4104, "f16", 0), (1500, 1000, 3000, "f32", 0), (2000, 192, 2056, "bf16", 3),
        (3001, 330, 2008, "f16", 0), (2500, 130, 5000, "bf16", 8), (1536, 4160, 2048, "bf16", 0)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("tokens,inp,out,dtype,gap", MANY)
def test_linear_many_tokens(fmt, tokens, inp, out, dtype, gap):
    x = _x(tokens, inp, dtype, 3 * tokens + inp)
    w = _x(out, inp, "f16", out + inp, 0.02)
    xa, wa = B.absmax(x), B.absmax(w)
    W = B.quantize_fp4(w, FMT[fmt], amax=wa)
    qx = F.quantize(_np(x), fmt, float(xa.item()))[2]
    qw = F.quantize(_np(w), fmt, float(wa.item()))[2]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for a, kw in ((x, {"x_amax": xa}), (B.quantize_fp4(x, FMT[fmt], amax=xa), {})):
        y = torch.full((tokens + 1, out + gap), -7.0, dtype=x.dtype, device="cuda")
        B.fp4_linear(a, W, y=y[:tokens, :out], status=status, **kw)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        assert bool((y[tokens] == -7.0).all().item()) and bool((y[:, out:] == -7.0).all().item())
        _assert_product(y[:tokens, :out], qx, qw, inp, dtype)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("counts,inp,out,dtype", [((700, 0, 901, 799), 330, 3000, "bf16"), ((1, 2047, 1252), 200, 4104, "f16"),
                                                  ((0, 1700, 33, 1650, 17, 1600), 96, 2600, "f32")])
def test_linear_grouped_many_tokens(fmt, counts, inp, out, dtype):
    off = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    E, rows, x_rows = len(counts), int(off[-1]) + 40, 500
    x = _x(x_rows, inp, dtype, inp)
    idx = torch.randint(0, x_rows, (rows,), generator=torch.Generator().manual_seed(3)).int().cuda()
    xa = B.absmax(x)
    ws = [_x(out, inp, "f16", 200 + e, 0.02) for e in range(E)]
    wa = torch.zeros(1, device="cuda")
    for w in ws:
        B.absmax(w, wa)
    W = B.Fp4Tensor(out, inp, FMT[fmt], experts=E)
    for e, w in enumerate(ws):
        B.quantize_fp4(w, FMT[fmt], amax=wa, q=W.expert(e))
    o = torch.as_tensor(off).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    qx = F.quantize(_np(x), fmt, float(xa.item()))[2][idx.cpu().numpy()]
    q = B.quantize_fp4(x, FMT[fmt], amax=xa, row_index=idx, offsets=o)
    for a, kw in ((x, {"row_index": idx, "x_amax": xa}), (q, {})):
        y = torch.full((rows, out), -7.0, dtype=x.dtype, device="cuda")
        B.fp4_linear_grouped(a, o, W, y=y, status=status, **kw)
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and bool((y[int(off[-1]):] == -7.0).all().item())
        for e in range(E):
            if counts[e]:
                _assert_product(y[off[e]:off[e + 1]], qx[off[e]:off[e + 1]],
                                F.quantize(_np(ws[e]), fmt, float(wa.item()))[2], inp, f"expert {e}")


def test_bad_offsets_are_reported_and_clamped():
    W = B.Fp4Tensor(64, 128, B.MXFP4, experts=3)
    x = torch.zeros(10, 128, dtype=torch.bfloat16, device="cuda")
    for off in ([0, 20, 20, 20], [0, 6, 4, 10], [-5, 0, 5, 10]):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.fp4_linear_grouped(x, torch.tensor(off, dtype=torch.int32, device="cuda"), W, status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 2


def test_another_stream_and_a_graph():
    x, w = _x(9, 384, "bf16", 1), _x(256, 384, "f16", 2, 0.02)
    W = B.quantize_fp4(w, B.NVFP4, amax=B.absmax(w))
    want = B.fp4_linear(x, W)
    y = torch.zeros_like(want)
    ws = torch.empty(B.workspace_bytes(B.WS_FP4, 9, 384, 4, 0), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.fp4_linear(x, W, y=y, workspace=ws)
    side.synchronize()
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.fp4_linear(x, W, y=y, workspace=ws)
    x.mul_(2.0)                                                      # a power of two: exactly twice the result
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want * 2)


def test_scales_offsets_beyond_32_bits_of_elements():
    """A result of more than 2^31 elements: rows far apart through the pitch."""
    x, w = _x(3, 64, "bf16", 1), _x(16, 64, "f16", 2)
    W = B.quantize_fp4(w, B.MXFP4)
    pitch = (1 << 30) + 64
    y = torch.empty(3 * pitch, dtype=torch.bfloat16, device="cuda").view(3, pitch)[:, :16]
    B.fp4_linear(x, W, y=y)
    assert torch.equal(y.contiguous(), B.fp4_linear(x, W))


def test_binding_refuses_what_does_not_match():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    W = B.Fp4Tensor(32, 128, B.MXFP4)
    with pytest.raises(ValueError):
        B.fp4_linear(x, W)
    with pytest.raises(ValueError):
        B.fp4_linear(B.Fp4Tensor(4, 128, B.NVFP4), W)
    with pytest.raises(ValueError):
        B.fp4_linear_grouped(torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda"),
                             torch.zeros(3, dtype=torch.int32, device="cuda"), W)
    with pytest.raises(ValueError):
        B.quantize_fp4(x, B.MXFP4, q=W)
    stack, amax = B.Fp4Tensor(4, 64, B.NVFP4, experts=2), B.absmax(x)
    B.quantize_fp4(x, B.NVFP4, amax=amax, q=stack.expert(0))
    with pytest.raises(ValueError):
        B.quantize_fp4(x, B.NVFP4, q=stack.expert(1))                # the experts of a stack share one amax
    stack.set_amax(None)
    B.quantize_fp4(x, B.NVFP4, q=stack.expert(1))
    with pytest.raises(B.AdadimError) as e:
        B.fp4_linear(torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda"), W,
                     workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 6
    big = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    for wrong in (dict(x_amax=torch.zeros(1)), dict(x_amax=torch.zeros(1, dtype=torch.float64, device="cuda")),
                  dict(status=torch.zeros(1, dtype=torch.int32)), dict(status=torch.zeros(1, device="cuda")),
                  dict(workspace=torch.empty(1 << 20, dtype=torch.uint8)), dict(y=torch.empty(4, 32, dtype=torch.bfloat16))):
        with pytest.raises(AssertionError):
            B.fp4_linear(big, W, **wrong)
        with pytest.raises(AssertionError):
            B.fp4_linear_grouped(big, torch.zeros(2, dtype=torch.int32, device="cuda"),
                                 B.Fp4Tensor(32, 128, B.MXFP4, experts=1), **wrong)


def test_products_of_many_streams_do_not_hold_each_other_up():
    """Products whose clusters exchange partial sums, on eight streams at a time: each gives what it gives alone."""
    shapes = [(12, 1024, 2048), (3, 640, 4096), (16, 512, 1920), (100, 384, 2048)] * 2
    jobs = []
    for i, (rows, out, inp) in enumerate(shapes):
        g = torch.Generator().manual_seed(i)
        x = torch.randn(rows, inp, generator=g).to(torch.bfloat16).cuda()
        W = B.quantize_fp4(torch.randn(out, inp, generator=g).to(torch.bfloat16).cuda(), B.MXFP4 if i % 2 else B.NVFP4)
        jobs.append((x, W, B.fp4_linear(x, W), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    ys = []
    for _ in range(25):
        for x, W, _, status, stream in jobs:
            with torch.cuda.stream(stream):
                ys.append(B.fp4_linear(x, W, status=status))
    torch.cuda.synchronize()
    for k, y in enumerate(ys):
        assert torch.equal(y, jobs[k % len(jobs)][2])
    assert all(int(status.item()) == 0 for _, _, _, status, _ in jobs)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("tokens", [5, 300])
def test_expert_ffn_flow_against_each_expert_alone(fmt, tokens):
    """The flow against the dense product of every expert on its rows.  The two may add up in another order (2^-22 of
    the sums), which can flip a bf16 rounding of an intermediate and then a 4-bit code now and then: the results agree
    to far better than the step between neighbouring codes, 2^-6 in the norm."""
    E, top, hidden, ffn = 6, 2, 256, 384
    x = _x(tokens, hidden, "bf16", 5)
    g = torch.Generator().manual_seed(6)
    experts = torch.stack([torch.randperm(E - 1, generator=g)[:top] for _ in range(tokens)]).cuda()     # the last gets nothing
    weights = torch.rand(tokens, top, generator=g).cuda()
    raw = {n: [_x(*s, "f16", 50 * k + e, 0.05) for e in range(E)] for k, (n, s) in
           enumerate({"gate": (ffn, hidden), "up": (ffn, hidden), "down": (hidden, ffn)}.items())}
    gate, up, down = (flows.fp4_weight(raw[n], FMT[fmt]) for n in ("gate", "up", "down"))
    xa, ha = B.absmax(x), torch.tensor([4000.0], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = flows.fp4_expert_ffn(x, experts, weights, gate, up, down, xa, ha, status=status)
    want = torch.zeros(tokens, hidden, device="cuda")
    for e in range(E):
        t, k = (experts == e).nonzero(as_tuple=True)
        if len(t) == 0:
            continue
        xe = x[t].contiguous()
        h = torch.nn.functional.silu(B.fp4_linear(xe, gate.expert(e), x_amax=xa)) * B.fp4_linear(xe, up.expert(e), x_amax=xa)
        want.index_add_(0, t, B.fp4_linear(h, down.expert(e), x_amax=ha).float() * weights[t, k, None])
    assert int(status.item()) == 0
    assert float((y.float() - want).norm() / want.norm()) < 2.0 ** -6
    order, row_index, offsets = flows.rows_by_expert(experts, E)
    flat = experts.reshape(-1)
    assert bool((flat[order][1:] >= flat[order][:-1]).all().item()) and offsets.tolist()[-1] == tokens * top
    assert row_index.tolist() == (order // top).tolist() and offsets.tolist()[E - 1] == tokens * top
