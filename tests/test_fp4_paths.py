"""Every way through the 4-bit products, at shapes that are known to take it: the plan is asked on the CPU, the numbers are
compared with the binary64 oracle on the GPU.

Bar as for the other products (exact products, binary32 accumulation of 64-deep steps that lose 2^-22 of what they add up
each, one rounding to the result's type):
    |y - y_ref| <= u |y_ref| + (ceil(in / 64) + 2) 2^-22 S + tiny,   S = sum_k |a_k b_k|
with u = 2^-8, 2^-11, 2^-23 for bf16, fp16 and fp32 results and tiny = 2^-24 for the smallest fp16 numbers.  Of weights with
many rows the oracle takes some: the first and last tile's, and others at random."""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from paper_2309_15531_b200 import binding as B
from paper_2309_15531_b200 import flows

FMT = {"mx": B.MXFP4, "nv": B.NVFP4}
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -23}

# quantized inside the product: (in, out, CTAs of a cluster, whether a CTA's stages are more than its ring has)
FUSED = [(16, 300, 1, False), (320, 300, 1, False), (4096, 300, 8, False), (4096, 11008, 1, True), (2304, 19200, 1, True),
         (1040, 57000, 1, True)]
FUSED_TOKENS = [1, 2, 3, 4, 5, 7, 8]
# many tokens, 16-bit results whose rows are not 16-byte aligned (no bulk stores) and that are
MANY = [(2500, 130, 5000, "bf16", 3), (1536, 4160, 2048, "f16", 1), (2500, 130, 5000, "f16", 8), (1536, 4160, 2048, "bf16", 0)]
GROUPED_MANY = [((700, 0, 941, 799), 330, 3000, "bf16", 3), ((1, 2047, 1292), 200, 4104, "f16", 5)]


@pytest.mark.parametrize("fmt", [B.MXFP4, B.NVFP4])
def test_the_shapes_below_take_the_ways_they_are_meant_for(fmt):
    for inp, out, splits, wraps in FUSED:
        for tokens in FUSED_TOKENS:
            p = B.fp4_plan(tokens, out, inp, fmt)
            assert p.fused and not p.many and p.splits == splits
            assert not B.fp4_plan(tokens, out, inp, fmt, aligned=False).fused
            # a ring has 8 stages at most, and those that fit into the CTA's share of 220 KB at 20 KB or more each
            stages = -(-inp // 256) // splits
            ring = min(8, 220 // p.ctas_per_sm // 19)
            assert (stages > ring) == wraps
    for tokens, inp, out, dtype, gap in MANY:
        assert B.fp4_plan(tokens, out, inp, fmt).many and B.fp4_plan(tokens, out, inp, fmt, quantized=True).many
    for counts, inp, out, dtype, gap in GROUPED_MANY:
        assert B.fp4_plan(sum(counts), out, inp, fmt, experts=len(counts)).many
        assert B.fp4_plan(sum(counts), out, inp, fmt, experts=len(counts), quantized=True).many


def test_plan_refuses_what_products_refuse():
    for args in ((0, 64, 64, B.MXFP4), (1, 0, 64, B.MXFP4), (1, 64, 0, B.MXFP4), (1, 64, 64, 2), (1, 64, 64, B.MXFP4, 1025),
                 (1, 64, 64, B.MXFP4, -1), ((1 << 22) + 1, 64, 64, B.NVFP4), (1, 64, (1 << 20) + 1, B.NVFP4)):
        with pytest.raises(B.AdadimError):
            B.fp4_plan(*args)


def _x(rows, cols, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * scale
    x[:, torch.rand(cols, generator=g) < 0.02] *= 60.0
    x[torch.rand(rows, cols, generator=g) < 0.05] = 0.0
    return x.to(DT[dtype]).cuda()


def _some_rows(out, seed):
    if out <= 600:
        return np.arange(out)
    rng = np.random.default_rng(seed)
    return np.unique(np.concatenate((np.arange(128), np.arange(out - 128, out), rng.integers(0, out, 256))))


def _quantized(m, fmt, amax, rows=None):
    m = m if rows is None else m[torch.as_tensor(rows, device="cuda")]
    return F.quantize(m.float().cpu().numpy(), fmt, float(amax.item()))[2]


def _check(y, xa, wb, inp, what):
    ref, S = xa @ wb.T, np.abs(xa) @ np.abs(wb).T
    tol = U[y.dtype] * np.abs(ref) + (-(-inp // 64) + 2) * 2.0 ** -22 * S + (2.0 ** -24 if y.dtype == torch.float16 else 0.0)
    err = np.abs(y.double().cpu().numpy() - ref)
    assert np.all(err <= tol), f"{what}: max err / tol {float(np.max(err / np.maximum(tol, 1e-300)))}"


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("inp,out,splits,wraps", FUSED)
def test_few_tokens_quantized_inside_the_product(fmt, inp, out, splits, wraps):
    w = _x(out, inp, "f16", out + inp, 0.02)
    wa = B.absmax(w)
    W = B.quantize_fp4(w, FMT[fmt], amax=wa)
    rows = _some_rows(out, inp)
    qw, at = _quantized(w, fmt, wa, rows), torch.as_tensor(rows, device="cuda")
    same = 0
    for tokens in FUSED_TOKENS:
        for dtype in ("bf16", "f16", "f32"):
            x = _x(tokens, inp, dtype, 7 * tokens + inp)
            xa = B.absmax(x)
            y = torch.full((tokens + 2, out), -7.0, dtype=x.dtype, device="cuda")
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            B.fp4_linear(x, W, x_amax=xa, y=y[1:tokens + 1], status=status)
            torch.cuda.synchronize()
            assert int(status.item()) == 0 and bool((y[0] == -7.0).all().item()) and bool((y[tokens + 1] == -7.0).all().item())
            y = y[1:tokens + 1]
            _check(y[:, at], _quantized(x, fmt, xa), qw, inp, f"{tokens} tokens, {dtype}")
            if B.fp4_plan(tokens, out, inp, FMT[fmt], quantized=True).splits == splits:      # the same order of sums
                X = B.quantize_fp4(x, FMT[fmt], amax=xa)
                assert torch.equal(B.fp4_linear(X, W, y=torch.empty_like(y)), y)
                same += 1
    assert same > 0


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("tokens,inp,out,dtype,gap", MANY)
def test_many_tokens(fmt, tokens, inp, out, dtype, gap):
    x, w = _x(tokens, inp, dtype, 3 * tokens + inp), _x(out, inp, "f16", out + inp, 0.02)
    xa, wa = B.absmax(x), B.absmax(w)
    W = B.quantize_fp4(w, FMT[fmt], amax=wa)
    rows = _some_rows(out, inp)
    qx, qw, at = _quantized(x, fmt, xa), _quantized(w, fmt, wa, rows), torch.as_tensor(rows, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for a, kw in ((x, {"x_amax": xa}), (B.quantize_fp4(x, FMT[fmt], amax=xa), {})):
        y = torch.full((tokens + 2, out + gap), -7.0, dtype=x.dtype, device="cuda")
        B.fp4_linear(a, W, y=y[1:tokens + 1, :out], status=status, **kw)
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and bool((y[:, out:] == -7.0).all().item())
        assert bool((y[0] == -7.0).all().item()) and bool((y[tokens + 1] == -7.0).all().item())
        _check(y[1:tokens + 1][:, at], qx, qw, inp, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("counts,inp,out,dtype,gap", GROUPED_MANY)
def test_many_tokens_grouped(fmt, counts, inp, out, dtype, gap):
    off = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    rows, x_rows = int(off[-1]), 500
    x = _x(x_rows, inp, dtype, inp)
    idx = torch.randint(0, x_rows, (rows,), generator=torch.Generator().manual_seed(3)).int().cuda()
    ws = [_x(out, inp, "f16", 200 + e, 0.02) for e in range(len(counts))]
    xa, wa = B.absmax(x), torch.zeros(1, device="cuda")
    for w in ws:
        B.absmax(w, wa)
    W = flows.fp4_weight(ws, FMT[fmt])
    o = torch.as_tensor(off).cuda()
    sample = _some_rows(out, inp)
    at = torch.as_tensor(sample, device="cuda")
    qx = _quantized(x, fmt, xa)[idx.cpu().numpy()]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = B.quantize_fp4(x, FMT[fmt], amax=xa, row_index=idx, offsets=o)
    for a, kw in ((x, {"row_index": idx, "x_amax": xa}), (q, {})):
        y = torch.full((rows + 2, out + gap), -7.0, dtype=x.dtype, device="cuda")
        B.fp4_linear_grouped(a, o, W, y=y[1:rows + 1, :out], status=status, **kw)
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and bool((y[:, out:] == -7.0).all().item())
        assert bool((y[0] == -7.0).all().item()) and bool((y[rows + 1] == -7.0).all().item())
        for e, n in enumerate(counts):
            if n:
                part = y[1 + off[e]:1 + off[e + 1]]
                _check(part[:, at], qx[off[e]:off[e + 1]], _quantized(ws[e], fmt, wa, sample), inp, f"expert {e}")


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("offsets,owner", [([0, 20, 20, 20], {0: range(10)}), ([-5, 0, 5, 10], {1: range(5), 2: range(5, 10)}),
                                           ([0, 6, 4, 10], {0: range(4), 2: range(6, 10)}), ([7, 7, 30, 9], {1: range(7, 10)})])
def test_rows_of_clamped_offsets(fmt, offsets, owner):
    """Rows that one expert's clamped range claims are its own; nothing outside the matrix is written."""
    x = _x(10, 128, "bf16", 5)
    ws = [_x(64, 128, "f16", 60 + e, 0.02) for e in range(3)]
    W = flows.fp4_weight(ws, FMT[fmt])
    xa = B.absmax(x)
    wa = torch.stack([w.abs().max().float() for w in ws]).max().reshape(1)
    buffer = torch.full((30, 64), -7.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.fp4_linear_grouped(x, torch.tensor(offsets, dtype=torch.int32, device="cuda"), W, x_amax=xa, y=buffer[10:20], status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 2
    assert bool((buffer[:10] == -7.0).all().item()) and bool((buffer[20:] == -7.0).all().item())
    qx = _quantized(x, fmt, xa)
    for e, rows in owner.items():
        rows = list(rows)
        _check(buffer[10:20][rows], qx[rows], _quantized(ws[e], fmt, wa), 128, f"expert {e}")
