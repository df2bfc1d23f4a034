"""NVFP4's tensor scale belongs to the codes it was used for: what the caller does with its amax tensor afterwards, in which
order views of a stack are made, and calls that are refused change no product.

Products are compared with products of the same library bit for bit (no order of sums depends on chance), so there is no
tolerance; the scales used are powers of two apart, which a wrong one would show in every element."""
import pytest
import torch

from paper_2309_15531_b200 import binding as B
from paper_2309_15531_b200 import flows

pytestmark = pytest.mark.gpu


def _data(tokens=6, inp=192, out=96, experts=2):
    g = torch.Generator().manual_seed(5)
    x = torch.randn(tokens, inp, generator=g).bfloat16().cuda()
    return x, [(torch.randn(out, inp, generator=g) * 0.02).half().cuda() for _ in range(experts)]


def _amax(v):
    return torch.tensor([float(v)], device="cuda")


def _offsets(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_a_callers_amax_that_changes_later_changes_no_product():
    x, (w, _) = _data()
    wa, xa = B.absmax(w), B.absmax(x)
    W, X = B.quantize_fp4(w, B.NVFP4, amax=wa), B.quantize_fp4(x, B.NVFP4, amax=xa)
    want = B.fp4_linear(X, W)
    B.absmax(w * 1000.0, wa)                              # the way to go over several chunks
    xa.mul_(64.0)
    assert torch.equal(B.fp4_linear(X, W), want)
    wa.zero_()
    assert torch.equal(B.fp4_linear(X, W), want)
    del wa, xa
    assert torch.equal(B.fp4_linear(X, W), want)


def test_a_stack_keeps_the_amax_of_its_first_expert():
    x, ws = _data()
    wa = B.absmax(ws[0])
    B.absmax(ws[1], wa)
    stack = flows.fp4_weight(ws, B.NVFP4)
    other = B.Fp4Tensor(96, 192, B.NVFP4, experts=2)
    for e in range(2):
        B.quantize_fp4(ws[e], B.NVFP4, amax=wa, q=other.expert(e))
    want = B.fp4_linear_grouped(x, _offsets(0, 4, 6), stack)
    wa.fill_(3.0)
    assert torch.equal(B.fp4_linear_grouped(x, _offsets(0, 4, 6), other), want)


def test_a_view_of_an_expert_follows_its_stack():
    x, ws = _data()
    wa = _amax(7.0)
    stack = B.Fp4Tensor(96, 192, B.NVFP4, experts=2)
    early = [stack.expert(e) for e in range(2)]
    for e in range(2):
        B.quantize_fp4(ws[e], B.NVFP4, amax=wa, q=stack.expert(e))
    for e in range(2):
        want = B.fp4_linear(x, B.quantize_fp4(ws[e], B.NVFP4, amax=wa))
        assert torch.equal(B.fp4_linear(x, early[e]), want) and torch.equal(B.fp4_linear(x, stack.expert(e)), want)
    assert float(early[0].amax.item()) == 7.0


def test_an_amax_of_the_stack_that_changes_asks_for_all_experts_again():
    x, ws = _data()
    a, off = _amax(0.1), _offsets(0, 4, 6)
    stack = B.Fp4Tensor(96, 192, B.NVFP4, experts=2)
    B.quantize_fp4(ws[0], B.NVFP4, amax=a, q=stack.expert(0))
    stack.set_amax(None)
    B.quantize_fp4(ws[1], B.NVFP4, q=stack.expert(1))
    with pytest.raises(ValueError):
        B.fp4_linear_grouped(x, off, stack)
    with pytest.raises(ValueError):
        B.fp4_linear_grouped(B.quantize_fp4(x, B.NVFP4, offsets=off), off, stack)
    with pytest.raises(ValueError):
        B.fp4_linear(x, stack.expert(0))
    plain = [B.quantize_fp4(w, B.NVFP4) for w in ws]
    assert torch.equal(B.fp4_linear(x, stack.expert(1)), B.fp4_linear(x, plain[1]))
    B.quantize_fp4(ws[0], B.NVFP4, q=stack.expert(0))
    y = B.fp4_linear_grouped(x, off, stack)
    for e, rows in ((0, slice(0, 4)), (1, slice(4, 6))):
        assert torch.equal(y[rows], B.fp4_linear(x, plain[e])[rows])
    b = _amax(9.0)                                        # the same for a matrix of its own
    one = B.quantize_fp4(ws[0], B.NVFP4, amax=a)
    B.quantize_fp4(ws[0], B.NVFP4, amax=b, q=one)
    assert torch.equal(B.fp4_linear(x, one), B.fp4_linear(x, B.quantize_fp4(ws[0], B.NVFP4, amax=b)))
    one.set_amax(one.amax)
    B.fp4_linear(x, one)
    one.set_amax(a)
    with pytest.raises(ValueError):
        B.fp4_linear(x, one)


def test_an_amax_set_in_advance_is_used():
    x, ws = _data()
    a, off = _amax(0.1), _offsets(0, 4, 6)
    stack = B.Fp4Tensor(96, 192, B.NVFP4, experts=2)
    stack.set_amax(a)
    for e in range(2):
        B.quantize_fp4(ws[e], B.NVFP4, amax=a if e == 0 else stack.amax, q=stack.expert(e))
    y = B.fp4_linear_grouped(x, off, stack)
    assert torch.equal(y[:4], B.fp4_linear(x, B.quantize_fp4(ws[0], B.NVFP4, amax=a))[:4])
    assert torch.equal(y[4:], B.fp4_linear(x, B.quantize_fp4(ws[1], B.NVFP4, amax=a))[4:])
    loaded = B.Fp4Tensor(96, 192, B.NVFP4)                # codes and scales that come from a file
    loaded.codes.copy_(stack.expert(1).codes)
    loaded.scales.copy_(stack.expert(1).scales)
    loaded.set_amax(a)
    a.mul_(2.0)
    assert torch.equal(B.fp4_linear(x, loaded), B.fp4_linear(x, stack.expert(1)))


def test_an_amax_that_grew_between_experts_is_refused():
    x, ws = _data()
    a = B.absmax(ws[0])
    stack = B.Fp4Tensor(96, 192, B.NVFP4, experts=2)
    B.quantize_fp4(ws[0], B.NVFP4, amax=a, q=stack.expert(0))
    want = B.fp4_linear(x, stack.expert(0))
    B.absmax(ws[1] * 100.0, a)
    for wrong in (a, None, _amax(0.5)):
        with pytest.raises(ValueError):
            B.quantize_fp4(ws[1], B.NVFP4, amax=wrong, q=stack.expert(1))
    assert torch.equal(B.fp4_linear(x, stack.expert(0)), want)


def test_a_refused_call_changes_nothing():
    x, (w, _) = _data()
    W = B.quantize_fp4(w, B.NVFP4, amax=B.absmax(w))
    want = B.fp4_linear(x, W)
    with pytest.raises(B.AdadimError):                    # values are bf16 or fp32
        B.quantize_fp4(w, B.NVFP4, amax=_amax(500.0), q=W, values=torch.empty(96, 192, dtype=torch.float16, device="cuda"))
    with pytest.raises(B.AdadimError):
        B.quantize_fp4(w, B.NVFP4, q=W, values=torch.empty(96, 192, dtype=torch.float16, device="cuda"))
    assert torch.equal(B.fp4_linear(x, W), want)


def test_graph_replays_take_the_amax_of_their_time():
    x, (w, _) = _data()
    W, xa = B.quantize_fp4(w, B.NVFP4, amax=B.absmax(w)), B.absmax(x)
    q, y = B.Fp4Tensor(6, 192, B.NVFP4), torch.zeros(6, 96, dtype=torch.bfloat16, device="cuda")

    def step():
        B.quantize_fp4(x, B.NVFP4, amax=xa, q=q)
        B.fp4_linear(q, W, y=y)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    x.mul_(300.0)
    xa.copy_(B.absmax(x))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, B.fp4_linear(x, W, x_amax=xa))


def test_an_amax_or_a_status_of_another_size_is_refused():
    x, (w, w2) = _data()
    W = B.quantize_fp4(w, B.NVFP4, amax=B.absmax(w))
    S = flows.fp4_weight([w, w2], B.NVFP4)
    none, two = torch.empty(0, device="cuda"), torch.ones(2, device="cuda")
    no_status = torch.empty(0, dtype=torch.int32, device="cuda")
    for wrong in (none, two):
        for call in (lambda: B.fp4_linear(x, W, x_amax=wrong), lambda: B.quantize_fp4(w, B.NVFP4, amax=wrong),
                     lambda: B.fp4_linear_grouped(x, _offsets(0, 4, 6), S, x_amax=wrong), lambda: B.absmax(x, wrong),
                     lambda: W.set_amax(wrong)):
            with pytest.raises(AssertionError):
                call()
    for call in (lambda: B.fp4_linear(x, W, status=no_status), lambda: B.fp4_linear(B.quantize_fp4(x, B.NVFP4), W, status=no_status),
                 lambda: B.fp4_linear_grouped(x, _offsets(0, 4, 6), S, status=no_status)):
        with pytest.raises(AssertionError):
            call()


def test_an_amax_that_is_assigned_is_set():
    x, (w, _) = _data()
    a = _amax(0.1)
    W = B.quantize_fp4(w, B.NVFP4, amax=a)
    loaded = B.Fp4Tensor(96, 192, B.NVFP4)
    loaded.codes, loaded.scales, loaded.amax = W.codes.clone(), W.scales.clone(), a
    a.zero_()
    assert torch.equal(B.fp4_linear(x, loaded), B.fp4_linear(x, W))
