"""The expert feed-forward flow: against the oracle, and at the ends of its range."""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from paper_2309_15531_b200 import binding as B
from paper_2309_15531_b200 import flows

pytestmark = pytest.mark.gpu


def _stacks(E, hidden, ffn, fmt, seed=1):
    g = torch.Generator().manual_seed(seed)
    raw = [[(torch.randn(*s, generator=g) * 0.05).half().cuda() for _ in range(E)]
           for s in ((ffn, hidden), (ffn, hidden), (hidden, ffn))]
    return raw, [flows.fp4_weight(w, fmt) for w in raw]


@pytest.mark.parametrize("fmt", [B.MXFP4, B.NVFP4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_a_batch_without_tokens(fmt, dtype):
    _, stacks = _stacks(3, 64, 96, fmt)
    x = torch.empty(0, 64, dtype=dtype, device="cuda")
    experts, weights = torch.empty(0, 2, dtype=torch.int64, device="cuda"), torch.empty(0, 2, device="cuda")
    amax = torch.ones(1, device="cuda")
    y = flows.fp4_expert_ffn(x, experts, weights, *stacks, amax, amax)
    assert y.shape == (0, 64) and y.dtype == dtype
    order, row_index, offsets = flows.rows_by_expert(experts, 3)
    assert order.numel() == row_index.numel() == 0 and offsets.tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("fmt", [B.MXFP4, B.NVFP4])
def test_places_of_no_expert_add_nothing(fmt):
    """Against the same places given to expert 0 with weight 0: a row's sums do not depend on the rows beside it, so the
    bits are the same."""
    E, tokens, top = 3, 40, 2
    _, stacks = _stacks(E, 128, 96, fmt)
    g = torch.Generator().manual_seed(3)
    x = torch.randn(tokens, 128, generator=g).bfloat16().cuda()
    experts = torch.randint(-1, E + 2, (tokens, top), generator=g).cuda()
    weights = torch.rand(tokens, top, generator=g).cuda()
    inside = (experts >= 0) & (experts < E)
    assert bool(inside.any().item()) and not bool(inside.all().item())
    weights[~inside] = float("nan")                       # nobody says what a router writes there
    amax = torch.tensor([8.0], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    trash = torch.full((1 << 22,), float("nan"), device="cuda")           # what freed memory may hold
    del trash
    y = flows.fp4_expert_ffn(x, experts, weights, *stacks, amax, amax, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and bool(torch.isfinite(y).all().item())
    assert not bool(y[~inside.any(1)].any().item()) and bool(y[inside.any(1)].any().item())
    want = flows.fp4_expert_ffn(x, torch.where(inside, experts, 0), torch.where(inside, weights, 0.0), *stacks, amax, amax)
    assert torch.equal(y, want)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens", [5, 260])
def test_the_flow_against_the_oracle(fmt, dtype, tokens):
    """Routing, gather, quantization, products and the weighted sum in binary64, rounded to x's type where the flow keeps a
    matrix (gate, up, silu, their product, down).  Sums in another order can flip such a rounding and, one step further, a
    4-bit code: with bf16 a flip moves an element of the intermediate by 2^-8, a code by up to a fourth of itself, for a
    small part of the elements only.  2^-5 in the norm allows for one element in sixty-four to be a whole code off
    ((1/4) / sqrt(64)); a wrong row, scale or expert is off by about 1."""
    E, top, hidden, ffn = 4, 2, 160, 224
    raw, stacks = _stacks(E, hidden, ffn, B.MXFP4 if fmt == "mx" else B.NVFP4, seed=9)
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn(tokens, hidden, generator=g).to(dtype).cuda()
    experts = torch.stack([torch.randperm(E, generator=g)[:top] for _ in range(tokens)]).cuda()
    weights = torch.rand(tokens, top, generator=g).cuda()
    xa, ha = B.absmax(x), torch.tensor([16.0], device="cuda")
    y = flows.fp4_expert_ffn(x, experts, weights, *stacks, xa, ha)

    def rounded(m):
        return torch.as_tensor(m).to(dtype).double().numpy()

    def quantized(m, amax):
        return F.quantize(m, fmt, float(amax))[2]

    wa = [max(float(w.abs().max().item()) for w in ws) for ws in raw]
    gate, up, down = ([quantized(w.double().cpu().numpy(), wa[k]) for w in ws] for k, ws in enumerate(raw))
    xq, want = quantized(x.double().cpu().numpy(), xa.item()), np.zeros((tokens, hidden))
    for t in range(tokens):
        for k, e in enumerate(experts[t].tolist()):
            a, b = rounded(xq[t] @ gate[e].T), rounded(xq[t] @ up[e].T)
            h = rounded(rounded(a / (1.0 + np.exp(-a))) * b)
            want[t] += float(weights[t, k]) * rounded(quantized(h[None], ha.item())[0] @ down[e].T)
    assert np.linalg.norm(y.double().cpu().numpy() - want) < 2.0 ** -5 * np.linalg.norm(want)
