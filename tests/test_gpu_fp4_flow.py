"""The expert feed-forward flow at the ends of its range."""
import pytest
import torch

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
