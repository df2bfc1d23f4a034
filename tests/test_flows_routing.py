"""rows_by_expert on the CPU: rows sorted by expert, and places of no expert."""
import pytest
import torch

from paper_2309_15531_b200 import flows


def _expected(experts, E):
    flat = experts.reshape(-1).tolist()
    order = [i for e in range(E) for i, v in enumerate(flat) if v == e] + [i for i, v in enumerate(flat) if not 0 <= v < E]
    offsets = [0]
    for e in range(E):
        offsets.append(offsets[-1] + flat.count(e))
    return order, [i // experts.shape[1] for i in order], offsets


@pytest.mark.parametrize("dtype", [torch.int64, torch.int32])
@pytest.mark.parametrize("tokens,top,E,low,high", [(7, 2, 4, 0, 4), (7, 2, 4, -2, 7), (1, 1, 1, 0, 1), (5, 3, 2, 2, 9), (0, 2, 3, 0, 3),
                                                   (64, 4, 33, -1, 40)])
def test_rows_by_expert(dtype, tokens, top, E, low, high):
    g = torch.Generator().manual_seed(tokens + top)
    experts = torch.randint(low, high, (tokens, top), generator=g).to(dtype)
    order, row_index, offsets = flows.rows_by_expert(experts, E)
    want = _expected(experts, E)
    assert order.tolist() == want[0] and row_index.tolist() == want[1] and offsets.tolist() == want[2]
    assert row_index.dtype == torch.int32 and offsets.dtype == torch.int32
