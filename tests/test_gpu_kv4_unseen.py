"""Attention over the 4-bit cache: rows that see nothing give zeros, whatever their queries and the scale are."""
import pytest
import torch

from kv4_helpers import Batch
from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=[0, 1 << 20], ids=["narrow", "wide"])
def reach(request, monkeypatch):
    """Tables that just hold the tokens, and wide ones, which take other kernels."""
    monkeypatch.setattr(Batch, "more_tokens", request.param)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [5, 60, 200])
def test_queries_that_are_not_finite_in_rows_that_see_nothing(rows, dim, dtype, bad):
    """The first rows of a request with more rows than tokens, beside rows that see some: those are NaN where their query is."""
    n = 3
    b = Batch([n, 40], [n, 1], 4, 2, dim, dtype=dtype)
    q = torch.randn(rows + 1, 4, dim, generator=torch.Generator().manual_seed(rows)).to(dtype).cuda()
    offsets = torch.tensor([0, rows, rows + 1], dtype=torch.int32).cuda()
    run = lambda **more: B.kv4_attention(q, b.cache, b.table, b.lengths, offsets, **more)
    want = run()
    q[0, 0, 1], q[1, 3, 0], q[rows - 4, 2, 3], q[rows - 2, 1, 5] = bad, bad, bad, bad
    for max_new in (0, rows, 1):
        got = run(max_new=max_new)
        assert not bool(got[:rows - n].any())
        assert bool(torch.isnan(got[rows - 2, 1]).all())
        rest = torch.ones(rows + 1, 4, dtype=torch.bool, device="cuda")
        rest[rows - 2, 1] = False
        assert not bool(torch.isnan(got[rest]).any())
        assert torch.equal(got[rest], run(max_new=max_new)[rest])
        if max_new == 0:
            assert torch.equal(got[rest], want[rest])


@pytest.mark.parametrize("rows", [5, 60, 200])
def test_pages_outside_the_cache_and_queries_that_are_not_finite(rows):
    b = Batch([rows + 20], [rows], 4, 2, 64)
    b.q[:, 1] = float("nan")
    b.table.fill_(-1)
    assert not bool(b.run(causal=False).any())


@pytest.mark.parametrize("rows", [5, 60, 200])
def test_a_scale_that_is_not_finite(rows):
    b = Batch([3], [3], 4, 2, 64)
    q = torch.ones(rows, 4, 64, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([0, rows], dtype=torch.int32).cuda()
    got = B.kv4_attention(q, b.cache, b.table, b.lengths, offsets, scale=float("nan"))
    assert not bool(got[:rows - 3].any()) and bool(torch.isnan(got[rows - 3:]).all())
