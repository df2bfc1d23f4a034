"""A cache and tables whose buffers were replaced: appends write to the new ones and attention reads them."""
import pytest
import torch

from kv4_helpers import Batch, check
from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [[1, 1], [3, 70]])
def test_a_cache_that_was_saved_and_loaded(new):
    b = Batch([200, 90], new, 4, 2, 80)
    want = b.run()
    saved = [t.cpu() for t in (b.cache.codes, b.cache.scales, b.cache.amax)]
    old = b.cache.codes, b.cache.scales, b.cache.amax
    cache = B.Kv4Cache(b.n_pages, b.page, b.kv_heads, b.dim)
    cache.codes, cache.scales, cache.amax = (t.cuda() for t in saved)
    b.cache = cache
    for t in old:
        t.zero_()
    assert torch.equal(b.run(), want)
    cache.codes = torch.zeros_like(cache.codes)
    cache.scales = torch.zeros_like(cache.scales)
    B.kv4_append(b.k, b.v, cache, b.slots)
    check(b.run(), *b.want())
    assert not bool(old[0].any()) and not bool(old[1].any())


def test_tables_and_rotary_whose_buffers_were_replaced():
    ints = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    table = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    step = B.PageTables(2, 5)
    old, step.slots = step.slots, torch.zeros_like(step.slots)
    B.page_tables(ints(3, 0), ints(2, 3), table, ints(5, 6, 7), 16, out=step)
    assert step.slots.tolist() == [3, 4, 80, 81, 82] and not bool(old.any())
    turn = B.Rotary.of(32)
    k = torch.randn(5, 2, 32, generator=torch.Generator().manual_seed(0)).cuda()
    cache = B.Kv4Cache(8, 16, 2, 32)
    run = lambda turn: B.kv4_append(k, k, cache, step.slots, q=k, rotary=turn, positions=step.positions)
    kept = turn.freq
    turn.freq = turn.freq * 0.25
    assert torch.equal(run(turn), run(B.Rotary(kept * 0.25))) and not torch.equal(run(turn), run(B.Rotary.of(32)))
