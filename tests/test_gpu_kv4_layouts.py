"""Attention over the 4-bit cache in the kernel for many rows (tables too wide for small calls): orders and alignments of queries and results,
pages beyond 2^32, numbers that are clamped."""
import numpy as np
import pytest
import torch

from kv4_helpers import Batch, check
from oracle import kv4_oracle as K
from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
WIDE = 1 << 20


@pytest.fixture(params=[0, WIDE], ids=["narrow", "wide"])
def reach(request, monkeypatch):
    monkeypatch.setattr(Batch, "more_tokens", request.param)


def _places(rows, heads, dim, dtype):
    """Results of one matrix's rows, with odd gaps, two bytes behind an aligned place, heads in front of tokens."""
    size = rows * (heads + 3) * (dim + 11) + 1
    raw = lambda: torch.full((size,), 9.0, dtype=dtype, device="cuda")
    pitch = (heads + 1) * (dim + 11)
    yield raw()[:rows * (heads + 3) * dim].view(rows, heads + 3, dim)[:, 1:heads + 1]
    yield raw().as_strided((rows, heads, dim), (pitch, dim + 11, 1))
    yield raw()[1:].as_strided((rows, heads, dim), (pitch, dim + 11, 1))
    yield raw()[1:].as_strided((rows, heads, dim), (heads * dim, dim, 1))
    yield raw()[:rows * heads * dim].view(heads, rows, dim).transpose(0, 1)


@pytest.mark.parametrize("heads,kv_heads,dim,dtype", [(6, 2, 80, F16), (4, 4, 128, BF16), (8, 1, 64, F16), (2, 1, 16, BF16)])
@pytest.mark.parametrize("lengths,new", [([40, 300, 150], [40, 150, 3]), ([70], [33])])
def test_orders_of_queries_and_results(reach, lengths, new, heads, kv_heads, dim, dtype):
    b = Batch(lengths, new, heads, kv_heads, dim, 16, dtype, seed=dim)
    want = b.run()
    check(want, *b.want())
    rows = sum(new)
    for q, out in zip(_places(rows, heads, dim, dtype), list(_places(rows, heads, dim, dtype))[::-1]):
        q.copy_(b.q)
        whole = out._base if out._base is not None else out
        before = whole.clone()
        got = B.kv4_attention(q, b.cache, b.table, b.lengths, b.offsets, out=out)
        assert torch.equal(got, want)
        out.fill_(9.0)                                   # nothing beside the results was written
        assert torch.equal(whole, before)
        assert torch.equal(B.kv4_attention(q, b.cache, b.table, b.lengths, b.offsets, out=q), want)


def test_a_cache_beyond_32_bits_for_many_rows():
    """Pages whose bytes lie beyond 2^32 of the buffers' start, and entries of the table beyond what the tokens need."""
    heads, page, n = 32, 1024, 40
    n_pages = (1 << 32) // (2 * heads * page * 64) + 3
    cache = B.Kv4Cache(n_pages, page, heads, 128)
    last = n_pages - 1
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(n, heads, 128, generator=g).bfloat16().cuda() for _ in range(3))
    B.kv4_append(k, v, cache, (last * page + torch.arange(n)).int().cuda())
    table = torch.full((1, WIDE // page), 10 ** 9, dtype=torch.int32, device="cuda")
    table[0, 0] = last
    ints = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    status = ints(0)
    out = B.kv4_attention(q, cache, table, ints(n), ints(0, n), status=status)
    kq, vq = (K.quantize(x.double().cpu().numpy())[2] for x in (k, v))
    want, spread = K.attend(q.double().cpu().numpy(), kq, vq, 128 ** -0.5)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * spread)
    assert int(status.item()) == 0


@pytest.mark.parametrize("new", [[1, 2], [40, 3], [3, 40], [150, 40]])
def test_requests_beside_one_whose_numbers_are_clamped(reach, new):
    """Offsets in front of the first row and behind the last one, lengths below zero and beyond the table: the other request's rows are
    right, and so are a request's whose rows were only clamped; rows around the results stay."""
    lengths, rows = [200, 170], sum(new)
    b = Batch(lengths, new, 4, 2, 64, seed=rows)
    want, bound = b.want()
    cut = new[0]
    for offsets, held, fine in (([0, cut, rows + 6], lengths, slice(0, rows)), ([-3, cut, rows], lengths, slice(0, rows)),
                                ([0, cut, rows], [200, 10 ** 9], slice(0, cut)), ([0, cut, rows], [-5, 170], slice(cut, rows)),
                                ([0, cut, 2 ** 31 - 1], [-2 ** 31, 170], slice(cut, rows))):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        around = torch.full((rows + 8, 4, 64), 5.0, dtype=BF16, device="cuda")
        out = around[4:4 + rows]
        B.kv4_attention(b.q, b.cache, b.table, torch.tensor(held, dtype=torch.int32).cuda(), torch.tensor(offsets, dtype=torch.int32).cuda(),
                        out=out, status=status)
        assert int(status.item()) in (2, 11)
        check(out[fine], want[fine], bound[fine])
        assert bool((around[:4] == 5).all()) and bool((around[4 + rows:] == 5).all())
        if held[0] < 0:
            assert not bool(out[:cut].any())
