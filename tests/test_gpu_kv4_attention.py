"""Attention over the 4-bit cache against the binary64 oracle."""
import numpy as np
import pytest
import torch

from kv4_helpers import Batch, check
from oracle import kv4_oracle as K
from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True, params=[0, 1 << 20], ids=["narrow", "wide"])
def reach(request, monkeypatch):
    """Every test with tables that just hold the tokens, and with tables for so many that no call counts as a small one."""
    monkeypatch.setattr(Batch, "more_tokens", request.param)


def _against(b, **more):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full(b.q.shape, 77.0, dtype=b.q.dtype, device="cuda")
    got = b.run(out=out, status=status, **more)
    more = {k: v for k, v in more.items() if k in ("scale", "causal", "window")}
    check(got, *b.want(**more))
    assert int(status.item()) == 0
    return got


# heads, key heads, head_dim, page
LAYOUTS = [(8, 1, 128, 16), (4, 4, 128, 64), (16, 2, 64, 16), (12, 4, 80, 32), (5, 1, 16, 16), (6, 2, 256, 16), (32, 2, 128, 128),
           (21, 3, 192, 64)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,kv_heads,dim,page", LAYOUTS)
def test_one_token_a_request(heads, kv_heads, dim, page, dtype):
    lengths = [1, 0, 15, 16, 17, 63, 64, 65, 333, 2, 1000]
    _against(Batch(lengths, [1 if n else 0 for n in lengths], heads, kv_heads, dim, page, dtype, seed=dim), max_new=1)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,kv_heads,dim,page", LAYOUTS)
def test_several_tokens_a_request(heads, kv_heads, dim, page, dtype):
    lengths, new = [5, 70, 200, 16, 0, 129, 3], [5, 3, 17, 0, 0, 40, 1]
    b = Batch(lengths, new, heads, kv_heads, dim, page, dtype, seed=dim + 1)
    one = _against(b)
    for max_new in (40, 500):
        two = _against(b, max_new=max_new)
        assert two.shape == one.shape


@pytest.mark.parametrize("heads,kv_heads,dim,page", [(8, 2, 128, 16), (4, 4, 64, 64), (16, 1, 128, 32)])
@pytest.mark.parametrize("lengths,new", [([256], [256]), ([1000, 300], [200, 300]), ([2000, 129, 127, 128], [130, 129, 127, 128])])
def test_prompts(lengths, new, heads, kv_heads, dim, page):
    _against(Batch(lengths, new, heads, kv_heads, dim, page, seed=3))


@pytest.mark.parametrize("window", [1, 5, 16, 17, 100, 5000])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 64), (4, 4, 128), (8, 1, 256)])
def test_windows(heads, kv_heads, dim, causal, window):
    b = Batch([1, 40, 300, 65, 18], [1, 1, 150, 3, 18], heads, kv_heads, dim, seed=window)
    _against(b, window=window, causal=causal)


def test_not_causal_and_a_scale_of_its_own():
    b = Batch([40, 300, 17, 1], [1, 150, 17, 1], 8, 2, 128, seed=1)
    _against(b, causal=False)
    _against(b, scale=0.02)
    _against(b, scale=-0.05)
    _against(b, scale=0.0)


def test_more_rows_than_tokens_and_no_tokens_at_all():
    """The first rows of such a request see nothing: zeros."""
    b = Batch([3, 0, 20], [3, 0, 2], 4, 2, 64)
    q = torch.randn(5 + 2 + 4, 4, 64).bfloat16().cuda()
    offsets = torch.tensor([0, 5, 7, 11], dtype=torch.int32).cuda()
    out = B.kv4_attention(q, b.cache, b.table, b.lengths, offsets)
    k, v = b.values()
    for first, n, lo, hi in ((0, 5, 0, 3), (5, 2, 3, 3), (7, 4, 3, 23)):
        want, spread = K.attend(q[first:first + n].double().cpu().numpy(), k[lo:hi], v[lo:hi], 0.125)
        got = out[first:first + n].double().cpu().numpy()
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * spread)
        assert not got[:max(0, n - (hi - lo))].any()
    assert not bool(B.kv4_attention(q, b.cache, b.table, torch.zeros_like(b.lengths), offsets, causal=False).any())


def test_rows_of_no_request_stay_as_they_were():
    b = Batch([30, 50], [2, 3], 4, 2, 64)
    out = torch.full((5 + 4, 4, 64), 3.0, dtype=BF16, device="cuda")
    q = torch.cat((torch.zeros_like(b.q[:2]), b.q, torch.zeros_like(b.q[:2])))
    B.kv4_attention(q, b.cache, b.table, b.lengths, b.offsets + 2, out=out)
    check(out[2:7], *b.want())
    assert bool((out[:2] == 3).all()) and bool((out[7:] == 3).all())


@pytest.mark.parametrize("new", [1, 4, 60, 140])
def test_what_a_row_does_not_see_does_not_reach_it(new):
    """NaN in keys and values of later tokens (memory behind a request's end is NaN in every test): rows before them stay
    finite, rows from them on are NaN, of a value's NaN in its sixteen channels alone."""
    n = 150
    g = torch.Generator().manual_seed(5)
    k, v = torch.randn(n, 2, 64, generator=g), torch.randn(n, 2, 64, generator=g)
    b0 = n - new
    k[b0 + new // 2, 1, 3] = float("nan")
    v[b0 + new // 3, 0, 20] = float("inf")
    b = Batch([n], [new], 4, 2, 64, k=k, v=v, amax=False)
    got = _against(b)
    assert bool(torch.isnan(got[new - 1, :2, 16:32]).all()) and not bool(torch.isnan(got[new - 1, :2, :16]).any())
    _against(b, window=7)


def test_queries_that_are_not_finite():
    """They spoil their own row and no other."""
    b = Batch([100, 33], [20, 1], 8, 2, 128)
    want, bound = b.want()
    b.q[3, 1, 5], b.q[7, 0, 0], b.q[20, 7, 100] = float("nan"), float("inf"), float("-inf")
    want[3, 1] = want[7, 0] = want[20, 7] = np.nan
    check(b.run(), want, bound)
    check(b.run(max_new=20), want, bound)


@pytest.mark.parametrize("dtype,size", [(BF16, 1e30), (BF16, 1e-30), (BF16, 1e-39), (F16, 60000.0), (F16, 1e-7)])
def test_queries_of_any_size(dtype, size):
    """bf16 queries are scaled by a power of two on their way to fp16; the caller's scale brings the scores back."""
    b = Batch([80], [3], 4, 2, 64, dtype=BF16)
    b.q = (b.q.float() * size / 4.0).to(dtype)
    got = b.run(scale=0.1 / size)
    check(got, *b.want(scale=0.1 / size))


def test_scores_far_apart():
    """A single key takes all the weight; scores that grow and fall along the cache."""
    n = 500
    for order in (1.0, -1.0):
        k = torch.zeros(n, 1, 64)
        k[:, 0, 0] = torch.linspace(-40, 40, n) * order
        b = Batch([n], [1], 8, 1, 64, k=k, v=torch.randn(n, 1, 64, generator=torch.Generator().manual_seed(1)))
        b.q = torch.ones_like(b.q)
        _against(b, scale=1.0)


def test_a_tensor_scale_of_any_size():
    """Keys and values whose amax is far from one: the powers of two enter scores and results."""
    for size in (1e-25, 1e25):
        b = Batch([70], [2], 4, 2, 64, k=torch.randn(70, 2, 64) * size, v=torch.randn(70, 2, 64) * size)
        check(b.run(scale=0.1 / size), *b.want(scale=0.1 / size))


def test_many_requests_of_one_token_and_a_long_one():
    g = np.random.default_rng(2)
    lengths = g.integers(0, 50, 700).tolist() + [20000] + g.integers(0, 50, 300).tolist()
    b = Batch(lengths, [1 if n else 0 for n in lengths], 8, 2, 64)
    _against(b, max_new=1)
    b = Batch([30000], [1], 8, 1, 128, page=64)
    _against(b, max_new=1)
    _against(b)


def test_the_most_requests():
    lengths = [1 + i % 3 for i in range(8192)]
    b = Batch(lengths, [1] * 8192, 2, 1, 16, page=16)
    _against(b, max_new=1)
    with pytest.raises(B.AdadimError):
        B.kv4_attention(b.q, b.cache, torch.cat((b.table, b.table[:1])), torch.cat((b.lengths, b.lengths[:1])),
                        torch.cat((b.offsets, b.offsets[-1:])))


def test_results_do_not_depend_on_timing_and_repeat_bit_by_bit():
    b = Batch([3000, 10, 777, 1500], [1, 1, 30, 140], 16, 2, 128)
    first = b.run()
    for _ in range(5):
        assert torch.equal(b.run(), first)


def test_strided_and_unaligned_queries_and_results():
    b = Batch([40, 90], [3, 2], 6, 2, 80, gap=3, dtype=F16)
    assert not b.q.is_contiguous()
    want = _against(b)
    raw = torch.empty(5 * 7 * 91 + 1, dtype=F16, device="cuda").fill_(9)
    out = raw[1:].as_strided((5, 6, 80), (7 * 91, 91, 1))
    odd = torch.empty(5 * 7 * 91 + 1, dtype=F16, device="cuda")[1:].as_strided((5, 6, 80), (7 * 91, 91, 1))
    odd.copy_(b.q)
    got = B.kv4_attention(odd, b.cache, b.table, b.lengths, b.offsets, out=out)
    assert torch.equal(got, want)
    mine = b.q.contiguous().clone()                      # the result in the queries' place
    B.kv4_attention(mine, b.cache, b.table, b.lengths, b.offsets, out=mine)
    assert torch.equal(mine, want)
    wide = torch.full((2, b.table.shape[1] + 3), 10 ** 9, dtype=torch.int32, device="cuda")
    wide[:, :b.table.shape[1]] = b.table
    assert torch.equal(B.kv4_attention(b.q, b.cache, wide[:, :b.table.shape[1]], b.lengths, b.offsets), want)


def test_pages_out_of_range_are_left_out_and_reported():
    b = Batch([64, 40], [1, 1], 4, 2, 64, amax=False)
    want, _ = b.want()
    for bad in (-1, b.n_pages, 2 ** 31 - 1):
        t, status = b.table.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
        t[0, 1] = bad                                    # tokens 16 .. 31 of request 0
        out = B.kv4_attention(b.q, b.cache, t, b.lengths, b.offsets, status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 11
        k, v = b.values()
        left = [p for p in range(64) if not 16 <= p < 32]
        o, spread = K.attend(b.q[:1].double().cpu().numpy(), k[left], v[left], 0.125)
        assert np.all(np.abs(out[:1].double().cpu().numpy() - o) <= 2.0 ** -8 * np.abs(o) + 2.0 ** -9 * spread)
        assert np.all(np.abs(out[1].double().cpu().numpy() - want[1]) <= 2.0 ** -8 * np.abs(want[1]) + 2.0 ** -9 * 4)


def test_offsets_and_lengths_out_of_range_are_clamped_and_reported():
    b = Batch([64, 40], [1, 2], 4, 2, 64)
    for offsets, lengths in (([0, 1, 9], [64, 40]), ([0, 5, 3], [64, 40]), ([-3, 1, 3], [64, 40]), ([0, 1, 3], [64, 10 ** 9]),
                             ([0, 1, 3], [-5, 40]), ([2 ** 31 - 1, 0, -2 ** 31], [64, 40])):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.kv4_attention(b.q, b.cache, b.table, torch.tensor(lengths, dtype=torch.int32).cuda(),
                        torch.tensor(offsets, dtype=torch.int32).cuda(), status=status)
        assert int(status.item()) in (2, 11)          # clamping may lead past the pages that the table has


def test_a_graph_follows_lengths_tables_and_queries():
    """Captured with other contents; two graphs with workspaces of their own on two streams at once."""
    b = Batch([50, 200, 33], [1, 1, 1], 8, 2, 128)
    lengths, offsets, table, q = b.lengths.clone().fill_(16), b.offsets.clone(), b.table.clone().fill_(0), torch.zeros_like(b.q)
    outs = [torch.empty_like(b.q) for _ in range(2)]
    ws = [torch.empty(B.kv4_workspace_bytes(3, 3, 8, 2, 128), dtype=torch.uint8, device="cuda") for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for gr, out, w in zip(graphs, outs, ws):
        with torch.cuda.graph(gr):
            B.kv4_attention(q, b.cache, table, lengths, offsets, max_new=1, out=out, workspace=w)
    lengths.copy_(b.lengths)
    table.copy_(b.table)
    q.copy_(b.q)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    want = b.want()
    for out in outs:
        check(out, *want)


def test_a_cache_beyond_32_bits():
    """Pages whose bytes and elements lie beyond 2^32 of the buffers' start."""
    heads, page = 32, 1024
    n_pages = (1 << 32) // (2 * heads * page * 64) + 3                # codes of 4.3 GB
    cache = B.Kv4Cache(n_pages, page, heads, 128)
    last = n_pages - 1
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn(20, heads, 128, generator=g).bfloat16().cuda() for _ in range(2))
    slots = (last * page + torch.arange(20)).int().cuda()
    B.kv4_append(k, v, cache, slots)
    q = torch.randn(1, heads, 128, generator=g).bfloat16().cuda()
    table, ints = torch.tensor([[last]], dtype=torch.int32).cuda(), lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    out = B.kv4_attention(q, cache, table, ints(20), ints(0, 1))
    kq, vq = (K.quantize(x.double().cpu().numpy())[2] for x in (k, v))
    want, spread = K.attend(q.double().cpu().numpy(), kq, vq, 128 ** -0.5)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * spread)
    assert not bool(cache.scales[0].any())


def test_nothing_to_do_and_refusals_of_the_binding():
    b = Batch([40, 20], [1, 1], 4, 2, 64)
    assert b.cache.amax is not None
    empty = B.kv4_attention(b.q[:0], b.cache, b.table, b.lengths, torch.zeros_like(b.offsets))
    assert empty.shape == (0, 4, 64)
    run = lambda **bad: B.kv4_attention(**{**dict(q=b.q, cache=b.cache, table=b.table, lengths=b.lengths, offsets=b.offsets), **bad})
    for bad in (dict(q=b.q[:, :3]), dict(q=b.q[..., :48]), dict(table=b.table[:1]), dict(offsets=b.offsets[:2])):
        with pytest.raises(ValueError):
            run(**bad)
    for bad in (dict(offsets=b.offsets.long()), dict(out=b.q.float()), dict(table=b.table.long()), dict(out=b.q[:1])):
        with pytest.raises(AssertionError):
            run(**bad)
    for bad in (dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), dict(window=-1)):
        with pytest.raises(B.AdadimError):
            run(**bad)
    with pytest.raises(KeyError):
        run(q=b.q.double())
    with pytest.raises(B.AdadimError):
        run(q=b.q.float(), out=b.q.float())


@pytest.mark.parametrize("lengths,new", [([300, 170, 40], [40, 130, 9]), ([700], [700])])
def test_many_calls_in_a_row_end_well(lengths, new):
    """No wait inside the kernels runs out, whatever the warps' timing: 600 calls, the status read at the end."""
    b = Batch(lengths, new, 8, 2, 128, seed=11)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    first, out = b.run(), torch.empty_like(b.q)
    for _ in range(600):
        b.run(out=out, status=status)
    assert int(status.item()) == 0 and torch.equal(out, first)


def test_many_rows_that_see_nothing_between_rows_that_do():
    """Requests with hundreds of query rows and fewer tokens, or none: whole 128-row tiles without a token, one after another, beside
    tiles that have work.  Every call gives the first one's bits."""
    heads, kv_heads, dim = 4, 2, 64
    lengths = [(0, 300, 40, 700, 0, 0, 129, 5)[i % 8] for i in range(120)]
    rows = [(200, 200, 130, 256, 150, 64, 300, 128)[i % 8] for i in range(120)]
    b = Batch(lengths, [min(n, m) for n, m in zip(lengths, rows)], heads, kv_heads, dim, seed=11)
    g = torch.Generator().manual_seed(12)
    q = torch.randn(sum(rows), heads, dim, generator=g).bfloat16().cuda()
    offsets = torch.tensor(np.concatenate(([0], np.cumsum(rows))), dtype=torch.int32).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = B.kv4_attention(q, b.cache, b.table, b.lengths, offsets, status=status)
    for _ in range(100):
        assert torch.equal(out, B.kv4_attention(q, b.cache, b.table, b.lengths, offsets, status=status))
    assert int(status.item()) == 0
    k, v = b.values()
    at = row = 0
    for n, m in zip(lengths, rows):
        mine = q[row:row + m].double().cpu().numpy()
        want, spread = K.attend(mine, k[at:at + n], v[at:at + n], dim ** -0.5)
        got = out[row:row + m].double().cpu().numpy()
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * spread)
        at, row = at + n, row + m


@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 8, 64), (16, 2, 128), (8, 1, 256)])
def test_a_hint_that_is_too_small(heads, kv_heads, dim):
    """max_new picks kernels; requests with more rows are worked on all the same."""
    b = Batch([300, 1000, 40, 5], [300, 77, 3, 1], heads, kv_heads, dim, seed=14)
    for hint in (1, 2, 20):
        _against(b, max_new=hint)
        _against(b, max_new=hint, window=60)


def test_many_requests_with_prompts_among_them():
    """More requests than the kernel for many rows takes, so that the one for few rows has them all."""
    n = 3600
    lengths, new = [3 + i % 5 for i in range(n)], [1] * n
    lengths[7], new[7], lengths[3599], new[3599] = 300, 200, 90, 90
    _against(Batch(lengths, new, 2, 1, 64, seed=15))


@pytest.mark.parametrize("heads,kv_heads,dim", [(300, 1, 64), (129, 1, 128), (40, 2, 256)])
def test_more_heads_of_a_key_head_than_rows_of_a_tile(heads, kv_heads, dim):
    b = Batch([200, 33, 1], [3, 1, 1], heads, kv_heads, dim, seed=16)
    for more in (dict(), dict(max_new=3), dict(window=20), dict(causal=False)):
        _against(b, **more)


def test_results_in_the_queries_place():
    for new in ([1, 1, 1], [200, 40, 3]):
        b = Batch([700, 40, 3], new, 8, 2, 128, seed=17)
        want = b.run()
        assert torch.equal(b.run(out=b.q), want)


@pytest.mark.parametrize("dim,dtype", [(128, BF16), (64, F16), (80, BF16)])
def test_rows_that_fill_a_part_of_a_tile(dim, dtype):
    """Query rows a key head around the halves and quarters of a tile, over many chunks, few, and none; some values are NaN."""
    new = [17, 31, 32, 33, 63, 64, 65, 96, 97, 127, 128, 129, 160, 161, 200, 257, 40]
    lengths = [n + (900, 0, 130, 300)[i % 4] for i, n in enumerate(new)]
    b = Batch(lengths, new, 2, 2, dim, dtype=dtype, seed=18)
    _against(b)
    _against(b, window=100)
    _against(b, causal=False)
    b = Batch([5000, 129, 257], [20, 64, 10], 8, 2, dim, dtype=dtype, seed=19)
    _against(b)
    b.v[100, 0, 3] = float("nan")
    B.kv4_append(b.k, b.v, b.cache, b.slots)
    _against(b)
