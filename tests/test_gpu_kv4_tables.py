"""Block tables and slot maps against the token-by-token oracle: whole numbers, equal."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as K
from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def _compare(past, new, table, free, page, rows, cursor=None):
    """Runs the call twice (a second one changes nothing) and returns the status."""
    want = K.page_tables(past, new, table, free, page, rows, cursor or 0)
    t, status = _i32(table), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = B.PageTables(len(past), rows)
    for o in (out.requests, out.positions, out.slots):
        o.fill_(123)
    for _ in range(2):
        B.page_tables(_i32(past), _i32(new), t, _i32(free), page, out, cursor=None if cursor is None else _i32([cursor]), status=status)
    got = (t, out.lengths, out.offsets, out.requests, out.positions, out.slots, out.cursor)
    for name, g, w in zip(("table", "lengths", "offsets", "requests", "positions", "slots", "cursor"), got, want):
        assert np.array_equal(g.cpu().numpy().ravel(), np.asarray(w).ravel()), name
    return int(status.item())


def _batch(n, page, seed, most_new=5, held=200, long=0):
    g = np.random.default_rng(seed)
    past, new = g.integers(0, held, n), g.integers(0, most_new + 1, n)
    past[g.random(n) < 0.2] = 0
    new[:long] = g.integers(100, 400, long)
    counts = -(-past // page)
    width = int((-(-(past + new) // page)).max(initial=0)) + 1
    order = g.permutation(int(counts.sum() + (-(-(past + new) // page) - counts).sum()) + 4)
    table, at = np.full((n, width), -1), 0
    for i, c in enumerate(counts):
        table[i, :c] = order[at:at + c]
        at += c
    return past.tolist(), new.tolist(), table, order[at:]


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("n,long", [(1, 0), (3, 1), (64, 0), (255, 2), (257, 0), (1000, 6), (8192, 0)])
def test_against_the_oracle(n, long, page):
    past, new, table, free = _batch(n, page, n + page, held=200 if n < 1000 else 40, long=long)
    assert _compare(past, new, table, free, page, sum(new) + 7) == 0


def test_a_request_at_its_page_s_end_and_requests_without_tokens():
    table = np.full((6, 3), -1)
    table[0, 0], table[1, 0], table[4, :2] = 11, 12, (13, 14)
    assert _compare([16, 15, 0, 0, 32, 0], [1, 1, 0, 16, 0, 0], table, [5, 6, 7], 16, 18) == 0
    assert _compare([0, 0], [0, 0], table[:2], [5], 16, 0) == 0


def test_a_cursor_goes_on_where_the_last_step_ended():
    past, new, table, free = _batch(40, 16, 3)
    free = np.concatenate((np.full(9, 7777), free))
    assert _compare(past, new, table, free, 16, sum(new), cursor=9) == 0


def test_a_list_that_is_used_up_and_a_table_that_is_too_narrow():
    past, new, table, free = _batch(40, 16, 5, most_new=30)
    assert _compare(past, new, table, free[:6], 16, sum(new)) == 11
    assert _compare(past, new, table[:, :6], free, 16, sum(new)) == 11
    assert _compare([0], [5], np.zeros((1, 0)), [3], 16, 5) == 11


def test_too_few_rows_and_bad_counts_are_reported():
    past, new, table, free = _batch(20, 16, 6)
    assert _compare(past, new, table, free, 16, sum(new) - 3) == 2
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = B.page_tables(_i32([3, -1, 2 ** 31 - 1]), _i32([1, 4, 1]), _i32(np.zeros((3, 1))), _i32([1]), 16, rows=2, status=status)
    assert int(status.item()) == 2 and out.lengths.tolist() == [4, 0, 0] and out.slots.tolist() == [3, -1]


def test_strided_tables_graphs_and_streams():
    past, new, table, free = _batch(50, 32, 8, long=2)
    want = K.page_tables(past, new, table, free, 32, sum(new))
    wide = torch.full((50, table.shape[1] + 5), 99, dtype=torch.int32, device="cuda")
    t = wide[:, :table.shape[1]]
    t.copy_(_i32(table))
    p, n, f, out = _i32(past), _i32(new), _i32(free), B.PageTables(50, sum(new))
    graph = torch.cuda.CUDAGraph()
    B.lib()
    with torch.cuda.graph(graph):
        B.page_tables(p, n, t, f, 32, out)
    out.slots.zero_()
    graph.replay()
    assert np.array_equal(out.slots.cpu().numpy(), want[5]) and np.array_equal(t.cpu().numpy(), want[0])
    assert bool((wide[:, table.shape[1]:] == 99).all())
    n.zero_()
    n[4] = 7                                             # other lengths, the same graph
    graph.replay()
    torch.cuda.synchronize()
    w = K.page_tables(past, n.tolist(), t.cpu().numpy(), free, 32, sum(new))
    assert np.array_equal(out.slots.cpu().numpy(), w[5]) and int(out.cursor.item()) == w[6]


def test_refusals_of_the_binding():
    t, two, out = _i32(np.zeros((2, 4))), _i32([1, 1]), B.PageTables(2, 2)
    with pytest.raises(ValueError):
        B.page_tables(two, _i32([1]), t, two, 16, out)
    with pytest.raises(ValueError):
        B.page_tables(two, two, t, two, 16)
    with pytest.raises(ValueError):
        B.page_tables(two, two, t, two, 16, out, rows=3)
    with pytest.raises(ValueError):
        B.page_tables(two, two, t, two, 16, out, cursor=out.cursor)
    with pytest.raises(B.AdadimError):
        B.page_tables(two, two, t, two, 20, out)
    with pytest.raises(AssertionError):
        B.page_tables(two.long(), two, t, two, 16, out)
