"""The append with its results in the places of its inputs, and between them."""
import pytest
import torch

from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("tokens", [3, 700])
def test_results_in_the_places_of_what_is_read(tokens, adjacent):
    g = torch.Generator().manual_seed(tokens)
    both = torch.randn(tokens, 8, 2, 64, generator=g).bfloat16().cuda()
    x = both[:, :, 0]                                    # heads with room behind each
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    slots, positions = torch.randperm(tokens + 20, generator=g)[:tokens].int().cuda(), torch.arange(tokens).int().cuda()
    turn, n_pages = B.Rotary.of(32, adjacent=adjacent), -(-(tokens + 20) // 16)

    def run(**more):
        cache = B.Kv4Cache(n_pages, 16, 2, 64)
        kv, vv = more.pop("k_values", torch.empty_like(k)), more.pop("v_values", torch.empty_like(v))
        q_out = B.kv4_append(k, v, cache, slots, q=q, rotary=turn, positions=positions, k_values=kv, v_values=vv, **more)
        return cache.codes, cache.scales, q_out.clone(), kv.clone(), vv.clone()

    want = run()
    room = both[:, :, 1]
    got = run(q_out=room[:, :4], k_values=room[:, 4:6], v_values=room[:, 6:])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    kept = both.clone()
    got = run(q_out=q, v_values=v, **(dict(k_values=k) if adjacent else {}))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    both.copy_(kept)
    if not adjacent:
        with pytest.raises(B.AdadimError):
            run(k_values=k)
    with pytest.raises(B.AdadimError):
        run(k_values=v)
    assert torch.equal(both, kept)


def test_tables_with_their_cursors_beside_them_in_one_buffer():
    ints = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    both = torch.zeros(3, 8, dtype=torch.int32, device="cuda")
    step = B.PageTables(3, 6)
    both[0, 5] = 1
    step.cursor = both[1, 6:7]
    B.page_tables(ints(0, 16, 3), ints(2, 3, 1), both[:, :4], ints(9, 5, 6, 7), 16, out=step, cursor=both[0, 5:6])
    assert both.tolist() == [[5, 0, 0, 0, 0, 1, 0, 0], [0, 6, 0, 0, 0, 0, 3, 0], [0] * 8] and step.slots.tolist() == [80, 81, 96, 97, 98, 3]
    step.cursor = both[2, 3:4]
    with pytest.raises(B.AdadimError):
        B.page_tables(ints(0, 16, 3), ints(2, 3, 1), both[:, :4], ints(9, 5, 6, 7), 16, out=step)
