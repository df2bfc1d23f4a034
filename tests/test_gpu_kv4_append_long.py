"""kv4_append of long prompts, whose CTAs have several tokens each: what the same tokens give in short pieces, bit by bit."""
import pytest
import torch

from paper_2309_15531_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("adjacent,sections", [(False, (8, 20, 12)), (True, None)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("tokens", [2371, 7103, 7104, 7106, 9001])
def test_long_prompts_and_their_pieces(tokens, dtype, adjacent, sections):
    g = torch.Generator().manual_seed(tokens)
    heads, kv, dim, page = 3, 2, 96, 16
    x = (3.0 * torch.randn(tokens, heads + 2 * kv, dim, generator=g)).to(dtype).cuda()
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
    turn = B.Rotary.of(80, sections=sections, adjacent=adjacent)
    positions = torch.randint(0, 1 << 17, (turn.axes, tokens), generator=g).int().cuda()
    n_pages = -(-tokens // page) + 1
    slots = torch.randperm(n_pages * page, generator=g)[:tokens].int().cuda()
    slots[tokens // 2], slots[tokens - 1] = -1, n_pages * page

    def run(step):
        cache = B.Kv4Cache(n_pages, page, kv, dim)
        out = torch.empty(tokens, heads, dim, dtype=dtype, device="cuda")
        kv_out = torch.empty(2, tokens, kv, dim, dtype=torch.float32, device="cuda")
        for a in range(0, tokens, step):
            at = slice(a, min(a + step, tokens))
            B.kv4_append(k[at], v[at], cache, slots[at], q=q[at], rotary=turn, positions=positions[:, at], q_out=out[at], k_values=kv_out[0, at],
                         v_values=kv_out[1, at])
        return cache.codes, cache.scales, out, kv_out

    assert all(torch.equal(a, b) for a, b in zip(run(tokens), run(500)))
