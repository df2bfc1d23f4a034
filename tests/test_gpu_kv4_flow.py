"""Block tables, append and attention together, as a server steps a growing batch: against the oracle, eager and in a graph."""
import numpy as np
import pytest
import torch

from oracle import fp4_oracle as F
from oracle import kv4_oracle as K
from paper_2309_15531_b200 import binding as B
from paper_2309_15531_b200 import flows

pytestmark = pytest.mark.gpu

HIDDEN, PAGE, WIDTH = 160, 16, 30


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Layer:
    """A layer's weights on the device and, requantized, with the oracle, which holds each request's keys and values."""

    def __init__(self, heads, kv_heads, dim, dtype, rotary, sections, requests, window):
        g = torch.Generator().manual_seed(dim + heads)
        self.heads, self.kv_heads, self.dim, self.dtype, self.window = heads, kv_heads, dim, dtype, window
        raw = [(torch.randn(o, i, generator=g) * i ** -0.5).to(dtype).cuda() for o, i in
               (((heads + 2 * kv_heads) * dim, HIDDEN), (HIDDEN, heads * dim))]
        self.weights = [flows.fp4_weight(w, B.NVFP4) for w in raw]
        self.plain = [F.quantize(w.double().cpu().numpy(), "nv", float(B.absmax(w).item()))[2] for w in raw]
        self.x_amax, self.out_amax, kv = (torch.tensor([a], device="cuda") for a in (5.0, 4.0, 8.0))
        self.cache = B.Kv4Cache(60, PAGE, kv_heads, dim, kv, kv)
        self.rotary = None if rotary == 0 else B.Rotary.of(rotary, sections=sections)
        self.held = [[np.zeros((0, kv_heads, dim))] * 2 for _ in range(requests)]

    def run(self, x, table, step, positions, max_new, status):
        return flows.fp4_attention(x, *self.weights, self.cache, table, step, self.heads, self.rotary, positions, self.window, max_new,
                                   self.x_amax, self.out_amax, status)

    def want(self, x, new, positions):
        def rounded(m):
            return torch.as_tensor(m).to(self.dtype).double().numpy()
        h, kv, d = self.heads, self.kv_heads, self.dim
        n = sum(new)
        y = rounded(F.quantize(x.double().cpu().numpy()[:n], "nv", 5.0)[2] @ self.plain[0].T).reshape(n, h + 2 * kv, d)
        q, k, v = y[:, :h], y[:, h:h + kv], y[:, h + kv:]
        if self.rotary is not None:
            freq, axis = self.rotary.freq.cpu().numpy(), None if self.rotary.axis is None else self.rotary.axis.cpu().numpy()
            q, k = rounded(K.rotate(q, positions[:, :n], freq, axis)), K.rotate(k, positions[:, :n], freq, axis)
        k, v = K.quantize(k, 8.0)[2], K.quantize(v, 8.0)[2]
        o, at = np.zeros((x.shape[0], h, d)), 0
        for i, m in enumerate(new):
            held = self.held[i] = [np.concatenate((a, b[at:at + m])) for a, b in zip(self.held[i], (k, v))]
            o[at:at + m] = rounded(K.attend(q[at:at + m], *held, d ** -0.5, True, self.window)[0])
            at += m
        return F.quantize(o.reshape(x.shape[0], h * d), "nv", 4.0)[2] @ self.plain[1].T


@pytest.mark.parametrize("heads,kv_heads,dim,dtype,rotary,sections,window", [
    (8, 2, 64, torch.bfloat16, 64, None, 0), (4, 4, 128, torch.float16, 64, (8, 12, 12), 50), (6, 1, 80, torch.bfloat16, 0, None, 0)])
def test_a_batch_that_grows_against_the_oracle(heads, kv_heads, dim, dtype, rotary, sections, window):
    """Prompts, drafted tokens, then single tokens from one captured step whose inputs are all on the device.

    Both sides round the projection to x's type after sums that agree to 2^-20, so about one element in 2^12 differs there.  The
    attention's weights are rounded to fp16, so its results differ by up to 2^-11 before they are rounded, one step of the type in up
    to one element of eight; a step of 2^-7 of an element moves it across the middle of two 4-bit codes, an eighth of its size apart or
    more, in up to a sixteenth of those, and a code is up to a half of the value off: (1/2) / sqrt(128) < 2^-4 of the norm.  A
    wrong page, position or head is off by about 1."""
    news = [(37, 0, 300, 1, 16), (1, 5, 1, 20, 0), (1, 1, 1, 1, 1), (1, 0, 1, 1, 1), (1, 1, 1, 1, 0)]
    n, g = 5, torch.Generator().manual_seed(1)
    layer = Layer(heads, kv_heads, dim, dtype, rotary, sections, n, window)
    table = torch.full((n, WIDTH), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(60, generator=g).int().cuda()
    past, cursor, status = _i32([0] * n), _i32([0]), _i32([0])
    graph = None
    for s, new in enumerate(news):
        rows = sum(new) if s < 2 else 8                               # the captured step has rows to spare
        x = torch.randn(rows, HIDDEN, generator=g).to(dtype).cuda()
        held = past.tolist()
        at = [p + t for p, m in zip(held, new) for t in range(m)] + [0] * (rows - sum(new))
        places = np.array([at, [t // 7 for t in at], [t % 7 for t in at]])
        positions = None if sections is None else _i32(places.tolist())
        if s < 2:
            step = B.page_tables(past, _i32(new), table, free, PAGE, rows=rows, cursor=cursor, status=status)
            y = layer.run(x, table, step, positions, max(new) if s else 0, status)
            past.copy_(step.lengths)
            cursor.copy_(step.cursor)
        else:
            if graph is None:
                static = [x.clone(), _i32(new), None if positions is None else positions.clone()]
                step = B.PageTables(n, rows)
                saved = [t.clone() for t in (past, cursor, table, layer.cache.codes, layer.cache.scales)]

                def body():
                    B.page_tables(past, static[1], table, free, PAGE, out=step, cursor=cursor, status=status)
                    result = layer.run(static[0], table, step, static[2], 1, status)
                    past.copy_(step.lengths)
                    cursor.copy_(step.cursor)
                    return result
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):
                    body()
                torch.cuda.current_stream().wait_stream(side)
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    out = body()
                for to, was in zip((past, cursor, table, layer.cache.codes, layer.cache.scales), saved):
                    to.copy_(was)
            static[0].copy_(x)
            static[1].copy_(_i32(new))
            if positions is not None:
                static[2].copy_(positions)
            graph.replay()
            y = out.clone()
        want = layer.want(x, new, places)
        got = y.double().cpu().numpy()
        assert not got[sum(new):].any()
        for r in range(sum(new)):                                     # row by row, so that a short request's fault is not lost among others
            assert np.linalg.norm(got[r] - want[r]) < 2.0 ** -4 * np.linalg.norm(want[r]), (s, r)
    assert int(status.item()) == 0 and past.tolist() == [sum(m) for m in zip(*news)]
    assert int(cursor.item()) == sum(-(-sum(m) // PAGE) for m in zip(*news))


def test_an_empty_step_and_what_does_not_match():
    layer = Layer(4, 2, 64, torch.bfloat16, 64, None, 0, 0)
    table = torch.zeros(0, 4, dtype=torch.int32, device="cuda")
    step = B.page_tables(_i32([]), _i32([]), table, _i32([3]), PAGE, rows=0)
    y = layer.run(torch.empty(0, HIDDEN, dtype=torch.bfloat16, device="cuda"), table, step, None, 0, None)
    assert y.shape == (0, HIDDEN) and y.dtype == torch.bfloat16
    x = torch.zeros(2, HIDDEN, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        layer.run(x, table, step, None, 0, None)
    step, layer.heads = B.PageTables(0, 2), 3
    with pytest.raises(ValueError):
        layer.run(x, table, step, None, 0, None)
