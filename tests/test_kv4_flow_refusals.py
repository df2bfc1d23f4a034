"""flows.fp4_attention refuses what one of its calls would refuse before any of them has run, so that the cache is as it was.  No GPU: the
calls are recorded."""
import types

import pytest
import torch

from paper_2309_15531_b200 import binding as B
from paper_2309_15531_b200 import flows

ROWS, HEADS, KV, D, HIDDEN = 5, 4, 2, 64, 96


@pytest.fixture
def calls(monkeypatch):
    made = []

    def linear(x, w, **more):
        made.append("linear")
        return torch.zeros(x.shape[0], w.rows, dtype=x.dtype)
    monkeypatch.setattr(B, "fp4_linear", linear)
    monkeypatch.setattr(B, "kv4_append", lambda *a, **k: made.append("append"))
    monkeypatch.setattr(B, "kv4_attention", lambda *a, **k: made.append("attention"))
    return made


def run(dtype=torch.bfloat16, heads=HEADS, kv_heads=KV, requests=3, rows=ROWS, table=None, **more):
    matrix = lambda r, c: types.SimpleNamespace(rows=r, cols=c)
    cache = types.SimpleNamespace(head_dim=D, kv_heads=kv_heads)
    step = types.SimpleNamespace(n_rows=rows, n_requests=3, slots=None, positions=None, lengths=None, offsets=None)
    table = torch.zeros(requests, 4, dtype=torch.int32) if table is None else table
    return flows.fp4_attention(torch.zeros(ROWS, HIDDEN, dtype=dtype), matrix((heads + 2 * kv_heads) * D, HIDDEN), matrix(HIDDEN, heads * D), cache,
                               table, step, heads, **more)


def test_a_step_that_fits(calls):
    assert run().shape == (ROWS, HIDDEN) and calls == ["linear", "append", "attention", "linear"]


@pytest.mark.parametrize("change", [
    dict(dtype=torch.float32), dict(heads=5), dict(requests=2), dict(requests=4), dict(rows=6), dict(table=torch.zeros(3, 4, dtype=torch.int64)),
    dict(window=-1), dict(max_new=-1)])
def test_a_step_that_does_not(calls, change):
    with pytest.raises(ValueError):
        run(**change)
    assert calls == []
