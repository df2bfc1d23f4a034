"""The calls around the 4-bit key-value cache run on the device of their tables or cache, whatever device is current, and take no tensor
of another device.  No GPU: tensors that only say where they are, and a library that records its calls."""
import pytest
import torch

from paper_2309_15531_b200 import binding as B
from test_binding_devices import Tensor, calls  # noqa: F401  (a fixture)


def _ints(dev, *shape):
    return Tensor(dev, *shape, dtype=torch.int32)


def _cache(dev):
    cache = object.__new__(B.Kv4Cache)
    cache.dev, cache.kv_heads, cache.head_dim, cache._ref = dev, 2, 64, None
    return cache


def _everything(dev, **other):
    """One call of each entry point with everything on `dev`, except what `other` names."""
    at = lambda name: other.get(name, dev)
    out = object.__new__(B.PageTables)
    out.n_requests, out.n_rows, out.dev, out._p = 3, 5, at("out"), [4096 * i for i in range(6)]
    turn = object.__new__(B.Rotary)
    turn.dim, turn.adjacent, turn.axes, turn.dev, turn._freq_p, turn._axis_p = 64, False, 1, at("rotary"), 4096, 0
    heads = lambda name, h: Tensor(at(name), 5, h, 64)
    return {
        "tables": lambda: B.page_tables(_ints(at("past"), 3), _ints(at("new"), 3), _ints(dev, 3, 4), _ints(at("free"), 9), 16, out=out,
                                        cursor=_ints(at("cursor"), 1), status=_ints(at("status"), 1)),
        "append": lambda: B.kv4_append(heads("k", 2), heads("v", 2), _cache(dev), _ints(at("slots"), 5), q=heads("q", 4), rotary=turn,
                                       positions=_ints(at("positions"), 5), q_out=heads("q_out", 4), k_values=heads("k_values", 2),
                                       v_values=heads("v_values", 2)),
        "attention": lambda: B.kv4_attention(heads("q", 4), _cache(dev), _ints(at("table"), 3, 4), _ints(at("lengths"), 3),
                                             _ints(at("offsets"), 4), out=heads("out", 4), status=_ints(at("status"), 1),
                                             workspace=Tensor(at("workspace"), 1024, dtype=torch.uint8)),
    }


@pytest.mark.parametrize("dev", [0, 1])
@pytest.mark.parametrize("entry", ["tables", "append", "attention"])
def test_a_call_runs_on_the_device_of_its_tables_or_cache(calls, entry, dev):  # noqa: F811
    _everything(dev)[entry]()
    assert len(calls) == 1 and calls[0][1:] == (100 + dev, dev)


@pytest.mark.parametrize("entry,name", [
    ("tables", n) for n in ("past", "new", "free", "out", "cursor", "status")] + [
    ("append", n) for n in ("k", "v", "slots", "q", "rotary", "positions", "q_out", "k_values", "v_values")] + [
    ("attention", n) for n in ("q", "table", "lengths", "offsets", "out", "status", "workspace")])
@pytest.mark.parametrize("dev", [0, 1])
def test_a_tensor_of_another_device_is_refused(calls, entry, name, dev):  # noqa: F811
    with pytest.raises((AssertionError, ValueError)):
        _everything(dev, **{name: 1 - dev})[entry]()
    assert calls == []
