"""A cache in host memory (to be saved, say) is refused by the calls that work on the device.  No GPU."""
import pytest
import torch

from paper_2309_15531_b200 import binding as B


def test_calls_on_a_cache_of_the_host():
    cache, ints = B.Kv4Cache(2, 16, 2, 64, device="cpu"), lambda *n: torch.zeros(*n, dtype=torch.int32)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        B.kv4_append(x, x, cache, ints(3))
    with pytest.raises(AssertionError):
        B.kv4_attention(x, cache, ints(1, 2), ints(1), ints(2))
    with pytest.raises(AssertionError):
        B.page_tables(ints(1), ints(1), ints(1, 2), ints(2), 16, rows=3)
