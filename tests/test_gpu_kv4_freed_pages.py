"""Attention with a window over tables whose pages behind the window were given back."""
import numpy as np
import pytest
import torch

from kv4_helpers import Batch, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("freed", [-1, 10 ** 9])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("more_tokens", [0, 1 << 20], ids=["narrow", "wide"])
@pytest.mark.parametrize("new", [[1] * 33, [3] * 33, [40] * 3])
def test_pages_that_no_row_sees_are_not_looked_at(monkeypatch, new, more_tokens, page, causal, freed):
    """Every place of the window's begin in two pages of 16; the status stays what it was."""
    monkeypatch.setattr(Batch, "more_tokens", more_tokens)
    window = 50
    lengths = [400 + i * (1 if len(new) > 3 else 16) for i in range(len(new))]
    b = Batch(lengths, new, 4, 2, 64, page)
    want = b.want(causal=causal, window=window)
    for i, (n, m) in enumerate(zip(lengths, new)):
        b.table[i, :(n - m - window + 1) // page] = freed
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = b.run(causal=causal, window=window, status=status)
    check(got, *want)
    assert int(status.item()) == 0
    b.table[0, (lengths[0] - new[0] - window + 1) // page] = freed      # one that the first row sees
    b.run(causal=causal, window=window, status=status)
    assert int(status.item()) == 11
