"""Windows whose begin leaves 32 bits in front of a request's first token are refused on the host (CPU)."""
import struct

import pytest

from paper_2309_15531_b200 import binding as B
from test_kv4_refusals import NULL, SHAPE, cache, heads

MOST = (1 << 31) - 4096


def attention(rows, window, causal, width=(1 << 27) - 256, page=16):
    """Two heads; as far as the workspace, which is missing."""
    qo = struct.pack("6q", *heads(ld=128), *heads(ld=128))
    return B.lib().adadim_kv4_attention(qo, B.BF16, rows, 2, 16, 16, 2, 16, width, width, cache(page=page), 0.1, causal, window, 0, None, None, 0, None)


@pytest.mark.parametrize("rows", [5000, 1 << 29, (1 << 30) - 4096])
def test_rows_and_window_together(rows):
    assert attention(rows, MOST - rows, 0) == NULL
    assert attention(rows, MOST - rows + 1, 0) == SHAPE
    assert attention(rows, MOST - rows + 1, 1) == NULL   # a causal row in front of token 0 sees nothing
    assert attention(rows, MOST, 0) == attention(rows, 0, 0) == NULL      # as long as any request may be: none
    assert attention(rows, 1 << 62, 0) == NULL
