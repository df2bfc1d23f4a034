"""Which parts of a head kv4_append rotates: multiples of 8 channels (CPU; as far as the list of slots, which is missing)."""
import pytest

from test_kv4_refusals import NULL, PARAM, append, heads, rotary


@pytest.mark.parametrize("dim", [8, 24, 40, 64])
def test_sizes(dim):
    more = dict(q=heads(1 << 16, 256, 64), qr=heads(2 << 16, 256, 64), slots=None)
    assert append(rotary=rotary(dim=dim), **more) == NULL
    assert append(rotary=rotary(dim=dim + 4), **more) == append(rotary=rotary(dim=dim - 1), **more) == PARAM
    assert append(rotary=rotary(dim=72), **more) == append(rotary=rotary(dim=0), **more) == append(rotary=rotary(dim=-8), **more) == PARAM
