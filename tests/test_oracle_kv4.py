"""Pins of the 4-bit key-value cache's oracle (CPU)."""
import numpy as np

from oracle import fp4_oracle as F
from oracle import kv4_oracle as K


def test_a_rotation_is_a_complex_product_and_keeps_lengths():
    g = np.random.default_rng(1)
    x, freq = g.normal(size=(5, 2, 48)), 10000.0 ** (-np.arange(16) / 16)
    pos, axis = g.integers(0, 100000, size=(3, 5)), np.arange(16) % 3
    for adjacent in (False, True):
        y = K.rotate(x, pos, freq, axis, adjacent)
        a, b = (np.arange(0, 32, 2), np.arange(1, 32, 2)) if adjacent else (np.arange(16), np.arange(16, 32))
        z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * (pos[axis].T * freq))[:, None]
        assert np.allclose(y[..., a], z.real, atol=1e-12) and np.allclose(y[..., b], z.imag, atol=1e-12)
        assert np.array_equal(y[..., 32:], x[..., 32:])
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    # what the rotation is for: products depend on distances alone
    q, k = g.normal(size=(1, 1, 32)), g.normal(size=(1, 1, 32))
    f = freq
    one = (K.rotate(q, [[70]], f) * K.rotate(k, [[50]], f)).sum()
    two = (K.rotate(q, [[1070]], f) * K.rotate(k, [[1050]], f)).sum()
    assert abs(one - two) < 1e-9


def test_page_tables_by_hand():
    table = np.full((3, 3), -1)
    table[0, 0], table[2, :2] = 9, (4, 5)
    got = K.page_tables([15, 0, 32], [2, 0, 1], table, [7, 8, 6], 16, 5, cursor=1)
    assert got[0].tolist() == [[9, 8, -1], [-1, -1, -1], [4, 5, 6]]
    assert got[1].tolist() == [17, 0, 33] and got[2].tolist() == [0, 2, 2, 3]
    assert got[3].tolist() == [0, 0, 2, -1, -1] and got[4].tolist() == [15, 16, 32, 0, 0]
    assert got[5].tolist() == [9 * 16 + 15, 8 * 16, 6 * 16, -1, -1] and got[6] == 3


def test_attention_against_explicit_sums():
    g = np.random.default_rng(2)
    q, k, v = g.normal(size=(3, 4, 8)), g.normal(size=(5, 2, 8)), g.normal(size=(5, 2, 8))
    o, spread = K.attend(q, k, v, 0.3, window=2)
    for j in range(3):
        for h in range(4):
            at = [p for p in range(5) if p <= 2 + j and p > j]
            w = [np.exp(0.3 * sum(q[j, h, d] * k[p, h // 2, d] for d in range(8))) for p in at]
            want = sum(x * v[p, h // 2] for x, p in zip(w, at)) / sum(w)
            assert np.allclose(o[j, h], want) and np.all(spread[j, h] >= np.abs(o[j, h]) - 1e-12)
    # a NaN behind a row's own place stays out of it; a row that sees nothing is zero
    v[4] = np.nan
    o, _ = K.attend(q, k, v, 0.3)
    assert np.isfinite(o[:2]).all() and np.isnan(o[2]).all()
    assert not K.attend(q, k[:1], v[:1], 0.3)[0][:2].any()


def test_values_of_the_cache_are_exact_in_fp16():
    levels = (F.LEVELS[:, None] * F.E4M3[None]).ravel()
    assert np.array_equal(levels.astype(np.float16).astype(np.float64), levels)
