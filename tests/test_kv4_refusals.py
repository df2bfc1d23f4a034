"""What the entry points around the 4-bit key-value cache refuse, found on the host before anything is launched (CPU)."""
import ctypes as C
import struct

import pytest

from paper_2309_15531_b200 import binding as B

OK, NULL, SHAPE, DTYPE, PARAM, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 5, 6


def heads(p=256, ld=1024, lh=64):
    return p, ld, lh


def cache(codes=256, scales=256, n_pages=4, page=16, kv_heads=2, dim=64):
    return C.byref(B.Kv4CacheC(codes, scales, None, n_pages, page, kv_heads, dim))


def test_sizes_of_the_cache():
    size = B.lib().adadim_kv4_bytes
    assert size(3, 16, 2, 128, 0) == 3 * 2 * 2 * 16 * 64 and size(3, 16, 2, 128, 1) == 3 * 2 * 2 * 16 * 8
    assert size(1, 16, 1, 16, 0) == size(1, 16, 1, 64, 0) and size(1, 16, 1, 80, 0) == size(1, 16, 1, 128, 0)
    assert size(1, 16, 1, 144, 1) == size(1, 16, 1, 256, 1) == 2 * 16 * 16
    for bad in ((3, 24, 2, 128), (3, 8, 2, 128), (3, 2048, 2, 128), (3, 16, 0, 128), (3, 16, 2, 0), (3, 16, 2, 72), (3, 16, 2, 272),
                (-1, 16, 2, 128), (1 << 28, 16, 2, 128)):
        assert size(*bad, 0) == 0


def tables(past=16, fresh=16, n=2, page=16, table=16, ldt=4, width=4, free=16, n_free=9, cursor=None, rows=3, lengths=16, offsets=16,
           requests=16, positions=16, slots=16, after=32):
    return B.lib().adadim_page_tables(past, fresh, n, page, table, ldt, width, free, n_free, cursor, rows, lengths, offsets, requests,
                                      positions, slots, after, None, None)


@pytest.mark.parametrize("change,status", [
    (dict(page=24), PARAM), (dict(page=8), PARAM), (dict(page=2048), PARAM), (dict(page=0), PARAM), (dict(n=-1), SHAPE), (dict(n=8193), SHAPE),
    (dict(ldt=3), SHAPE), (dict(width=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(n_free=-1), SHAPE),
    (dict(past=None), NULL), (dict(fresh=None), NULL), (dict(table=None), NULL), (dict(free=None), NULL), (dict(lengths=None), NULL),
    (dict(offsets=None), NULL), (dict(slots=None), NULL), (dict(after=None), NULL), (dict(cursor=32), NULL)])
def test_page_tables(change, status):
    assert tables(**change) == status


def append(q=(0, 0, 0), qr=(0, 0, 0), q_heads=4, k=heads(), v=heads(), dtype=B.F16, n=3, slots=16, rotary=None, c=None, kv=(0, 0, 0), vv=(0, 0, 0), vdt=B.BF16):
    return B.lib().adadim_kv4_append(struct.pack("18q", *k, *v, *q, *qr, *kv, *vv), q_heads, dtype, n, slots, rotary, c or cache(), vdt, None)


def rotary(positions=16, freq=16, axis=16, axes=1, dim=64, adjacent=0):
    return struct.pack("4q4i", positions, freq, axis, 8, axes, dim, adjacent, 0)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), DTYPE), (dict(kv=heads(), vdt=B.F16), DTYPE), (dict(n=-1), SHAPE), (dict(k=heads(0)), NULL), (dict(v=heads(0)), NULL),
    (dict(slots=None), NULL), (dict(q=heads(), rotary=rotary()), NULL), (dict(q=heads(), qr=heads()), PARAM),
    (dict(q=heads(0), qr=heads(), rotary=rotary()), NULL), (dict(rotary=rotary(positions=0)), NULL), (dict(rotary=rotary(freq=0)), NULL),
    (dict(rotary=rotary(axes=0)), PARAM), (dict(rotary=rotary(dim=72)), PARAM), (dict(rotary=rotary(dim=80)), PARAM), (dict(rotary=rotary(dim=0)), PARAM),
    (dict(rotary=rotary(axes=3, axis=0)), NULL), (dict(c=cache(page=48)), PARAM), (dict(c=cache(dim=40)), PARAM), (dict(c=cache(codes=None)), NULL),
    (dict(c=cache(scales=264)), ALIGN), (dict(n=0, k=heads(0), v=heads(0), slots=None), OK)])
def test_append(change, status):
    assert append(**change) == status


def attention(q=heads(), dtype=B.BF16, rows=3, q_heads=4, offsets=16, lengths=16, n=2, table=16, ldt=4, width=4, c=None, window=0, max_new=0,
              o=heads(), ws=256, ws_bytes=None, no_heads=False):
    need = B.lib().adadim_kv4_workspace_bytes(2, 3, 4, 2, 64)
    qo = None if no_heads else struct.pack("6q", *q, *o)
    return B.lib().adadim_kv4_attention(qo, dtype, rows, q_heads, offsets, lengths, n, table, ldt, width, c or cache(), 0.1, 1, window, max_new,
                                        None, ws, need if ws_bytes is None else ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=B.F32), DTYPE), (dict(q_heads=3), PARAM), (dict(q_heads=0), PARAM), (dict(window=-1), PARAM), (dict(max_new=-1), PARAM),
    (dict(rows=-1), SHAPE), (dict(rows=1 << 30), SHAPE), (dict(n=8193), SHAPE), (dict(n=-1), SHAPE), (dict(ldt=3), SHAPE), (dict(width=1 << 30, ldt=1 << 30), SHAPE),
    (dict(no_heads=True), NULL), (dict(q=heads(0)), NULL), (dict(o=heads(0)), NULL), (dict(offsets=None), NULL), (dict(lengths=None), NULL), (dict(table=None), NULL),
    (dict(ws=None), NULL), (dict(ws=264), ALIGN), (dict(ws_bytes=100), WORKSPACE), (dict(c=cache(n_pages=1 << 28)), SHAPE),
    (dict(rows=0, no_heads=True, ws=None), OK), (dict(n=0), OK)])
def test_attention(change, status):
    assert attention(**change) == status


def test_workspace_of_bad_sizes():
    f = B.kv4_workspace_bytes
    assert f(2, 3, 4, 2, 64) > 0
    assert f(-1, 3, 4, 2, 64) == f(2, -1, 4, 2, 64) == f(2, 3, 4, 0, 64) == f(2, 3, 1, 2, 64) == f(2, 3, 4, 2, 300) == 0


def test_rotary_of_bad_sizes():
    import torch
    for bad in (torch.ones(7), torch.ones(129), torch.ones(2, 8)):
        with pytest.raises(ValueError):
            B.Rotary(bad)
    with pytest.raises(ValueError):
        B.Rotary.of(64, sections=(16, 8), device="cpu")


@pytest.mark.parametrize("change", [
    dict(rows=1 << 60), dict(rows=(1 << 29) - 1000), dict(width=1 << 60, ldt=1 << 60), dict(width=(1 << 27) - 1, ldt=1 << 27)])
def test_attention_over_more_than_32_bits_hold(change):
    """Products that would wrap, and rows and tokens whose numbers leave no room for a tile or a chunk beyond the last one."""
    assert attention(**change) == SHAPE
    assert attention(rows=1 << 28, width=1 << 26, ldt=1 << 26, ws=None) == NULL


@pytest.mark.parametrize("change", [
    dict(past=4096, lengths=4096), dict(past=4096, lengths=4100), dict(past=4100, lengths=4096), dict(fresh=4096, lengths=4096),
    dict(past=4096, offsets=4096), dict(fresh=4104, offsets=4096)])
def test_tables_that_would_be_written_over_what_is_read(change):
    apart = dict(past=1024, fresh=1280, lengths=1536, offsets=1792)
    assert tables(**{**apart, **change}) == PARAM
