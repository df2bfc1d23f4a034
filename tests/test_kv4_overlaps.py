"""Results of the calls around the 4-bit key-value cache that would be written over what is read: refused on the host, before anything is
launched.  What may lie where gets as far as the next check, a missing list of slots or a missing workspace (CPU)."""
import pytest

from paper_2309_15531_b200 import binding as B
from test_kv4_refusals import NULL, PARAM, append, attention, cache, rotary, tables

N, D, HEADS, KV = 3, 64, 4, 2                            # tokens, and what the calls of test_kv4_refusals have
FAR = 1 << 20
ROW = (HEADS + 2 * KV) * D                               # one projection's result: queries, keys and values side by side


def column(head, base=FAR, size=2):
    return base + head * D * size, ROW, D


QKV = dict(q=column(0), k=column(HEADS), v=column(HEADS + KV))


def run(rotated=True, adjacent=0, **places):
    """As far as the list of slots, which is missing."""
    given = {**QKV, **places}
    if not rotated:
        given.pop("q")
    return append(**given, slots=None, rotary=rotary(dim=64, adjacent=adjacent) if rotated else None, dtype=given.pop("dtype", B.BF16))


OWN = dict(qr=(4 * FAR, HEADS * D, D), kv=(5 * FAR, KV * D, D), vv=(6 * FAR, KV * D, D))


@pytest.mark.parametrize("places", [
    OWN, dict(qr=column(0)), dict(qr=column(0), kv=OWN["kv"], vv=column(HEADS + KV)),
    # behind one another without a gap
    dict(qr=OWN["qr"], kv=(FAR + N * ROW * 2, KV * D, D)), dict(qr=OWN["qr"], kv=(FAR - N * KV * D * 2, KV * D, D)),
    # another part of the same matrix's rows, every second head, the second half of every head
    dict(q=(FAR, 2 * ROW, D), k=(FAR + 512, 2 * ROW, D), v=(FAR + 768, 2 * ROW, D), qr=(FAR + ROW * 2, 2 * ROW, D), kv=(FAR + ROW * 2 + 512, 2 * ROW, D)),
    dict(q=(FAR, 2 * ROW, 2 * D), k=(FAR + 1024, 2 * ROW, 2 * D), v=(FAR + 1536, 2 * ROW, 2 * D), qr=(FAR + 2 * D, 2 * ROW, 2 * D),
         kv=(FAR + 1024 + 2 * D, 2 * ROW, 2 * D)),
    # heads in front of tokens
    dict(q=(FAR, D, N * D), k=(FAR + 4 * N * D * 2, D, N * D), v=(FAR + 6 * N * D * 2, D, N * D), qr=(FAR, D, N * D), vv=(FAR + 6 * N * D * 2, D, N * D)),
    dict(q=(FAR, D, 2 * N * D), k=(2 * FAR, D, N * D), v=(3 * FAR, D, N * D), qr=(FAR + N * D * 2, D, 2 * N * D))])
def test_results_that_share_nothing(places):
    assert run(**{**dict(qr=OWN["qr"]), **places}) == NULL


@pytest.mark.parametrize("places", [
    dict(kv=column(HEADS)),                              # a key's halves: other threads' numbers
    dict(kv=column(HEADS + KV)), dict(vv=column(HEADS)), dict(kv=column(0)), dict(vv=column(0)),
    dict(kv=OWN["vv"], vv=OWN["vv"]), dict(kv=OWN["qr"]), dict(vv=OWN["qr"]),
    dict(qr=column(1)), dict(qr=column(HEADS)), dict(qr=column(2)), dict(qr=(FAR + 2, ROW, D)), dict(qr=(FAR, ROW + D, D)),
    dict(kv=(FAR + N * ROW * 2 - 2, KV * D, D)), dict(kv=(FAR - N * KV * D * 2 + 2, KV * D, D)),
    dict(vv=(*column(HEADS + KV),), vdt=B.F32),          # the same place in another size
    dict(kv=(5 * FAR, 0, D)), dict(kv=(5 * FAR, KV * D, 0)), dict(vv=(5 * FAR, KV * D, D - 1)), dict(qr=(5 * FAR, D, D)), dict(qr=(5 * FAR, -D + 1, D * N))])
def test_results_over_what_is_read_or_written_beside_them(places):
    assert run(**{**dict(qr=OWN["qr"]), **places}) == PARAM


def test_keys_that_are_not_turned_in_halves_may_be_replaced_by_their_values():
    assert run(rotated=False, kv=column(HEADS)) == NULL
    assert run(adjacent=1, qr=OWN["qr"], kv=column(HEADS)) == NULL
    assert run(adjacent=1, qr=OWN["qr"], kv=column(HEADS, base=FAR + 2)) == PARAM
    assert run(rotated=False, kv=column(HEADS), vdt=B.F32) == PARAM
    assert append(k=(FAR, ROW, D), v=(2 * FAR, ROW, D), kv=(FAR, ROW, D), vdt=B.F32, dtype=B.F32, slots=None) == NULL


def test_one_token_and_one_head_have_no_strides():
    assert append(n=1, k=(FAR, 0, D), v=(2 * FAR, 5, D), kv=(3 * FAR, 0, D), slots=None) == NULL
    assert append(n=3, k=(FAR, D, 0), v=(2 * FAR, D, 0), kv=(3 * FAR, D, 0), vv=(2 * FAR, D, 7), c=cache(kv_heads=1), slots=None) == NULL


def attend(q, o, rows=N, q_heads=HEADS):
    """As far as the workspace, which is missing."""
    return attention(q=q, o=o, rows=rows, q_heads=q_heads, ws=None)


@pytest.mark.parametrize("q,o", [
    (column(0), column(0)), (column(0), column(HEADS)), (column(0), column(HEADS, size=2, base=FAR + 2 * N * ROW)), (column(0), (FAR + 2 * N * ROW, HEADS * D, D)),
    ((FAR, D, N * D), (FAR, D, N * D)), ((FAR, 2 * HEADS * D, 2 * D), (FAR + 2 * D, 2 * HEADS * D, 2 * D))])
def test_attention_in_the_place_of_its_queries_or_apart_from_them(q, o):
    assert attend(q, o) == NULL


@pytest.mark.parametrize("q,o", [
    (column(0), column(1)), (column(0), (FAR, HEADS * D, D)), (column(0), (FAR + 2 * ROW, ROW, D)), (column(0), (FAR, ROW, 2 * D)),
    (column(0), (4 * FAR, 0, D)), (column(0), (4 * FAR, HEADS * D, 0)), (column(0), (4 * FAR, HEADS * D, D - 8)), (column(0), (4 * FAR, D, D))])
def test_attention_partly_over_its_queries(q, o):
    assert attend(q, o) == PARAM


def test_attention_of_one_row_and_of_one_head():
    assert attend((FAR, 0, D), (4 * FAR, 0, D), rows=1) == NULL
    assert attend((FAR, D, 0), (4 * FAR, D, 0), q_heads=2) == PARAM
    assert attention(q=(FAR, D, 0), o=(4 * FAR, D, 0), q_heads=1, c=cache(kv_heads=1), ws=None) == NULL


PLACES = dict(past=1 << 12, fresh=2 << 12, free=3 << 12, cursor=4 << 12, table=5 << 12, lengths=6 << 12, offsets=7 << 12, requests=8 << 12,
              positions=9 << 12, slots=10 << 12, after=11 << 12)
SIZES = dict(past=2, fresh=2, free=9, cursor=1, lengths=2, offsets=3, requests=3, positions=3, slots=3, after=1)     # what `tables` has
WRITTEN = ("lengths", "offsets", "requests", "positions", "slots", "after")


@pytest.mark.parametrize("name", WRITTEN)
@pytest.mark.parametrize("other", [n for n in PLACES if n != "table"])
def test_tables_written_over_one_another_or_what_is_read(name, other):
    if name == other or (name, other) == ("after", "cursor"):        # the latter has a status of its own
        return
    assert tables(**{**PLACES, name: PLACES[other] + 4 * SIZES[other] - 4}) == PARAM
    assert tables(**{**PLACES, name: PLACES[other] - 4 * SIZES[name] + 4}) == PARAM


@pytest.mark.parametrize("name", [n for n in PLACES if n != "table"])
def test_a_table_over_what_is_read_or_written(name):
    """Rows of 6 entries, 4 of them used, of which the call's is the first 10."""
    for at in (0, 3, 6, 9):
        assert tables(**{**PLACES, name: PLACES["table"] + 4 * at}, ldt=6) == PARAM
    assert tables(**{**PLACES, name: PLACES["table"] - 4 * SIZES[name] + 4}, ldt=6) == PARAM
