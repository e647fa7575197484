"""Refusals of the packed-row operators and the 8-bit cache: on the host, before any launch (no GPU is needed)."""
import ctypes as C
import os

import pytest

import paper_2504_08838_amd as sd2

A = 0x10000  # an aligned address that nothing reads
NULL, SHAPE, BUFFER, RANGE = -1, -2, -4, -6


def _status(fn, *args):
    with pytest.raises(sd2.SD2Error) as e:
        fn(*args)
    return e.value.status


def _cache(**over):
    a = dict(k=A, v=A, ks=A, vs=A, n_slots=4, n_kv=2, max_pos=128, head_dim=64, **{})
    a.update(over)
    return sd2.kv8_cache_init(a["k"], a["v"], a["ks"], a["vs"], a["n_slots"], a["n_kv"], a["max_pos"], a["head_dim"])


def test_cache_descriptor():
    c = _cache()
    assert (c.n_slots, c.n_kv, c.max_pos, c.head_dim, c.k_dev) == (4, 2, 128, 64, A)
    for name in ("k", "v", "ks", "vs"):
        assert _status(lambda: _cache(**{name: 0})) == NULL
        assert _status(lambda: _cache(**{name: A + 4})) == BUFFER
    for bad in (dict(n_slots=0), dict(n_slots=65537), dict(n_kv=0), dict(n_kv=4097), dict(max_pos=0), dict(max_pos=100), dict(max_pos=(1 << 20) + 32),
                dict(head_dim=0), dict(head_dim=24), dict(head_dim=272), dict(head_dim=-16)):
        assert _status(lambda: _cache(**bad)) == SHAPE, bad
    assert sd2.lib().sd2_kv8_cache_init(None, A, A, A, A, 1, 1, 32, 64) == NULL


APPEND = dict(qkv=A, n_heads=4, row_start=A, pos0=A, n_seq=2, n_rows=0, theta=10000.0, rows=A)


@pytest.mark.parametrize("over,status", [
    (dict(qkv=0), NULL), (dict(row_start=0), NULL), (dict(pos0=0), NULL), (dict(rows=0), NULL), (dict(qkv=A + 8), BUFFER), (dict(row_start=A + 4), BUFFER),
    (dict(pos0=A + 4), BUFFER), (dict(rows=A + 2), BUFFER), (dict(n_heads=3), SHAPE), (dict(n_heads=0), SHAPE), (dict(n_heads=2 * 65), SHAPE),
    (dict(n_seq=-1), RANGE), (dict(n_seq=5), RANGE), (dict(n_rows=-1), RANGE), (dict(n_rows=(1 << 24) + 1), RANGE), (dict(theta=1.0), RANGE),
    (dict(theta=float("nan")), RANGE), (dict(theta=float("inf")), RANGE), (dict(n_heads=128, n_rows=1 << 24), RANGE)])
def test_append_refuses(over, status):
    a = {**APPEND, **over}
    assert _status(sd2.kv8_append, _cache(), a["qkv"], a["n_heads"], a["row_start"], a["pos0"], a["n_seq"], a["n_rows"], a["theta"], a["rows"]) == status


PROMPT = dict(q=A, k=A, v=A, qs=256, kvs=128, row_start=A, n_seq=2, n_rows=0, n_heads=4, n_kv=2, head_dim=64, out=A)


@pytest.mark.parametrize("over,status", [
    *[({n: 0}, NULL) for n in ("q", "k", "v", "row_start", "out")], *[({n: A + 8}, BUFFER) for n in ("q", "k", "v", "row_start", "out")],
    (dict(qs=248), SHAPE), (dict(qs=260), SHAPE), (dict(kvs=120), SHAPE), (dict(kvs=132), SHAPE), (dict(qs=(1 << 24) + 8), SHAPE), (dict(kvs=-128), SHAPE),
    (dict(n_heads=5), SHAPE), (dict(n_kv=0), SHAPE), (dict(n_heads=130), SHAPE), (dict(head_dim=20), SHAPE), (dict(head_dim=288), SHAPE),
    (dict(n_seq=-1), RANGE), (dict(n_seq=65537), RANGE), (dict(n_rows=-1), RANGE), (dict(n_rows=(1 << 24) + 1), RANGE)])
def test_prompt_attention_refuses(over, status):
    assert _status(sd2.prompt_attention, *{**PROMPT, **over}.values()) == status


ATTEND = dict(q=A, qs=256, n_heads=4, row_start=A, pos0=A, n_seq=2, n_rows=0, max_new=5, out=A, ws=A, ws_bytes=1 << 40)


@pytest.mark.parametrize("over,status", [
    *[({n: 0}, NULL) for n in ("q", "row_start", "pos0", "out", "ws")], *[({n: A + 8}, BUFFER) for n in ("q", "row_start", "pos0", "out", "ws")],
    (dict(ws_bytes=64), BUFFER), (dict(qs=248), SHAPE), (dict(qs=257), SHAPE), (dict(n_heads=3), SHAPE), (dict(n_seq=-1), RANGE), (dict(n_seq=5), RANGE),
    (dict(n_rows=-1), RANGE), (dict(max_new=0), RANGE), (dict(max_new=65), RANGE)])
def test_cached_attention_refuses(over, status):
    assert _status(sd2.kv8_attention, _cache(), *{**ATTEND, **over}.values()) == status


def test_cached_attention_workspace():
    c = _cache()
    small, large = sd2.kv8_attention_workspace_size(c, 4, 1, 1), sd2.kv8_attention_workspace_size(c, 4, 4, 64)
    assert 0 < small <= large
    for args, status in (((3, 1, 1), SHAPE), ((4, 5, 1), RANGE), ((4, -1, 1), RANGE), ((4, 1, 0), RANGE), ((4, 1, 65), RANGE)):
        assert _status(sd2.kv8_attention_workspace_size, c, *args) == status
    large = _cache(n_slots=65536, n_kv=1)
    assert sd2.kv8_attention_workspace_size(large, 64, 65536, 64) > 0
    many = _cache(n_slots=65536, n_kv=4096)
    assert _status(sd2.kv8_attention_workspace_size, many, 4096, 65536, 64) == RANGE  # more than 2^30 rows of heads
    assert sd2.lib().sd2_kv8_attention_workspace_size(C.byref(c), 4, 1, 1, None) == NULL
    assert sd2.lib().sd2_kv8_attention_workspace_size(None, 4, 1, 1, C.byref(C.c_size_t())) == NULL


def test_a_spoiled_descriptor_is_refused_by_every_call():
    c = _cache()
    c.max_pos = 100
    assert _status(sd2.kv8_append, c, *APPEND.values()) == SHAPE
    assert _status(sd2.kv8_attention, c, *ATTEND.values()) == SHAPE


def test_no_rows_or_sequences_is_a_call_that_does_nothing():
    for over in (dict(n_rows=0), dict(n_seq=0, n_rows=7)):
        sd2.kv8_append(_cache(), *{**APPEND, **over}.values())
        sd2.prompt_attention(*{**PROMPT, **over}.values())
        sd2.kv8_attention(_cache(), *{**ATTEND, **over}.values())


def test_largest_counts_as_the_header_has_them():
    """Sequences up to 65536 and rows up to 2^24, in every call; one more is refused."""
    wide = _cache(n_slots=65536, n_kv=1)
    for n_seq, n_rows in ((65536, 0), (0, 1 << 24)):
        sd2.kv8_append(wide, *{**APPEND, "n_seq": n_seq, "n_rows": n_rows}.values())
        sd2.prompt_attention(*{**PROMPT, "n_seq": n_seq, "n_rows": n_rows}.values())
        sd2.kv8_attention(wide, *{**ATTEND, "n_seq": n_seq, "n_rows": n_rows}.values())
    for over in (dict(n_seq=65537), dict(n_rows=(1 << 24) + 1)):
        assert _status(sd2.kv8_append, wide, *{**APPEND, **over}.values()) == RANGE
        assert _status(sd2.prompt_attention, *{**PROMPT, **over}.values()) == RANGE
        assert _status(sd2.kv8_attention, wide, *{**ATTEND, **over}.values()) == RANGE
    with open(os.path.join(os.path.dirname(__file__), "..", "include", "sd2.h")) as f:
        assert "n_seq (0 .. 65536) and n_rows (0 .. 2^24)" in f.read()
