"""Pins of the oracle of packed attention and the 8-bit cache: number format by table, scales by hand, attention against oracle/decode.py."""
import numpy as np
import pytest

from oracle import decode as odec
from oracle import kv8


def test_e4m3_decode_by_definition():
    for c in range(256):
        sign, e, f = -1.0 if c >> 7 else 1.0, (c >> 3) & 15, c & 7
        got = kv8.e4m3_decode(np.uint8(c))
        if e == 15 and f == 7:
            assert np.isnan(got)
        else:
            assert got == sign * (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
    assert kv8.e4m3_decode(np.uint8(0x7E)) == 448.0


def test_e4m3_encode_is_nearest_even_among_all_codes():
    codes = np.array([c for c in range(256) if c & 0x7F != 0x7F], dtype=np.uint8)
    assert np.array_equal(kv8.e4m3_encode(kv8.e4m3_decode(codes)), codes)
    mags = kv8.e4m3_decode(np.arange(127, dtype=np.uint8))
    for i in range(126):
        mid = (mags[i] + mags[i + 1]) / 2
        assert kv8.e4m3_encode(mid) == i + (i & 1)
        assert kv8.e4m3_encode(np.nextafter(mid, 0)) == i and kv8.e4m3_encode(np.nextafter(mid, 500)) == i + 1
    assert kv8.e4m3_encode(np.array([np.nan, np.inf, -np.inf])).tolist() == [0x7F] * 3


@pytest.mark.parametrize("largest,exponent", [(448.0, 0), (449.0, 1), (224.0, -1), (225.0, 0), (0.0, -100), (2.0 ** -120, -100), (1.0, -8), (1.75, -8), (1.76, -7)])
def test_block_scale(largest, exponent):
    assert kv8.block_scale(largest) == 2.0 ** exponent


def test_open_block_keeps_the_larger_scale_and_rounds_what_it_holds():
    codes, scales = np.zeros((1, 64, 16), dtype=np.uint8), np.full((1, 2), np.nan)
    kv8.append(codes, scales, np.full((3, 1, 16), 1.0), 0)
    assert scales[0, 0] == 2.0 ** -8 and (kv8.e4m3_decode(codes[0, :3]) == 256.0).all()
    kv8.append(codes, scales, np.full((1, 1, 16), 0.5), 3)          # fits the scale that is there
    assert scales[0, 0] == 2.0 ** -8 and (kv8.e4m3_decode(codes[0, 3]) == 128.0).all()
    kv8.append(codes, scales, np.full((30, 1, 16), 100.0), 4)       # 28 positions here, two in the next block
    assert scales[0].tolist() == [2.0 ** -2, 2.0 ** -2]
    # 100 / 2^-2 = 400 lies half way between 384 (mantissa 100, even) and 416 (101): 384 * 2^-2 = 96
    expected = np.concatenate([np.full((3, 16), 1.0), np.full((1, 16), 0.5), np.full((30, 16), 96.0)])
    assert np.array_equal(kv8.values(codes, scales)[0, :34], expected)


def test_attention_is_the_decode_oracles():
    rng = np.random.default_rng(7)
    q, k, v = rng.standard_normal((3, 6, 16)), rng.standard_normal((2, 20, 16)), rng.standard_normal((2, 20, 16))
    ref = odec.cached_attention(q.reshape(3, 96), k, v, 17, 6, 2, 16)
    out, mass, _ = kv8.attention(q, k, v, [17, 18, 19])
    assert np.allclose(out.reshape(3, 96), ref, rtol=1e-13, atol=1e-13)
    assert (mass >= np.abs(out) - 1e-12).all()
    assert not kv8.attention(q, k, v, [-1, -5, -1])[0].any()


def test_prompt_attention_by_loops():
    rng = np.random.default_rng(8)
    q, k, v = rng.standard_normal((7, 4, 8)), rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 2, 8))
    out = kv8.prompt_attention(q, k, v, [0, 3, 3, 6])[0]
    assert not out[6].any()
    assert np.allclose(out[0], np.repeat(v[0], 2, axis=0)) and np.allclose(out[3], np.repeat(v[3], 2, axis=0))
    s = np.array([q[5, 3] @ k[j, 1] for j in (3, 4, 5)]) / np.sqrt(8.0)
    w = np.exp(s) / np.exp(s).sum()
    assert np.allclose(out[5, 3], w @ v[3:6, 1])


def test_attention_all_rows_at_once_is_row_by_row():
    rng = np.random.default_rng(9)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((2, 9, 8)), rng.standard_normal((2, 9, 8))
    reach = [3, -1, 0, 20, 5]
    odd = v.copy()
    odd[:, 7] = np.nan  # a position that only the fourth row attends to: the others' results are those without it
    for whole, single in zip(kv8.attention(q, k, v, reach), kv8.attention(q, k, odd, reach)):
        assert np.allclose(np.delete(whole, 3, axis=0), np.delete(single, 3, axis=0), rtol=1e-13, atol=1e-13)
    assert np.isnan(kv8.attention(q, k, odd, reach)[0][3]).all()
