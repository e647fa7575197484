"""Oracle for attention of several requests at once and the key/value cache in 8 bits.

TEST INFRASTRUCTURE: only tests, the smoke check and the bench's CPU baseline may import this.

The decoder is that of oracle/decode.py; what is added is bookkeeping (packed rows, a slot per sequence) and the cache's
number format (a choice of this library, the paper has none):

  * a value is an e4m3 code times its block's scale; a block is 32 positions of one head;
  * e4m3: sign, 4 exponent bits with bias 7, 3 mantissa bits; 0x7f and 0xff are NaN, there is no infinity, the largest value is 448;
  * the scale is the smallest power of two 2^e, e >= -100, that brings the block's largest finite magnitude to at most 448;
    when positions are added to a block that needs a larger one, the codes in it are rounded to the new scale.

All arithmetic is float64; powers of two make the divisions exact, so a code is rounded once.
"""

import numpy as np

BLOCK = 32
MIN_EXPONENT = -100

_CODE = np.arange(128)
_MAGNITUDE = np.where(_CODE < 8, _CODE * 2.0 ** -9, (8 + _CODE % 8) * 2.0 ** (_CODE // 8 - 10.0))  # codes 0 .. 0x7e
_MAGNITUDE[127] = np.nan


def e4m3_decode(codes: np.ndarray) -> np.ndarray:
    c = np.asarray(codes, dtype=np.uint8)
    return np.where(c & 0x80, -1.0, 1.0) * _MAGNITUDE[c & 0x7F]


def e4m3_encode(x: np.ndarray) -> np.ndarray:
    """To nearest, ties to even; magnitudes up to 448.  Anything that is not finite becomes 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    mag = np.abs(np.where(finite, x, 0.0))
    if (mag > 448.0).any():
        raise ValueError("beyond the range")
    exponent = np.maximum(np.floor(np.log2(np.where(mag > 0, mag, 1.0))), -6.0)
    step = 2.0 ** (exponent - 3.0)
    code = np.searchsorted(_MAGNITUDE[:127], np.rint(mag / step) * step).astype(np.uint8)
    return np.where(finite, code | np.where(np.signbit(x), 0x80, 0).astype(np.uint8), np.uint8(0x7F))


def block_scale(largest: float) -> float:
    """Smallest 2^e, e >= -100, with largest <= 448 * 2^e."""
    e = MIN_EXPONENT
    while largest > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append(codes: np.ndarray, scales: np.ndarray, x: np.ndarray, pos0: int) -> None:
    """Values x [rows][n_kv][head_dim] enter one slot's codes [n_kv][max_pos][head_dim] and scales [n_kv][max_pos / 32], in place."""
    n_kv, max_pos, _ = codes.shape
    for g in range(n_kv):
        for block in range(max_pos // BLOCK):
            at = [p for p in range(block * BLOCK, (block + 1) * BLOCK) if pos0 <= p < pos0 + len(x)]
            if not at:
                continue
            new = np.stack([x[p - pos0, g] for p in at])
            mag = np.abs(new[np.isfinite(new)])
            scale = block_scale(mag.max() if mag.size else 0.0)
            older = slice(block * BLOCK, max(min(pos0, (block + 1) * BLOCK), block * BLOCK))
            if older.stop > older.start and scales[g, block] > scale:
                scale = float(scales[g, block])
            if older.stop > older.start and scales[g, block] != scale:
                values = e4m3_decode(codes[g, older])
                codes[g, older] = e4m3_encode(values * (float(scales[g, block]) / scale))
            scales[g, block] = scale
            codes[g, at] = e4m3_encode(new / scale)


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """What [n_kv][max_pos][head_dim] codes and their scales stand for."""
    return e4m3_decode(codes) * np.repeat(np.asarray(scales, dtype=np.float64), BLOCK, axis=1)[:, :, None]


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, reach) -> np.ndarray:
    """q [rows][n_heads][D] over k, v [n_kv][positions][D]; row i attends to positions 0 .. reach[i].  Also returns, for error
    bounds, the weighted magnitudes sum_j w_j |v_j| and the largest sum of |q_d k_d| of a row."""
    rows, n_heads, dim = q.shape
    rep = n_heads // k.shape[0]
    reach = np.minimum(np.asarray(reach), k.shape[1] - 1)
    out, mass, dot = np.zeros_like(q), np.zeros_like(q), np.zeros((rows, n_heads))
    some = np.flatnonzero(reach >= 0)
    if not some.size:
        return out, mass, dot
    last = int(reach.max()) + 1
    finite = all(np.isfinite(x).all() for x in (q, k[:, :last], v[:, :last]))
    for h in range(n_heads):
        kk, vv = k[h // rep, :last], v[h // rep, :last]
        if finite:  # all rows at once: a weight of zero for what a row does not attend to
            off = np.arange(last)[None, :] > reach[some, None]
            s = np.where(off, -np.inf, q[some, h] @ kk.T / np.sqrt(float(dim)))
            e = np.exp(s - s.max(axis=1, keepdims=True))
            w = e / e.sum(axis=1, keepdims=True)
            out[some, h], mass[some, h] = w @ vv, w @ np.abs(vv)
            dot[some, h] = np.where(off, 0.0, np.abs(q[some, h]) @ np.abs(kk).T).max(axis=1) / np.sqrt(float(dim))
            continue
        with np.errstate(invalid="ignore", over="ignore"):  # infinities and NaN go their way: only what a row attends to enters
            for i in some:
                n = int(reach[i]) + 1
                s = kk[:n] @ q[i, h] / np.sqrt(float(dim))
                e = np.exp(s - s.max())
                w = e / e.sum()
                out[i, h] = w @ vv[:n]
                mass[i, h] = w @ np.abs(vv[:n])
                dot[i, h] = (np.abs(kk[:n]) @ np.abs(q[i, h])).max() / np.sqrt(float(dim))
    return out, mass, dot


def prompt_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, row_start):
    """Packed rows q [rows][n_heads][D], k, v [rows][n_kv][D]: causal attention inside each sequence; rows of none stay zero."""
    parts = [np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:2])]
    for a, b in zip(row_start[:-1], row_start[1:]):
        got = attention(q[a:b], k[a:b].transpose(1, 0, 2), v[a:b].transpose(1, 0, 2), np.arange(b - a))
        for whole, part in zip(parts, got):
            whole[a:b] = part
    return parts
