"""Rows into the 8-bit cache and attention over it, on the GPU against the oracle in 64 bits.

Codes and scales are exact: they follow from the bf16 rows that the call itself returns.  Rows: an angle is off by at most 2^-23
(its fraction of a revolution, up to 1/2, as fp32), sine and cosine by two units of 2^-24, two products and a sum by one each, so a
row's value by at most 2^-21 of |lo| + |hi|, and then half a step of bf16.  Attention: see `bound`.
"""
import numpy as np
import pytest
import torch

import paper_2504_08838_amd as sd2
from oracle import decode as odec
from oracle import kv8
from oracle.bf16 import bits_to_f64
from sd2_workload import gen as wl

import gpu_util as gu

pytestmark = pytest.mark.gpu
THETA = 500000.0
BF16_HALF = 2.0 ** -8  # torch.finfo(bfloat16).eps / 2


def bound(out, mass, dot, dim):
    """How far attention may be off, element by element: half a step for the result, half a step for each weight (together at most that part of
    sum w |v|), and what a score's error does to its weight twice (above and below the fraction): dim sums in fp32 of magnitude `dot` with
    2^-24 each, as much again for the scaling, subtraction and power of two."""
    score = (2 * dim + 16) * 2.0 ** -24 * (dot[..., None] + 1.0)
    return BF16_HALF * np.abs(out) + (1.01 * BF16_HALF + 2 * score) * mass + 1e-30


class Slots:
    """A cache on the GPU; what nothing has been stored in holds NaN codes and NaN scales."""

    def __init__(self, n_slots, n_kv, max_pos, dim):
        self.k, self.v = (torch.full((n_slots, n_kv, max_pos, dim), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.ks, self.vs = (torch.full((n_slots, n_kv, max_pos // 32), float("nan"), device="cuda") for _ in range(2))
        self.c = sd2.kv8_cache_init(self.k.data_ptr(), self.v.data_ptr(), self.ks.data_ptr(), self.vs.data_ptr(), n_slots, n_kv, max_pos, dim)
        self.shape = (n_slots, n_kv, max_pos, dim)

    def host(self):
        return [t.cpu().numpy().copy() for t in (self.k, self.v, self.ks, self.vs)]


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def starts(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def append(slots, x, n_heads, lens, pos0, theta=THETA, n_rows=None):
    rows = torch.full(x.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    rs, p0 = i32(starts(lens)), i32(pos0)
    sd2.kv8_append(slots.c, x.data_ptr(), n_heads, rs.data_ptr(), p0.data_ptr(), len(lens), x.shape[0] if n_rows is None else n_rows, theta,
                   rows.data_ptr(), gu.stream_ptr())
    torch.cuda.synchronize()
    return rows


def attend(slots, q, n_heads, lens, pos0, max_new=None, n_rows=None, out=None):
    dim = slots.shape[3]
    out = torch.full((q.shape[0], n_heads * dim), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    rs, p0 = i32(starts(lens)), i32(pos0)
    max_new = max(lens) if max_new is None else max_new
    nb = sd2.kv8_attention_workspace_size(slots.c, n_heads, len(lens), max_new)
    ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
    sd2.kv8_attention(slots.c, q.data_ptr(), q.stride(0), n_heads, rs.data_ptr(), p0.data_ptr(), len(lens), q.shape[0] if n_rows is None else n_rows,
                      max_new, out.data_ptr(), ws.data_ptr(), nb, gu.stream_ptr())
    torch.cuda.synchronize()
    return out


def f64(t):
    return bits_to_f64(t.view(torch.int16).cpu().numpy().view(np.uint16))


def qkv(seed, n, n_heads, n_kv, dim):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, n_heads + 2 * n_kv, dim)) * np.exp(0.5 * rng.standard_normal((1, n_heads + 2 * n_kv, dim)))
    return torch.from_numpy(x.reshape(n, -1).astype(np.float32)).cuda()


def check_store(before, slots, rows, n_heads, lens, pos0):
    """Codes and scales are those that the returned rows give, everything else is as it was (NaN is any NaN code)."""
    n_slots, n_kv, max_pos, dim = slots.shape
    x = f64(rows).reshape(-1, n_heads + 2 * n_kv, dim)
    k, v, ks, vs = before
    for b, (a, n) in enumerate(zip(starts(lens), lens)):
        at = np.arange(n) + pos0[b]
        on = (at >= 0) & (at < max_pos)
        if on.any():
            kv8.append(k[b], ks[b], x[a:a + n, n_heads:n_heads + n_kv][on], max(pos0[b], 0))
            kv8.append(v[b], vs[b], x[a:a + n, n_heads + n_kv:][on], max(pos0[b], 0))
    for got, want in zip(slots.host(), (k, v, ks, vs)):
        if got.dtype == np.uint8:
            got, want = (np.where(c & 0x7F == 0x7F, np.uint8(0x7F), c) for c in (got, want))
        assert np.array_equal(got, want, equal_nan=True)


HEADS = [(4, 2, 128), (3, 1, 64), (8, 8, 16), (6, 2, 80), (8, 1, 256), (7, 7, 144), (12, 2, 128), (2, 1, 240)]


@pytest.mark.parametrize("n_heads,n_kv,dim", HEADS)
@pytest.mark.parametrize("lens,pos0,max_pos", [
    ([1], [0], 32), ([1], [31], 64), ([1, 1, 1], [32, 63, 95], 96), ([5, 0, 33, 2], [30, 7, 0, 94], 96), ([32], [32], 96), ([64, 65], [1, 31], 128),
    ([40], [-9], 64), ([40], [50], 64), ([3, 4], [-10, 64], 64)])
def test_append(n_heads, n_kv, dim, lens, pos0, max_pos):
    slots, n = Slots(len(lens), n_kv, max_pos, dim), sum(lens)
    before = slots.host()
    x = qkv(11 * dim + n, n, n_heads, n_kv, dim)
    rows = append(slots, x, n_heads, lens, pos0)
    h = x.cpu().numpy().astype(np.float64).reshape(n, -1, dim)
    pos = np.concatenate([np.arange(m) + p for m, p in zip(lens, pos0)])
    turned = n_heads + n_kv
    want = h.copy()
    want[:, :turned] = odec.rope(h[:, :turned].reshape(n, -1), pos, dim, THETA).reshape(n, turned, dim)
    pair = np.abs(h) + np.abs(np.roll(h, dim // 2, axis=2))
    assert (np.abs(f64(rows).reshape(h.shape) - want) <= BF16_HALF * np.abs(want) + 2.0 ** -21 * pair).all()
    check_store(before, slots, rows, n_heads, lens, pos0)


def test_append_step_by_step_is_what_the_oracle_stores():
    """Tokens of growing and shrinking magnitude enter open blocks one or a few at a time; scales never shrink."""
    n_heads, n_kv, dim, max_pos = 2, 1, 64, 96
    slots, at = Slots(2, n_kv, max_pos, dim), 0
    rng = np.random.default_rng(3)
    while at < max_pos:
        n = min(int(rng.integers(1, 6)), max_pos - at)
        before = slots.host()
        x = qkv(100 + at, 2 * n, n_heads, n_kv, dim) * float(2.0 ** rng.integers(-12, 12))
        rows = append(slots, x, n_heads, [n, n], [at, at])
        check_store(before, slots, rows, n_heads, [n, n], [at, at])
        at += n


def test_append_every_bf16_value():
    """All 65536 patterns as values, 32 positions of one magnitude a block, so that every code and every scale occurs."""
    n_heads, n_kv, dim = 1, 1, 64
    bits = np.arange(65536, dtype=np.uint32).reshape(256, 2, 128).transpose(1, 0, 2).reshape(-1, dim)  # sign, exponent, mantissa
    n = len(bits)
    slots = Slots(1, n_kv, n, dim)
    x = torch.zeros((n, 3 * dim), device="cuda")
    x[:, 2 * dim:] = torch.from_numpy((bits << 16).view(np.float32).reshape(n, dim)).cuda()
    before = slots.host()
    rows = append(slots, x, n_heads, [n], [0])
    kept = rows.view(torch.int16).cpu().numpy().view(np.uint16)[:, 2 * dim:]
    nan = (bits & 0x7FFF) > 0x7F80
    assert np.array_equal(np.where(nan, 0, kept), np.where(nan, 0, bits)) and ((kept[nan] & 0x7FFF) > 0x7F80).all()
    check_store(before, slots, rows, n_heads, [n], [0])


def test_append_infinities_and_nan_do_not_set_the_scale():
    slots = Slots(1, 1, 32, 16)
    x = qkv(5, 4, 1, 1, 16)
    x[1, 16], x[2, 33], x[3, 40] = float("inf"), float("nan"), float("-inf")
    before = slots.host()
    rows = append(slots, x, 1, [4], [0])
    check_store(before, slots, rows, 1, [4], [0])
    assert torch.isfinite(slots.ks[0, 0, 0]) and float(slots.ks[0, 0, 0]) < 1.0


@pytest.mark.parametrize("pos", [1 << 17, (1 << 20) - 2, (1 << 31) - 4])
def test_append_far_positions(pos):
    """Angles of a hundred thousand revolutions: the fraction is what counts.  Positions past the cache are rotated and not stored."""
    n_heads, n_kv, dim = 2, 1, 128
    slots = Slots(1, n_kv, 1 << 20, dim)
    x = qkv(6, 2, n_heads, n_kv, dim)
    rows = append(slots, x, n_heads, [2], [pos])
    h = x.cpu().numpy().astype(np.float64)
    want = odec.rope(h[:, :3 * dim], [pos, pos + 1], dim, THETA).reshape(2, 3, dim)
    pair = np.abs(h[:, :3 * dim].reshape(2, 3, dim))
    pair = pair + np.roll(pair, dim // 2, axis=2)
    # a frequency is off by a few units of 2^-53, the angle by the position times that
    tol = BF16_HALF * np.abs(want) + (2.0 ** -21 + pos * 2.0 ** -49) * pair
    assert (np.abs(f64(rows)[:, :3 * dim].reshape(2, 3, dim) - want) <= tol).all()
    stored = ((slots.k & 0x7F) != 0x7F).any(dim=3)[0, 0].nonzero().flatten().tolist()
    assert stored == ([pos, pos + 1] if pos < 1 << 20 else [])


def test_append_leaves_rows_behind_the_last_sequence():
    slots = Slots(2, 1, 64, 32)
    x = qkv(9, 9, 2, 1, 32)
    rows = append(slots, x, 2, [3, 2], [0, 5])
    assert torch.isnan(rows[5:].float()).all() and not torch.isnan(rows[:5].float()).any()


def filled(lens, pos0, n_heads, n_kv, dim, max_pos, seed=1, n_slots=None):
    """A cache with its history and new rows, filled by the operator itself; also what its codes stand for."""
    slots = Slots(n_slots or len(lens), n_kv, max_pos, dim)
    whole = [max(p + n, 0) for p, n in zip(pos0, lens)]
    append(slots, qkv(seed, sum(whole), n_heads, n_kv, dim), n_heads, whole, [0] * len(lens))
    q = (torch.randn(sum(lens) + 3, n_heads * dim + 16, generator=torch.Generator().manual_seed(seed)) * 1.5).to(torch.bfloat16).cuda()
    k, v, ks, vs = slots.host()
    return slots, q, [kv8.values(k[b], ks[b]) for b in range(len(lens))], [kv8.values(v[b], vs[b]) for b in range(len(lens))]


def check_attention(out, q, k, v, n_heads, lens, pos0, dim, max_new=64):
    qd, got = f64(q[:, :n_heads * dim].contiguous()).reshape(-1, n_heads, dim), f64(out).reshape(-1, n_heads, dim)
    for b, (a, n) in enumerate(zip(starts(lens), lens)):
        n = min(n, max_new)
        want, mass, dot = kv8.attention(qd[a:a + n], k[b], v[b], pos0[b] + np.arange(n))
        off = np.abs(got[a:a + n] - want)
        assert np.array_equal(np.isnan(got[a:a + n]), np.isnan(want)), b
        assert (off <= bound(want, mass, dot, dim))[~np.isnan(want)].all(), (b, np.nanmax(off / bound(want, mass, dot, dim)))
    assert (got[sum(lens):] == 7.0).all()


@pytest.mark.parametrize("n_heads,n_kv,dim", HEADS)
@pytest.mark.parametrize("lens,pos0,max_pos", [
    ([1], [0], 32), ([1], [30], 32), ([1, 1], [31, 32], 128), ([5], [428], 1024), ([8, 0, 3, 1], [127, 40, 128, 300], 352), ([64], [0], 64),
    ([33, 64, 17], [0, 70, 255], 288), ([8, 5], [1000, 1019], 1024), ([1, 5], [1500, 3], 1536), ([33, 17, 1, 0], [1290, 40, 0, 7], 1344), ([6, 4], [-3, -4], 32), ([6], [60], 64)])
def test_attention(n_heads, n_kv, dim, lens, pos0, max_pos):
    history = [min(p, max_pos - n) for p, n in zip(pos0, lens)]  # the last case's rows reach past the cache
    slots, q, k, v = filled(lens, history, n_heads, n_kv, dim, max_pos)
    check_attention(attend(slots, q, n_heads, lens, pos0, n_rows=sum(lens)), q, k, v, n_heads, lens, pos0, dim)


@pytest.mark.parametrize("n_heads,n_kv,dim", [(24, 8, 128), (32, 8, 64), (24, 8, 112)])
@pytest.mark.parametrize("max_new", [1, 5, 64])
def test_attention_of_caches_between_one_and_two_thousand_positions(n_heads, n_kv, dim, max_new):
    """So many workgroups that these are not cut either."""
    pos0 = [1200, 0, 700, 33, 1400, 255, 256, 90, 1024, 5, 800, 1300]
    lens = [max(max_new - i % 3, 1) for i in range(12)]
    slots, q, k, v = filled(lens, pos0, n_heads, n_kv, dim, 1472)
    check_attention(attend(slots, q, n_heads, lens, pos0, n_rows=sum(lens)), q, k, v, n_heads, lens, pos0, dim)


@pytest.mark.parametrize("n_heads,n_kv", [(1, 1), (64, 1), (20, 20)])
def test_attention_few_and_many_heads_a_group(n_heads, n_kv):
    lens, pos0 = [2, 9], [200, 77]
    slots, q, k, v = filled(lens, pos0, n_heads, n_kv, 64, 256)
    check_attention(attend(slots, q, n_heads, lens, pos0, n_rows=11), q, k, v, n_heads, lens, pos0, 64)


def test_attention_many_sequences():
    """More than a wavefront has lanes, idle ones among them."""
    rng = np.random.default_rng(21)
    lens, pos0 = rng.integers(0, 4, 150).tolist(), rng.integers(0, 300, 150).tolist()
    slots, q, k, v = filled(lens, pos0, 2, 1, 64, 320)
    check_attention(attend(slots, q, 2, lens, pos0, n_rows=sum(lens)), q, k, v, 2, lens, pos0, 64)


@pytest.mark.parametrize("n_heads,n_kv,dim", [(16, 8, 64), (24, 8, 128), (8, 4, 256), (24, 8, 96)])
def test_attention_more_row_tiles_than_places(n_heads, n_kv, dim):
    """So many sequences that whole stretches go first and what is left of each follows; some idle, some of one position."""
    n_seq = 160
    rng = np.random.default_rng(22)
    lens = rng.choice([0, 1, 1, 2, 5], n_seq).tolist()
    pos0 = (rng.random(n_seq) ** 3 * 1400).astype(int).tolist()
    slots, q, k, v = filled(lens, pos0, n_heads, n_kv, dim, 1440)
    check_attention(attend(slots, q, n_heads, lens, pos0, n_rows=sum(lens)), q, k, v, n_heads, lens, pos0, dim)


def test_attention_of_stretches_of_many_tiles():
    """So many heads that a stretch is longer than what a wavefront holds scales for; three heads against the oracle."""
    n_kv, dim, max_pos, lens, pos0 = 512, 16, 33 * 1024, [2, 1], [33 * 1024 - 2, 20011]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(23)
    slots = Slots(2, n_kv, max_pos, dim)
    for c in (slots.k, slots.v):
        c.copy_((torch.randn(c.shape, generator=gen, device="cuda") * 95).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    for c in (slots.ks, slots.vs):
        c.copy_(torch.exp2(torch.randint(-9, -5, c.shape, generator=gen, device="cuda").float()))
    q = torch.randn(3, n_kv * dim, generator=torch.Generator().manual_seed(24)).to(torch.bfloat16).cuda()
    got = f64(attend(slots, q, n_kv, lens, pos0)).reshape(3, n_kv, dim)
    for h in (0, 77, 511):
        for b, rows in ((0, slice(0, 2)), (1, slice(2, 3))):
            k, v = (kv8.values(c[b, h:h + 1].cpu().numpy(), s[b, h:h + 1].cpu().numpy()) for c, s in ((slots.k, slots.ks), (slots.v, slots.vs)))
            want, mass, dot = kv8.attention(f64(q).reshape(3, n_kv, dim)[rows, h:h + 1], k, v, pos0[b] + np.arange(lens[b]))
            assert (np.abs(got[rows, h:h + 1] - want) <= bound(want, mass, dot, dim)).all()


@pytest.mark.parametrize("n_heads,n_kv,dim", [(4, 2, 64), (24, 8, 128), (8, 2, 256)])
def test_same_bits_every_time(n_heads, n_kv, dim):
    """Over and over, other values in between: what a buffer of LDS or the workspace holds from before never shows."""
    lens, pos0 = [5, 1, 17], [900, 3000, 130]
    slots, q, _, _ = filled(lens, pos0, n_heads, n_kv, dim, 3104)
    first = attend(slots, q, n_heads, lens, pos0, n_rows=23).view(torch.int16)
    for _ in range(20):
        attend(slots, q * 20, n_heads, [3, 20], [2500, 1000], n_rows=23)
        assert torch.equal(attend(slots, q, n_heads, lens, pos0, n_rows=23).view(torch.int16), first)


def test_attention_of_the_first_rows_only():
    lens, pos0 = [7, 5], [50, 60]
    slots, q, k, v = filled(lens, pos0, 4, 2, 64, 96)
    out = attend(slots, q, 4, lens, pos0, max_new=3, n_rows=12)
    got = f64(out)
    assert (got[3:7] == 7.0).all() and (got[10:] == 7.0).all()
    check_attention(out[:12], q, k, v, 4, lens, pos0, 64, max_new=3)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("where", [41, 43])
@pytest.mark.parametrize("max_pos", [64, 1056])  # a cache that is not cut, and one that may be
def test_nan_of_a_later_token_does_not_reach_earlier_rows(dim, where, max_pos):
    """A draft's value is NaN: rows that attend to it have NaN in that dimension, the others the result without it."""
    lens, pos0 = [5], [40]
    slots, q, k, v = filled(lens, pos0, 4, 2, dim, max_pos)
    slots.v[0, 1, where, 3] = 0xFF
    slots.v[0, 0, where, dim - 1] = 0x7F
    v[0][1, where, 3] = v[0][0, where, dim - 1] = np.nan
    out = attend(slots, q, 4, lens, pos0, n_rows=5)
    check_attention(out, q, k, v, 4, lens, pos0, dim)
    assert np.isnan(f64(out)).sum() == 4 * (45 - where)


@pytest.mark.parametrize("max_pos", [64, 1056])
def test_nan_key_reaches_the_rows_that_attend_to_it(max_pos):
    lens, pos0 = [4], [30]
    slots, q, k, v = filled(lens, pos0, 2, 1, 64, max_pos)
    slots.k[0, 0, 32, 5] = 0x7F
    k[0][0, 32, 5] = np.nan
    out = attend(slots, q, 2, lens, pos0, n_rows=4)
    check_attention(out, q, k, v, 2, lens, pos0, 64)
    assert torch.isnan(out[2:4].float()).all() and torch.isfinite(out[:2].float()).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("max_pos,pos0", [(64, 40), (1056, 40), (4096, 700)])  # not cut, in one stretch, in stretches that are joined
def test_values_stored_as_a_number_that_bf16_does_not_have(dim, max_pos, pos0):
    """Drafts' values of nearly 2^128 are stored as 256 times 2^120, more than bf16 and fp32 hold.  Rows in front of them have the result
    without them, the others their part of them, which is finite."""
    n_heads, n_kv, lens = 4, 2, [5]
    slots, q, _, _ = filled([1], [pos0 - 1], n_heads, n_kv, dim, max_pos)
    q = torch.cat([q, q * 0.5])[:5]
    x = qkv(71, 5, n_heads, n_kv, dim)
    at = (n_heads + n_kv) * dim
    x[1, at + dim + 3], x[3, at + dim - 1] = 3.38e38, -3.38e38
    before = slots.host()
    rows = append(slots, x, n_heads, lens, [pos0])
    check_store(before, slots, rows, n_heads, lens, [pos0])
    k, v, ks, vs = slots.host()
    assert v[0, 1, pos0 + 1, 3] == 0x78 and v[0, 0, pos0 + 3, dim - 1] == 0xF8 and (vs[0, :, (pos0 + 1) // 32] == 2.0 ** 120).all()
    k, v = [kv8.values(k[0], ks[0])], [kv8.values(v[0], vs[0])]
    check_attention(attend(slots, q, n_heads, lens, [pos0]), q, k, v, n_heads, lens, [pos0], dim)


def test_large_scores():
    """Scores of thousands: one position takes all the weight, and every running maximum is left far behind."""
    lens, pos0 = [3], [500]
    slots, q, k, v = filled(lens, pos0, 4, 2, 128, 512)
    q = q * 200.0
    want = kv8.attention(f64(q[:3, :512].contiguous()).reshape(3, 4, 128), k[0], v[0], [500, 501, 502])
    got = f64(attend(slots, q, 4, lens, pos0, n_rows=3))[:3].reshape(3, 4, 128)
    # a score's error is a larger part of a weight here: 2^-24 for each of its sums
    assert (np.abs(got - want[0]) <= bound(*want, 128)).all()


def test_offsets_past_32_bits():
    """The second slot of a cache of 8 GiB; its last positions."""
    n_kv, dim, max_pos = 8, 256, 1 << 20
    k = torch.zeros((2, n_kv, max_pos, dim), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    ks, vs = torch.ones((2, n_kv, max_pos // 32), device="cuda"), torch.ones((2, n_kv, max_pos // 32), device="cuda")
    c = sd2.kv8_cache_init(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), 2, n_kv, max_pos, dim)
    x = qkv(31, 4, 8, n_kv, dim)
    slots = Slots.__new__(Slots)
    slots.k, slots.v, slots.ks, slots.vs, slots.c, slots.shape = k, v, ks, vs, c, (2, n_kv, max_pos, dim)
    at = max_pos - 2
    rows = append(slots, x, 8, [2, 2], [0, at])
    h = f64(rows).reshape(4, 24, dim)
    last = v[1, :, at:].cpu().numpy()
    scale = vs[1, :, -1].cpu().numpy()
    for g in range(n_kv):
        want = kv8.block_scale(np.abs(h[2:, 16 + g]).max())
        # positions in front of the two hold zeros under scale 1, which the block keeps
        assert scale[g] == max(want, 1.0)
        assert np.array_equal(last[g], kv8.e4m3_encode(h[2:, 16 + g] / float(scale[g])))
    # keys and values of all other positions are zero: every score is zero or the last two's
    out = f64(attend(slots, rows, 8, [0, 2], [0, at], n_rows=2, out=torch.full((4, 8 * dim), 7.0, dtype=torch.bfloat16, device="cuda")))
    q = h[:2, :8]  # the call's rows are the sequence's: rows 0 and 1
    for i in range(2):
        for g in range(n_kv):
            kk = kv8.e4m3_decode(k[1, g, at:].cpu().numpy())[: i + 1] * float(ks[1, g, -1])
            vv = kv8.e4m3_decode(last[g])[: i + 1] * float(scale[g])
            s = kk @ q[i, g] / 16.0
            top = max(s.max(), 0.0)
            e = np.exp(s - top)
            total = e.sum() + at * np.exp(-top)
            w = e / total
            want = w @ vv
            # sums of a million weights in fp32, 2^-24 of the running sum each time it passes a lane's: far below a step of bf16
            assert (np.abs(out[i].reshape(8, dim)[g] - want) <= 3 * BF16_HALF * (w @ np.abs(vv)) + 1e-30).all()


@pytest.mark.parametrize("max_pos", [512, 2048])
def test_captured_call_serves_new_lengths(max_pos):
    """A graph of append and attention; between replays the offsets, positions and rows change, and so do the results."""
    n_heads, n_kv, dim = 6, 2, 128
    slots = Slots(3, n_kv, max_pos, dim)
    width = (n_heads + 2 * n_kv) * dim
    x = torch.zeros((8, width), device="cuda")
    rows = torch.zeros((8, width), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((8, n_heads * dim), dtype=torch.bfloat16, device="cuda")
    rs, p0 = i32([0, 0, 0, 0]), i32([0, 0, 0])
    nb = sd2.kv8_attention_workspace_size(slots.c, n_heads, 3, 5)
    ws = torch.zeros(nb, dtype=torch.uint8, device="cuda")

    def step(stream):
        sd2.kv8_append(slots.c, x.data_ptr(), n_heads, rs.data_ptr(), p0.data_ptr(), 3, 8, THETA, rows.data_ptr(), stream)
        sd2.kv8_attention(slots.c, rows.data_ptr(), width, n_heads, rs.data_ptr(), p0.data_ptr(), 3, 8, 5, out.data_ptr(), ws.data_ptr(), nb, stream)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(side.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side.cuda_stream)
    whole = [400, 90, 3]
    append(slots, qkv(50, sum(whole), n_heads, n_kv, dim), n_heads, whole, [0, 0, 0])
    for seed, lens in ((1, [5, 1, 2]), (2, [0, 5, 3]), (3, [1, 1, 1]), (4, [4, 0, 0])):
        x.copy_(qkv(seed, 8, n_heads, n_kv, dim))
        rs.copy_(i32(starts(lens)))
        p0.copy_(i32(whole))
        before = slots.host()
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_store(before, slots, rows, n_heads, lens, whole)
        k, v, ks, vs = slots.host()
        check_attention(out, rows, [kv8.values(k[b], ks[b]) for b in range(3)], [kv8.values(v[b], vs[b]) for b in range(3)], n_heads, lens, whole, dim)
        again = attend(slots, rows, n_heads, lens, whole, max_new=5, out=torch.full_like(out, 7.0))
        assert torch.equal(again.view(torch.int16), out.view(torch.int16))
        whole = [w + n for w, n in zip(whole, lens)]


@pytest.mark.parametrize("max_pos", [1024, 1056])
def test_two_streams_at_once(max_pos):
    """Two calls that may overlap, each with its own workspace, give what they give one after the other."""
    lens, pos0 = [5, 3], [900, 30]
    a, qa, _, _ = filled(lens, pos0, 8, 2, 128, max_pos, seed=61)
    b, qb, _, _ = filled(lens, pos0, 8, 2, 128, max_pos, seed=62)
    want = [attend(s, q, 8, lens, pos0, n_rows=8) for s, q in ((a, qa), (b, qb))]
    nb = sd2.kv8_attention_workspace_size(a.c, 8, 2, 5)
    ws, out = [torch.empty(nb, dtype=torch.uint8, device="cuda") for _ in range(2)], [torch.full_like(want[0], 7.0) for _ in range(2)]
    rs, p0, streams = i32(starts(lens)), i32(pos0), [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, (s, q) in enumerate(((a, qa), (b, qb))):
            sd2.kv8_attention(s.c, q.data_ptr(), q.stride(0), 8, rs.data_ptr(), p0.data_ptr(), 2, 8, 5, out[i].data_ptr(), ws[i].data_ptr(), nb,
                              streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(out[i].view(torch.int16), want[i].view(torch.int16))


def test_offsets_that_break_the_rules_stay_inside_the_buffers():
    """Unspecified results, but nothing outside: rows past n_rows and the cache's other slots keep what they hold."""
    slots = Slots(4, 1, 64, 64)
    whole = torch.full((12, 4 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros((12, 6 * 64), device="cuda")
    rows = torch.full((12, 6 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    rs, p0 = i32([5, -3, 1 << 30, 2]), i32([-(1 << 31), (1 << 31) - 1, 40])
    nb = sd2.kv8_attention_workspace_size(slots.c, 4, 3, 4)
    ws = torch.zeros(nb, dtype=torch.uint8, device="cuda")
    sd2.kv8_append(slots.c, x.data_ptr(), 4, rs.data_ptr(), p0.data_ptr(), 3, 8, THETA, rows.data_ptr(), gu.stream_ptr())
    sd2.kv8_attention(slots.c, rows.data_ptr(), 6 * 64, 4, rs.data_ptr(), p0.data_ptr(), 3, 8, 4, whole.data_ptr(), ws.data_ptr(), nb, gu.stream_ptr())
    torch.cuda.synchronize()
    assert (rows[8:] == 7.0).all() and (whole[8:] == 7.0).all() and (slots.k[3] == 0x7F).all() and (slots.v[3] == 0x7F).all()


def test_offsets_that_break_the_rules_where_stretches_are_joined():
    """Sequences that share rows, more of them than the rows allow, and a workspace whose records nobody wrote: nothing outside."""
    slots = Slots(6, 1, 4096, 64)
    whole = torch.full((36, 4 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    rows = torch.ones((36, 6 * 64), dtype=torch.bfloat16, device="cuda")
    rs, p0 = i32([0, 32, 0, 32, 0, 32, 0]), i32([4000, -(1 << 31), 3000, (1 << 31) - 1, 4095, 0])
    nb = sd2.kv8_attention_workspace_size(slots.c, 4, 6, 32)
    for fill in (0xFF, 0x00, 0x01):
        ws = torch.full((nb + 4096,), fill, dtype=torch.uint8, device="cuda")
        sd2.kv8_attention(slots.c, rows.data_ptr(), 6 * 64, 4, rs.data_ptr(), p0.data_ptr(), 6, 32, 32, whole.data_ptr(), ws.data_ptr(), nb, gu.stream_ptr())
        torch.cuda.synchronize()
        assert (whole[32:] == 7.0).all() and (ws[nb:] == fill).all()


def test_the_path_of_a_layer():
    """q|k|v linear, append, prompt attention, output linear; then drafts against the cache: as a serving program runs them, against the
    oracle link by link (every link takes the library's own values of the link before)."""
    hidden, n_heads, n_kv, dim = 512, 4, 2, 128
    width = (n_heads + 2 * n_kv) * dim
    wqkv, wo = wl.gen_weight(77, 0, "q", width, hidden, 50), wl.gen_weight(77, 0, "o", hidden, n_heads * dim, 50)
    mats = [gu.SparseMat(w) for w in (wqkv, wo)]
    dense = [bits_to_f64(w) for w in (wqkv, wo)]
    lens = [70, 33, 1]
    slots = Slots(3, n_kv, 128, dim)

    def linear(mat, x, y):
        for t in range(0, x.shape[0], 64):
            n = min(64, x.shape[0] - t)
            nb = sd2.linear_workspace_size(mat.m, n)
            ws = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
            sd2.sparse_linear(mat.m, x[t:].data_ptr(), n, y[t:].data_ptr(), ws.data_ptr(), nb, gu.stream_ptr())
        torch.cuda.synchronize()
        return y

    done = [0, 0, 0]
    for seed, new in ((1, lens), (2, [5, 5, 5]), (3, [1, 0, 2])):
        n = sum(new)
        x = gu.dev(wl.gen_x(seed, 0, "q", n, hidden))
        x = x.view(torch.bfloat16)
        y = linear(mats[0], x, torch.empty((n, width), device="cuda"))
        ref = f64(x) @ dense[0].T
        assert np.linalg.norm(y.cpu().numpy() - ref) <= 1e-3 * np.linalg.norm(ref)
        rows = append(slots, y, n_heads, new, done)
        r = f64(rows).reshape(n, -1, dim)
        if seed == 1:
            out = torch.empty((n, n_heads * dim), dtype=torch.bfloat16, device="cuda")
            rs, at = i32(starts(new)), rows.data_ptr()
            sd2.prompt_attention(at, at + 2 * n_heads * dim, at + 2 * (n_heads + n_kv) * dim, width, width, rs.data_ptr(), 3, n, n_heads, n_kv, dim,
                                 out.data_ptr(), gu.stream_ptr())
            torch.cuda.synchronize()
            want, mass, dot = kv8.prompt_attention(r[:, :n_heads], r[:, n_heads:n_heads + n_kv], r[:, n_heads + n_kv:], starts(new))
            assert (np.abs(f64(out).reshape(want.shape) - want) <= bound(want, mass, dot, dim)).all()
        else:
            out = attend(slots, rows, n_heads, new, done, max_new=5)
            k, v, ks, vs = slots.host()
            check_attention(out, rows, [kv8.values(k[b], ks[b]) for b in range(3)], [kv8.values(v[b], vs[b]) for b in range(3)], n_heads, new, done, dim)
        o = linear(mats[1], out, torch.empty((n, hidden), device="cuda"))
        ref = f64(out) @ dense[1].T
        assert np.linalg.norm(o.cpu().numpy() - ref) <= 1e-3 * np.linalg.norm(ref)
        done = [d + m for d, m in zip(done, new)]


def test_more_rows_to_join_than_a_grid_dimension_has_threads():
    """16384 sequences of up to 64 rows of 64 heads: 2^26 of them may have been cut, four a workgroup of 256 threads.  Three sequences have
    rows, the first, the last and one in between."""
    n_seq, n_heads, dim, max_pos, n_rows = 16384, 64, 16, 160, 1024
    some = {0: (64, 90), 9000: (5, 150), n_seq - 1: (59, 96)}  # rows, position of the first
    slots = Slots(n_seq, 1, max_pos, dim)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(81)
    lens, pos0 = np.zeros(n_seq, dtype=np.int64), np.zeros(n_seq, dtype=np.int64)
    for b, (n, p) in some.items():
        lens[b], pos0[b] = n, p
        for c in (slots.k, slots.v):
            c[b] = (torch.randn(c[b].shape, generator=gen, device="cuda") * 95).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        slots.ks[b], slots.vs[b] = 2.0 ** -7, 2.0 ** -8
    q = torch.randn(n_rows, n_heads * dim, generator=gen, device="cuda").to(torch.bfloat16)
    rs, p0 = i32(np.concatenate([[0], np.cumsum(lens)]).tolist()), i32(pos0.tolist())
    out = torch.full((n_rows, n_heads * dim), 7.0, dtype=torch.bfloat16, device="cuda")
    nb = sd2.kv8_attention_workspace_size(slots.c, n_heads, n_seq, 64)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")  # 17 GiB
    sd2.kv8_attention(slots.c, q.data_ptr(), q.stride(0), n_heads, rs.data_ptr(), p0.data_ptr(), n_seq, n_rows, 64, out.data_ptr(), ws.data_ptr(), nb,
                      gu.stream_ptr())
    torch.cuda.synchronize()
    del ws
    torch.cuda.empty_cache()
    k, v = ([kv8.values(c[b].cpu().numpy(), s[b].cpu().numpy()) for b in some] for c, s in ((slots.k, slots.ks), (slots.v, slots.vs)))
    check_attention(out, q, k, v, n_heads, [n for n, _ in some.values()], [p for _, p in some.values()], dim)


def test_more_workgroups_than_a_grid_dimension_has_threads():
    """4096 sequences of a token with 4096 key/value heads: 2^24 workgroups of 256 threads.  Every token attends to itself alone, so that its
    result is its value."""
    n_seq, n_heads, dim = 4096, 4096, 16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(82)
    slots = Slots(n_seq, n_heads, 32, dim)  # 16 GiB
    for c in (slots.k, slots.v):
        c[:, :, 0] = torch.randint(-60, 60, (n_seq, n_heads, dim), generator=gen, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)
    slots.ks.fill_(2.0 ** -6)
    slots.vs.copy_(torch.exp2(torch.randint(-9, 9, slots.vs.shape, generator=gen, device="cuda").float()))
    q = torch.empty(n_seq, n_heads * dim, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    rs, p0 = i32(list(range(n_seq + 1))), i32([0] * n_seq)
    out = torch.full_like(q, 7.0)
    nb = sd2.kv8_attention_workspace_size(slots.c, n_heads, n_seq, 1)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")  # 66 GiB
    sd2.kv8_attention(slots.c, q.data_ptr(), q.stride(0), n_heads, rs.data_ptr(), p0.data_ptr(), n_seq, n_seq, 1, out.data_ptr(), ws.data_ptr(), nb,
                      gu.stream_ptr())
    torch.cuda.synchronize()
    del ws
    want = (slots.v[:, :, 0].view(torch.float8_e4m3fn).float() * slots.vs).to(torch.bfloat16).view(n_seq, -1)
    same = bool((out == want).all())
    del slots, want, q, out
    torch.cuda.empty_cache()
    assert same


@pytest.mark.parametrize("again", [3, 4])  # four wavefronts a row join in one launch, one in the other
def test_records_that_nobody_wrote_are_not_followed_past_the_workspace(again):
    """Sequences that share rows 0 .. 63, so that there are more units of work than the rows allow and the last ones are left out: those of
    the last 16 tokens of the last sequence.  The joining launch finds in their records what the workspace held before."""
    n_heads, dim, max_pos, max_new, n_rows = 4, 64, 2048, 64, 128
    offsets = [0, 64] * again + [64, 128]
    n_seq = len(offsets) - 1
    slots = Slots(n_seq, 1, max_pos, dim)
    for t, x in ((slots.k, 0), (slots.v, 0), (slots.ks, 1.0), (slots.vs, 1.0)):
        t.fill_(x)
    nb, guard = sd2.kv8_attention_workspace_size(slots.c, n_heads, n_seq, max_new), 4096
    records = n_seq * max_new * n_heads
    slot = 64 * (dim * 4 + 8)  # of a unit: 64 rows of sums, each with its maximum and sum of weights
    bound = (nb - 16 * records) // slot
    assert bound * slot == nb - 16 * records
    # 16 spans of 128 positions for each of 4 row tiles a sequence: one workgroup each, as far as the rows allow
    run, units = 16 * (n_rows * n_heads // 64 + n_seq), 16 * 4 * (again + 1)
    assert units - 16 <= bound and units - 64 <= run <= units - 16
    rest = 1 << 31
    cases = [((bound - 4, 4, 0), True), ((bound - 4, 5, 0), False), ((bound, 2, 0), False), ((0xFFFFFFFF, 2, 0), False), ((2, rest - 1, 0), False),
             ((bound - 4, rest | 3, bound - 1), True), ((bound - 4, rest | 3, bound), False), ((bound - 4, rest | 3, 0xFFFFFFFF), False),
             ((bound - 1, 1, 0), False), ((bound - 1, 0, 0), False), ((bound - 1, rest | 1, bound - 2), True), ((bound - 2, 2, 0xFFFFFFFF), True)]
    held = np.full(nb + 2 * guard, 0xAB, dtype=np.uint8)
    inside = held[guard:-guard]
    inside[:bound * 64 * dim * 4].view(np.float32)[:] = 3.0
    inside[bound * 64 * dim * 4:-16 * records].view(np.float32).reshape(-1, 2)[:] = [0.0, 1.0]
    table = inside[-16 * records:].view(np.uint32).reshape(n_seq, max_new, n_heads, 4)
    table[:] = 0
    for i, (record, _) in enumerate(cases):
        table[-1, 48 + i, :, :3] = record
    ws = torch.from_numpy(held).cuda()
    q = torch.ones((n_rows + 4, n_heads * dim), dtype=torch.bfloat16, device="cuda")
    out, rs, p0 = torch.full_like(q, 7.0), i32(offsets), i32([max_pos - 64] * n_seq)
    sd2.kv8_attention(slots.c, q.data_ptr(), q.stride(0), n_heads, rs.data_ptr(), p0.data_ptr(), n_seq, n_rows, max_new, out.data_ptr(),
                      ws.data_ptr() + guard, nb, gu.stream_ptr())
    torch.cuda.synchronize()
    assert (ws[:guard] == 0xAB).all() and (ws[-guard:] == 0xAB).all() and (out[n_rows:] == 7.0).all()
    for i, (record, followed) in enumerate(cases):  # sums of a workspace are held at 2^-8 of their size
        assert (out[64 + 48 + i] == (3.0 * 256 if followed else 7.0)).all(), record


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("max_pos,n", [(320, 300), (2048, 2000)])  # taken whole (heads of 256: cut); cut and joined
def test_values_as_large_as_sums_of_weighted_values_allow(dim, max_pos, n):
    """Values of one sign just below 2^127 / n under scores that rise by 7.5 powers of two, which the running maximum need not follow."""
    slots, x = Slots(1, 1, max_pos, dim), torch.zeros(n, 3 * dim, device="cuda")
    x[:, 2 * dim:] = torch.rand(n, dim, generator=torch.Generator().manual_seed(83)).cuda() * (2.0 ** 127 / n) * 0.9  # codes round up by 1/16
    append(slots, x, 1, [n], [0])
    # keys as they are to be, in place of rotated ones
    slots.k.zero_()
    slots.k[0, 0, :n, 0] = (torch.arange(n, device="cuda") * (7.5 / n * 32)).to(torch.float8_e4m3fn).view(torch.uint8)
    slots.ks.fill_(1.0)
    q = torch.zeros(3, dim, dtype=torch.bfloat16, device="cuda")
    q[:, 0] = np.log(2.0) * dim ** 0.5 / 32
    k, v, ks, vs = slots.host()
    k, v = [kv8.values(k[0], ks[0])], [kv8.values(v[0], vs[0])]
    check_attention(attend(slots, q, 1, [2], [n - 2], n_rows=2), q, k, v, 1, [2], [n - 2], dim)
