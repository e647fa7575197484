"""Causal attention over packed prompts on the GPU against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2504_08838_amd as sd2
from oracle import kv8

import gpu_util as gu
from test_gpu_kv8 import bound, f64, i32, starts

pytestmark = pytest.mark.gpu
HEADS = [(4, 2, 128), (3, 1, 64), (8, 8, 16), (6, 2, 80), (8, 1, 256), (7, 7, 144), (12, 2, 128), (2, 1, 48)]


def rows(seed, n, heads, dim, stride=None):
    """bf16 [n][heads * dim] inside rows of `stride` values, the rest of them NaN."""
    stride = heads * dim if stride is None else stride
    t = torch.full((n, stride), float("nan"), dtype=torch.bfloat16)
    t[:, :heads * dim] = torch.randn(n, heads * dim, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
    return t.cuda()


def run(q, k, v, lens, n_heads, n_kv, dim, n_rows=None, out=None):
    out = torch.full((q.shape[0], n_heads * dim), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    rs = i32(starts(lens))
    sd2.prompt_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), q.stride(0), k.stride(0), rs.data_ptr(), len(lens),
                         q.shape[0] if n_rows is None else n_rows, n_heads, n_kv, dim, out.data_ptr(), gu.stream_ptr())
    torch.cuda.synchronize()
    return out


def split(t, heads, dim):
    return f64(t[:, :heads * dim].contiguous()).reshape(-1, heads, dim)


def check(out, q, k, v, lens, n_heads, n_kv, dim):
    want, mass, dot = kv8.prompt_attention(split(q, n_heads, dim), split(k, n_kv, dim), split(v, n_kv, dim), starts(lens))
    got, n = f64(out).reshape(want.shape), sum(lens)
    assert (got[n:] == 7.0).all()
    got, want, mass, dot = got[:n], want[:n], mass[:n], dot[:n]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    infinite = np.isinf(want)
    assert np.array_equal(got[infinite], want[infinite])
    fine = np.isfinite(want)
    with np.errstate(invalid="ignore"):
        off, tol = np.abs(got - want), bound(want, mass, dot, dim)
    assert (off <= tol)[fine].all(), np.max((off / tol)[fine])


@pytest.mark.parametrize("n_heads,n_kv,dim", HEADS)
@pytest.mark.parametrize("lens", [[1], [2], [16, 1, 0, 31], [32, 33], [63, 64, 65], [127, 128, 129, 1], [0, 257, 0], [520]])
def test_lengths_and_heads(n_heads, n_kv, dim, lens):
    n = sum(lens)
    q, k, v = rows(1, n, n_heads, dim), rows(2, n, n_kv, dim), rows(3, n, n_kv, dim)
    check(run(q, k, v, lens, n_heads, n_kv, dim), q, k, v, lens, n_heads, n_kv, dim)


@pytest.mark.parametrize("n_heads,n_kv", [(1, 1), (64, 1), (10, 10), (30, 3)])
def test_few_and_many_heads_a_group(n_heads, n_kv):
    lens = [70, 3]
    q, k, v = rows(4, 73, n_heads, 64), rows(5, 73, n_kv, 64), rows(6, 73, n_kv, 64)
    check(run(q, k, v, lens, n_heads, n_kv, 64), q, k, v, lens, n_heads, n_kv, 64)


@pytest.mark.parametrize("dim", [64, 128, 80])
def test_strides_and_rows_behind_the_last_sequence(dim):
    """Rows inside longer ones; rows that belong to no sequence hold NaN and are neither read nor written."""
    lens, n = [40, 90], 135
    q, k, v = rows(7, n, 6, dim, 6 * dim + 8), rows(8, n, 2, dim, 4 * dim), rows(9, n, 2, dim, 4 * dim)
    for t in (q, k, v):
        t[130:] = float("nan")
    check(run(q, k, v, lens, 6, 2, dim), q, k, v, lens, 6, 2, dim)


def test_q_k_v_in_one_array():
    lens, h, g, dim = [100, 29], 4, 2, 128
    whole = rows(10, 129, h + 2 * g, dim)
    q, k, v = (whole[:, a * dim:] for a in (0, h, h + g))
    out = torch.full((129, h * dim), 7.0, dtype=torch.bfloat16, device="cuda")
    check(run(q, k, v, lens, h, g, dim, out=out), q[:, :h * dim], k[:, :g * dim], v[:, :g * dim], lens, h, g, dim)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", [37, 150])
def test_values_that_are_not_finite_reach_the_rows_that_attend_to_them(dim, value, where):
    lens, n_heads, n_kv = [20, 180], 4, 2
    q, k, v = rows(11, 200, n_heads, dim), rows(12, 200, n_kv, dim), rows(13, 200, n_kv, dim)
    v[20 + where, 5] = value
    v[20 + where, dim + dim - 1] = value
    out = run(q, k, v, lens, n_heads, n_kv, dim)
    check(out, q, k, v, lens, n_heads, n_kv, dim)
    assert (~torch.isfinite(out.float())).sum() == 4 * (180 - where)


def test_infinities_of_both_signs_and_odd_keys():
    lens, n_heads, n_kv, dim = [150], 2, 1, 128
    q, k, v = rows(14, 150, n_heads, dim), rows(15, 150, n_kv, dim), rows(16, 150, n_kv, dim)
    v[10, 3], v[90, 3], v[70, 4] = float("inf"), float("-inf"), float("inf")
    k[120, 9] = float("nan")
    out = run(q, k, v, lens, n_heads, n_kv, dim)
    check(out, q, k, v, lens, n_heads, n_kv, dim)
    o = out.float().view(150, 2, dim)
    assert torch.isinf(o[10:90, :, 3]).all() and torch.isnan(o[90:, :, 3]).all() and torch.isnan(o[120:]).all()


def test_an_infinite_key():
    """Scores of plus and minus infinity: a row with a positive one is NaN, a negative one has no weight (oracle and kernel alike)."""
    lens, n_heads, n_kv, dim = [140], 2, 1, 64
    q, k, v = rows(17, 140, n_heads, dim), rows(18, 140, n_kv, dim), rows(19, 140, n_kv, dim)
    k[66, 2] = float("inf")
    check(run(q, k, v, lens, n_heads, n_kv, dim), q, k, v, lens, n_heads, n_kv, dim)


@pytest.mark.parametrize("dim", [64, 128])
def test_large_and_tiny_magnitudes(dim):
    lens = [200, 75]
    for scale in (300.0, 1e-30):
        q, k, v = rows(20, 275, 4, dim) * scale, rows(21, 275, 2, dim), rows(22, 275, 2, dim) * (1e30 if scale > 1 else 1e-30)
        check(run(q, k, v, lens, 4, 2, dim), q, k, v, lens, 4, 2, dim)


def test_growing_scores():
    """Keys that grow along the prompt: the running maximum moves in every tile."""
    n, dim = 700, 128
    q, k, v = rows(23, n, 2, dim), rows(24, n, 1, dim), rows(25, n, 1, dim)
    k = (k.float() * torch.linspace(0.1, 30.0, n, device="cuda")[:, None]).to(torch.bfloat16)
    q = (q.float() * 0.2 + k.float().roll(-1, 0).repeat(1, 2) * 0.1).to(torch.bfloat16)
    check(run(q, k, v, [n], 2, 1, dim), q, k, v, [n], 2, 1, dim)


def test_a_long_prompt_row_by_row():
    """Rows of a prompt of 6000 tokens picked by hand, among them the first, the last and those around tiles."""
    n, n_heads, n_kv, dim = 6000, 3, 1, 128
    q, k, v = rows(26, n, n_heads, dim), rows(27, n, n_kv, dim), rows(28, n, n_kv, dim)
    out = f64(run(q, k, v, [n], n_heads, n_kv, dim)).reshape(n, n_heads, dim)
    pick = [0, 1, 41, 42, 43, 63, 64, 127, 128, 2047, 2048, 4095, 4096, 5503, 5504, 5998, 5999]
    want, mass, dot = kv8.attention(split(q, n_heads, dim)[pick], split(k, n_kv, dim).transpose(1, 0, 2), split(v, n_kv, dim).transpose(1, 0, 2), pick)
    assert (np.abs(out[pick] - want) <= bound(want, mass, dot, dim)).all()


def test_many_sequences():
    lens = np.random.default_rng(29).integers(0, 7, 200).tolist()
    n = sum(lens)
    q, k, v = rows(30, n, 2, 64), rows(31, n, 1, 64), rows(32, n, 1, 64)
    check(run(q, k, v, lens, 2, 1, 64), q, k, v, lens, 2, 1, 64)


def test_same_bits_on_every_call_and_inside_a_batch():
    """A prompt's result does not depend on what it is packed with."""
    q, k, v = rows(33, 600, 6, 128), rows(34, 600, 2, 128), rows(35, 600, 2, 128)
    alone = run(q[200:], k[200:], v[200:], [400], 6, 2, 128)
    batch = [run(q, k, v, [200, 400], 6, 2, 128) for _ in range(3)]
    for b in batch:
        assert torch.equal(b[200:].view(torch.int16), alone.view(torch.int16))


def test_captured_call_serves_new_lengths():
    n, h, g, dim = 300, 6, 2, 128
    q, k, v = rows(36, n, h, dim), rows(37, n, g, dim), rows(38, n, g, dim)
    rs, out = i32([0, 0, 0, 0]), torch.full((n, h * dim), 7.0, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()

    def call():
        sd2.prompt_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), q.stride(0), k.stride(0), rs.data_ptr(), 3, n, h, g, dim, out.data_ptr(),
                             side.cuda_stream)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for seed, lens in ((40, [300, 0, 0]), (41, [1, 64, 235]), (42, [100, 7, 90])):
        rs.copy_(i32(starts(lens)))
        q.copy_(rows(seed, n, h, dim))
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(out, q, k, v, lens, h, g, dim)


def test_offsets_that_break_the_rules_stay_inside_the_buffers():
    q, k, v = rows(43, 60, 2, 64), rows(44, 60, 1, 64), rows(45, 60, 1, 64)
    out = torch.full((60, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    rs = i32([30, -5, 1 << 30, 10, (1 << 31) - 1, -(1 << 31)])
    sd2.prompt_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), 128, 64, rs.data_ptr(), 5, 50, 2, 1, 64, out.data_ptr(), gu.stream_ptr())
    torch.cuda.synchronize()
    assert (out[50:] == 7.0).all()


# Which kernel a call gets goes by its rows times query heads of a group: what is above gets the one for few.  SOME (4500 and 6000 of them
# for each key/value head) gets the one with two teams, MANY (12000 and 16000) the one of the longest calls; prompts of all lengths in both.
SOME = [300, 1, 0, 129, 640, 64, 33, 2, 331]
MANY = [40 + 7 * i for i in range(24)] + [0, 1, 65, 700, 128, 250]
WIDE = [(24, 8, 128), (32, 8, 64), (24, 8, 80), (32, 8, 48)]


@pytest.mark.parametrize("n_heads,n_kv,dim", WIDE)
@pytest.mark.parametrize("lens", [SOME, MANY], ids=["some", "many"])
def test_more_rows_than_the_chip_takes_at_once(n_heads, n_kv, dim, lens):
    n = sum(lens)
    q, k, v = rows(50, n, n_heads, dim), rows(51, n, n_kv, dim), rows(52, n, n_kv, dim)
    check(run(q, k, v, lens, n_heads, n_kv, dim), q, k, v, lens, n_heads, n_kv, dim)


@pytest.mark.parametrize("n_heads,n_kv,dim", WIDE[:3])
@pytest.mark.parametrize("lens", [SOME, MANY], ids=["some", "many"])
def test_more_rows_with_values_that_are_not_finite(n_heads, n_kv, dim, lens):
    """One prompt's values hold NaN and infinities; the others' results stay as they are, and its own rows get what they attend to."""
    n, b = sum(lens), lens.index(640 if 640 in lens else 700)
    at = starts(lens)[b]
    q, k, v = rows(53, n, n_heads, dim), rows(54, n, n_kv, dim), rows(55, n, n_kv, dim)
    clean = run(q, k, v, lens, n_heads, n_kv, dim)
    v[at + 70, 3], v[at + 200, dim], v[at + 333, dim - 1] = float("nan"), float("inf"), float("-inf")
    out = run(q, k, v, lens, n_heads, n_kv, dim)
    part, m = slice(at, at + lens[b]), lens[b]
    check(out[part], q[part], k[part], v[part], [m], n_heads, n_kv, dim)
    outside = torch.ones(n, dtype=torch.bool)
    outside[part] = False
    assert torch.equal(out[outside.cuda()].view(torch.int16), clean[outside.cuda()].view(torch.int16))


@pytest.mark.parametrize("lens", [SOME, MANY], ids=["some", "many"])
def test_more_rows_inside_longer_ones_and_rows_behind_the_last_sequence(lens):
    n, dim = sum(lens) + 5, 128
    q, k, v = rows(56, n, 24, dim, 24 * dim + 64), rows(57, n, 8, dim, 8 * dim + 8), rows(58, n, 8, dim, 8 * dim + 8)
    for t in (q, k, v):
        t[sum(lens):] = float("nan")
    check(run(q, k, v, lens, 24, 8, dim), q, k, v, lens, 24, 8, dim)


def test_a_long_prompt_of_the_largest_kernel_row_by_row():
    n, n_heads, n_kv, dim = 5000, 24, 8, 128
    q, k, v = rows(59, n, n_heads, dim), rows(60, n, n_kv, dim), rows(61, n, n_kv, dim)
    out = f64(run(q, k, v, [n], n_heads, n_kv, dim)).reshape(n, n_heads, dim)
    pick = [0, 1, 41, 42, 43, 63, 64, 127, 128, 2047, 2048, 4095, 4096, 4998, 4999]
    want, mass, dot = kv8.attention(split(q, n_heads, dim)[pick], split(k, n_kv, dim).transpose(1, 0, 2), split(v, n_kv, dim).transpose(1, 0, 2), pick)
    assert (np.abs(out[pick] - want) <= bound(want, mass, dot, dim)).all()


@pytest.mark.parametrize("n,repeats", [(500, 20), (1500, 20), (4000, 10)])
def test_same_bits_every_time(n, repeats):
    """Each kernel, over and over on other values in between: what a buffer of LDS holds from before never shows."""
    q, k, v = rows(62, n, 24, 128), rows(63, n, 8, 128), rows(64, n, 8, 128)
    other = [rows(65 + i, n, h, 128) * 30 for i, h in enumerate((24, 8, 8))]
    first = run(q, k, v, [n], 24, 8, 128).view(torch.int16)
    for _ in range(repeats):
        run(*other, [n], 24, 8, 128)
        assert torch.equal(run(q, k, v, [n], 24, 8, 128).view(torch.int16), first)


@pytest.mark.parametrize("n_heads,n_kv", [(4096, 4096), (4096, 2048)])
def test_more_workgroups_than_a_grid_dimension_has_threads(n_heads, n_kv):
    """Sequences of a token: 4096 with 4096 key/value heads, 8192 with 2048, 2^24 workgroups of 256 threads.  Every token attends to itself
    alone, so that its result is its value."""
    n_seq, dim = (1 << 24) // n_kv, 16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(70)
    q, k, v = (torch.empty(n_seq, h * dim, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for h in (n_heads, n_kv, n_kv))
    rs, out = i32(list(range(n_seq + 1))), torch.full_like(q, 7.0)
    sd2.prompt_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), q.stride(0), k.stride(0), rs.data_ptr(), n_seq, n_seq, n_heads, n_kv, dim,
                         out.data_ptr(), gu.stream_ptr())
    torch.cuda.synchronize()
    same = bool((out.view(n_seq, n_kv, n_heads // n_kv, dim) == v.view(n_seq, n_kv, 1, dim)).all())
    del q, k, v, out
    torch.cuda.empty_cache()
    assert same


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("n,n_heads,n_kv", [(300, 4, 2), (1024, 48, 16)])  # teams of a wavefront; of four
def test_values_as_large_as_sums_of_weighted_values_allow(dim, n, n_heads, n_kv):
    """Values of one sign just below 2^119 / n under scores that rise by 7.5 powers of two, which the running maximum need not follow."""
    q, k, v = torch.zeros(n, n_heads * dim), torch.zeros(n, n_kv * dim), rows(71, n, n_kv, dim)
    q[:, ::dim], k[:, ::dim] = 1.0, (torch.arange(n) * (7.5 / n * np.log(2.0) * dim ** 0.5))[:, None]
    q, k = (t.to(torch.bfloat16).cuda() for t in (q, k))
    v = (v.float().sigmoid() * (2.0 ** 119 / n)).to(torch.bfloat16)
    check(run(q, k, v, [n], n_heads, n_kv, dim), q, k, v, [n], n_heads, n_kv, dim)
