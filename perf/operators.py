"""Attention of several requests at once: prompts as a whole, and new tokens against a key/value cache held in 8 bits.

Three operators that a serving program calls one after the other in every layer, between the q|k|v linear and the output
linear: ``sd2_kv8_append`` (rotary embedding, rounding to bf16, keys and values into the cache), ``sd2_prompt_attention``
(prompts of different lengths, packed) and ``sd2_kv8_attention`` (single tokens, drafts and chunks against the cache).

The cache holds e4m3 codes [slots][n_kv][max_pos][head_dim] and a power-of-two scale per 32 positions and head,
[slots][n_kv][max_pos / 32].  Sequence b of a call uses slot b; its rows are row_start[b] .. row_start[b + 1] - 1, its
first row sits at position pos0[b].  Head layouts are those of the drafters in ``sd2_workload.CONFIGS`` or generic.
``own`` false: the same in elementary torch operations.
"""

import math

import torch

own = False

BLOCK = 32  # positions that share a scale
E4M3_MAX = 448.0
MIN_EXPONENT = -100
ROPE_THETA = 500000.0

HEADS_3B = {"n_heads": 24, "n_kv": 8, "head_dim": 128}
HEADS_1_5B = {"n_heads": 12, "n_kv": 2, "head_dim": 128}
HEADS_64 = {"n_heads": 32, "n_kv": 8, "head_dim": 64}


def listed():
    return [
        # the smallest call of a decode step: one token of one request enters the cache, latency and little else
        {"name": "append-1", "kind": "append", **HEADS_3B, "rows": "1", "pos0": "428", "max_pos": 1024},
        # drafts of a batch of requests enter blocks that are open already, at ragged positions
        {"name": "append-drafts", "kind": "append", **HEADS_1_5B, "rows": "5,1,3,8,5,5,2,6,1,4,5,7,5,3,1,5,6,5,2,5,8,1,5,4,5,3,7,5,5,2,1,6",
         "pos0": "31,64,100,7,2000,511,830,1500,45,96,333,1027,680,12,700,1299,3,402,64,950,1777,18,259,1153,90,601,1408,77,1650,222,39,1001",
         "max_pos": 2048},
        # prompts of a few requests fill their slots: the most bytes
        {"name": "append-prompts", "kind": "append", **HEADS_3B, "rows": "2900,17,640,1333,4000,255,1,411", "pos0": "0,0,0,0,0,0,0,0",
         "max_pos": 4096},
        # a question of a few words
        {"name": "prompt-37", "kind": "prompt", **HEADS_1_5B, "rows": "37"},
        # the usual prompt of the decode benchmark
        {"name": "prompt-300", "kind": "prompt", **HEADS_3B, "rows": "300"},
        # a batch of prompts of different lengths, packed
        {"name": "prompts-packed", "kind": "prompt", **HEADS_3B, "rows": "120,1500,33,64,910,410,1,257,700,95,1204,18,333,512"},
        # a long document
        {"name": "prompt-8192", "kind": "prompt", **HEADS_3B, "rows": "8192"},
        # few long prompts of a drafter with small heads, one of a single token among them
        {"name": "prompts-64", "kind": "prompt", **HEADS_64, "rows": "3001,1,2500,777"},
        # one token against the cache in the middle of a short answer: latency
        {"name": "cached-1", "kind": "cached", **HEADS_3B, "rows": "1", "pos0": "428", "max_pos": 1024},
        # a draft of five tokens against one long history: work has to be found along the positions
        {"name": "cached-long", "kind": "cached", **HEADS_1_5B, "rows": "5", "pos0": "30011", "max_pos": 32768},
        # serving: drafts of 64 requests with histories of all lengths, some requests idle
        {"name": "cached-batch", "kind": "cached", **HEADS_3B,
         "rows": "5,5,1,5,0,3,5,5,8,5,5,2,5,5,5,0,5,4,5,5,1,5,5,5,6,5,5,5,5,0,5,5,5,7,5,5,5,3,5,5,5,5,1,5,5,5,5,5,2,5,5,5,0,5,5,4,5,5,5,5,5,5,1,5",
         "pos0": "5000,812,120,9000,0,431,15500,2222,64,7001,333,1900,12007,48,5555,0,600,3100,10400,27,8200,950,1450,4096,77,13333,2700,510,6100,"
                 "0,1234,180,3900,255,7777,1601,40,11111,2048,690,5200,14,4410,333,8888,1020,150,6400,2951,505,12500,1777,0,96,3500,740,9600,"
                 "31,2500,415,16000,1111,5801,210", "max_pos": 16384},
        # chunks of prompts against what is in the cache already: the most rows of a request
        {"name": "cached-chunks", "kind": "cached", **HEADS_64, "rows": "64,64,51,64", "pos0": "4000,448,1777,3008", "max_pos": 8192},
    ]


def _ints(text):
    return [int(v) for v in text.split(",")]


# ------------------------------------------------------------------ drawn cases


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_heads(rng):
    n_kv = rng.choice([1, 2, 3, 4, 8, 8])
    rep = rng.choice([1, 2, 3, 3, 4, 6, 7, 8])
    return {"n_heads": min(n_kv * rep, 32) // n_kv * n_kv, "n_kv": n_kv, "head_dim": rng.choice([64, 64, 80, 96, 128, 128, 128, 128, 256])}


def draw(rng):
    case = {"kind": rng.choice(["append", "prompt", "prompt", "cached", "cached"]), **_draw_heads(rng)}
    width = case["n_heads"] * case["head_dim"]
    if case["kind"] == "prompt":
        n_seq = _log_int(rng, 1, 32)
        longest = _log_int(rng, 1, 8192)
        # the plain form holds n_seq * n_heads * longest^2 scores; the work stays below the longest listed prompt's
        while n_seq * case["n_heads"] * longest ** 2 > 1 << 31 or n_seq * width * longest ** 2 > 24 * 128 * 8192 ** 2:
            n_seq, longest = max(1, n_seq // 2), max(1, longest * 3 // 4)
        rows = [longest] + [_log_int(rng, 1, longest) for _ in range(n_seq - 1)]
        rng.shuffle(rows)
        return {**case, "rows": ",".join(map(str, rows))}
    n_seq = _log_int(rng, 1, 64)
    if case["kind"] == "append":
        prompts = rng.random() < 0.5
        most = _log_int(rng, 1, 4096) if prompts else rng.randint(1, 8)
        rows = [_log_int(rng, 1, most) for _ in range(n_seq)]
        while sum(rows) * (width + 2 * case["n_kv"] * case["head_dim"]) > 9000 * 5120:
            rows = rows[:max(1, len(rows) // 2)]
        n_seq = len(rows)
        pos0 = [rng.choice([0, _log_int(rng, 1, 2000)]) if prompts else _log_int(rng, 1, 4000) for _ in range(n_seq)]
        return {**case, "rows": ",".join(map(str, rows)), "pos0": ",".join(map(str, pos0)),
                "max_pos": BLOCK * (max(p + r for p, r in zip(pos0, rows)) // BLOCK + 1 + rng.randint(0, 30))}
    most = rng.choice([1, 1, 5, 8, 64])
    farthest = _log_int(rng, 16, 32000)
    # sequences times positions times bytes of a position: at most the listed batch's cache
    while n_seq * farthest * case["n_kv"] * case["head_dim"] > 64 * 8192 * 1024 or n_seq * farthest * most * width > 64 * 4096 * 5 * 24 * 128:
        n_seq, farthest = max(1, n_seq // 2), max(16, farthest * 3 // 4)
    rows = [rng.choice([most, most, most, rng.randint(0, most)]) for _ in range(n_seq)]
    rows[rng.randrange(n_seq)] = most
    pos0 = [farthest] + [_log_int(rng, 1, farthest) for _ in range(n_seq - 1)]
    rng.shuffle(pos0)
    return {**case, "rows": ",".join(map(str, rows)), "pos0": ",".join(map(str, pos0)),
            "max_pos": BLOCK * ((farthest + most) // BLOCK + 1 + rng.randint(0, 30))}


# ------------------------------------------------------------------ what a program has in hand before the call


class _State:
    pass


def _normal(gen, *shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=gen)


def _rows(gen, n, case):
    """q|k|v rows as a decoder's linear leaves them: some dimensions of a head are larger than others."""
    heads, d = case["n_heads"] + 2 * case["n_kv"], case["head_dim"]
    return (_normal(gen, n, heads, d) * torch.exp(0.4 * _normal(gen, 1, heads, d))).reshape(n, heads * d)


def _codes(gen, *shape):
    """Codes as a block's scale leaves them: the largest of a block near the end of the range."""
    out = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    for part in out.view(shape[0], -1):
        part.copy_((_normal(gen, part.numel()) * 95.0).clamp_(-E4M3_MAX, E4M3_MAX))
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = _State()
    s.case, s.lens = case, _ints(case["rows"])
    s.n_seq, s.n_rows, s.max_rows = len(s.lens), sum(s.lens), max(s.lens)
    h, g, d = case["n_heads"], case["n_kv"], case["head_dim"]
    starts = [sum(s.lens[:i]) for i in range(s.n_seq + 1)]
    s.row_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s.qkv = _rows(gen, s.n_rows, case)  # fp32, [rows][(h + 2 g) d]
    if case["kind"] != "append":
        s.qkv = s.qkv.to(torch.bfloat16)
        s.out = torch.zeros((s.n_rows, h * d), dtype=torch.bfloat16, device="cuda")
    if case["kind"] != "prompt":
        s.pos0_list = _ints(case["pos0"])
        s.pos0 = torch.tensor(s.pos0_list, dtype=torch.int32, device="cuda")
        s.farthest = max(p + n for p, n in zip(s.pos0_list, s.lens))
        cache, blocks = (s.n_seq, g, case["max_pos"], d), (s.n_seq, g, case["max_pos"] // BLOCK)
        s.k, s.v = _codes(gen, *cache), _codes(gen, *cache)
        # values of about 0.4 to 1.5
        s.k_scale = torch.exp2(torch.randint(-8, -5, blocks, generator=gen, device="cuda").float())
        s.v_scale = torch.exp2(torch.randint(-8, -5, blocks, generator=gen, device="cuda").float())
    if case["kind"] == "append":
        s.rows_bf16 = torch.zeros((s.n_rows, (h + 2 * g) * d), dtype=torch.bfloat16, device="cuda")
    if own:
        import paper_2504_08838_amd as sd2

        s.sd2 = sd2
        if case["kind"] != "prompt":
            s.cache = sd2.kv8_cache_init(s.k.data_ptr(), s.v.data_ptr(), s.k_scale.data_ptr(), s.v_scale.data_ptr(), s.n_seq, g,
                                         case["max_pos"], d)
        if case["kind"] == "cached":
            s.ws_bytes = sd2.kv8_attention_workspace_size(s.cache, h, s.n_seq, s.max_rows)
            s.ws = torch.empty(max(s.ws_bytes, 16), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms


def _softmax_of_scores(scores, keep):
    scores = torch.where(keep, scores, torch.full_like(scores, -math.inf))
    e = torch.exp(scores - scores.amax(dim=-1, keepdim=True))
    return e / e.sum(dim=-1, keepdim=True)


def _seq_and_index(s):
    """Per row: its sequence, and its place in it."""
    row = torch.arange(s.n_rows, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s.row_start[1:], row, right=True)
    return seq, (row - s.row_start[seq]).long()


def _padded(x, seq, index, s):
    """[rows][heads][d] -> [sequences][heads][longest][d], zeros behind a sequence's end."""
    out = torch.zeros((s.n_seq, s.max_rows) + x.shape[1:], dtype=torch.float32, device="cuda")
    out[seq, index] = x.float()
    return out.transpose(1, 2)


def _plain_prompt(s):
    h, g, d = (s.case[n] for n in ("n_heads", "n_kv", "head_dim"))
    seq, index = _seq_and_index(s)
    heads = s.qkv.view(s.n_rows, h + 2 * g, d)
    q = _padded(heads[:, :h], seq, index, s).reshape(s.n_seq, g, h // g * s.max_rows, d)  # a group's heads one after the other
    k, v = (_padded(x, seq, index, s) for x in (heads[:, h:h + g], heads[:, h + g:]))
    at = torch.arange(s.max_rows, device="cuda")
    keep = (at[None, :] <= at[:, None]).repeat(h // g, 1)
    p = _softmax_of_scores(torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d)), keep)
    o = torch.matmul(p, v.contiguous()).view(s.n_seq, h, s.max_rows, d).transpose(1, 2)
    return o[seq, index].reshape(s.n_rows, h * d).to(torch.bfloat16)


def _plain_cached(s):
    h, g, d = (s.case[n] for n in ("n_heads", "n_kv", "head_dim"))
    seq, index = _seq_and_index(s)
    n_blocks = -(-s.farthest // BLOCK)
    span = n_blocks * BLOCK

    def values(codes, scale):
        x = codes[:, :, :span].to(torch.float32).view(s.n_seq, g, n_blocks, BLOCK, d)
        return (x * scale[:, :, :n_blocks, None, None]).view(s.n_seq, g, span, d)

    q = _padded(s.qkv.view(s.n_rows, h + 2 * g, d)[:, :h], seq, index, s).reshape(s.n_seq, g, h // g * s.max_rows, d)
    reach = (s.pos0[:, None] + torch.arange(s.max_rows, device="cuda")[None, :]).repeat(1, h // g)  # per sequence and query row
    keep = (torch.arange(span, device="cuda") <= reach[:, :, None])[:, None]
    scores = torch.matmul(q, values(s.k, s.k_scale).transpose(2, 3).contiguous())
    p = _softmax_of_scores(scores * (1.0 / math.sqrt(d)), keep)
    o = torch.matmul(p, values(s.v, s.v_scale)).view(s.n_seq, h, s.max_rows, d).transpose(1, 2)
    return o[seq, index].reshape(s.n_rows, h * d).to(torch.bfloat16)


def _plain_store(x, codes, scale, seq, pos, s):
    """bf16 values x [rows][g][d] into codes and scale."""
    g, d = s.case["n_kv"], s.case["head_dim"]
    block = pos // BLOCK
    flat = torch.zeros((s.n_seq * scale.shape[2], g), dtype=torch.float32, device="cuda")
    at = seq * scale.shape[2] + block
    flat.scatter_reduce_(0, at[:, None].expand(-1, g), x.float().abs().amax(dim=2), "amax")
    mantissa, exponent = torch.frexp(flat.view(s.n_seq, -1, g).transpose(1, 2))  # largest = mantissa 2^exponent, 448 = 0.875 2^9
    exponent = torch.where(mantissa > 0, exponent - 9 + (mantissa > 0.875).int(), torch.full_like(exponent, MIN_EXPONENT))
    needed = torch.exp2(exponent.clamp_min(MIN_EXPONENT).float())
    rows = torch.zeros((s.n_seq, scale.shape[2]), dtype=torch.bool, device="cuda")
    rows[seq, block] = True
    first = torch.arange(scale.shape[2], device="cuda")[None, :] * BLOCK
    opened = (first < s.pos0[:, None])[:, None]  # blocks that held positions before this call
    new = torch.where(rows[:, None], torch.where(opened, torch.maximum(scale, needed), needed), scale)
    # the only block of a sequence that can hold older positions beside new ones
    every, b0 = torch.arange(s.n_seq, device="cuda"), (s.pos0 // BLOCK).long()
    older = codes.view(s.n_seq, g, -1, BLOCK, d)[every, :, b0].float()
    ratio = (scale[every, :, b0] / new[every, :, b0])[:, :, None, None]
    is_old = (b0[:, None] * BLOCK + torch.arange(BLOCK, device="cuda") < s.pos0[:, None])[:, None, :, None]
    codes.view(s.n_seq, g, -1, BLOCK, d)[every, :, b0] = torch.where(is_old, older * ratio, older).to(codes.dtype)
    codes[seq, :, pos] = (x.float() / new[seq, :, block][:, :, None]).to(codes.dtype)
    scale.copy_(new)


def _plain_append(s):
    h, g, d = (s.case[n] for n in ("n_heads", "n_kv", "head_dim"))
    seq, index = _seq_and_index(s)
    pos = s.pos0[seq].long() + index
    angle = pos.double()[:, None] * torch.pow(torch.tensor(ROPE_THETA, dtype=torch.float64, device="cuda"),
                                              -2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    c, sn = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x = s.qkv.view(s.n_rows, h + 2 * g, d)
    lo, hi = x[:, :h + g, :d // 2], x[:, :h + g, d // 2:]
    rows = torch.cat([torch.cat([lo * c - hi * sn, hi * c + lo * sn], dim=2), x[:, h + g:]], dim=1).to(torch.bfloat16)
    _plain_store(rows[:, h:h + g], s.k, s.k_scale, seq, pos, s)
    _plain_store(rows[:, h + g:], s.v, s.v_scale, seq, pos, s)
    return rows.view(s.n_rows, -1)


# ------------------------------------------------------------------ one pass


def run(s):
    h, g, d = (s.case[n] for n in ("n_heads", "n_kv", "head_dim"))
    if own:
        stream = torch.cuda.current_stream().cuda_stream
        if s.case["kind"] == "append":
            s.sd2.kv8_append(s.cache, s.qkv.data_ptr(), h, s.row_start.data_ptr(), s.pos0.data_ptr(), s.n_seq, s.n_rows, ROPE_THETA,
                             s.rows_bf16.data_ptr(), stream)
            rows = s.rows_bf16
        elif s.case["kind"] == "prompt":
            at, width = s.qkv.data_ptr(), (h + 2 * g) * d
            s.sd2.prompt_attention(at, at + 2 * h * d, at + 2 * (h + g) * d, width, width, s.row_start.data_ptr(), s.n_seq, s.n_rows, h, g, d,
                                   s.out.data_ptr(), stream)
            return s.out
        else:
            s.sd2.kv8_attention(s.cache, s.qkv.data_ptr(), (h + 2 * g) * d, h, s.row_start.data_ptr(), s.pos0.data_ptr(), s.n_seq, s.n_rows,
                                s.max_rows, s.out.data_ptr(), s.ws.data_ptr(), s.ws_bytes, stream)
            return s.out
    elif s.case["kind"] == "append":
        rows = _plain_append(s)
    else:
        return _plain_prompt(s) if s.case["kind"] == "prompt" else _plain_cached(s)
    return {"rows": rows, "k": s.k, "v": s.v, "k_scale": s.k_scale, "v_scale": s.v_scale}


def work(case):
    h, g, d = (case[n] for n in ("n_heads", "n_kv", "head_dim"))
    lens = _ints(case["rows"])
    rows = sum(lens)
    if case["kind"] == "append":
        return {"bytes": rows * d * ((h + 2 * g) * 6 + 2 * g), "flops": rows * d * (h + g) * 3}
    if case["kind"] == "prompt":
        return {"bytes": rows * d * 2 * (2 * h + 2 * g), "flops": 4 * d * h * sum(n * (n + 1) // 2 for n in lens)}
    pos0 = _ints(case["pos0"])
    # an idle request's history is not read
    positions = sum(p + n for p, n in zip(pos0, lens) if n)
    return {"bytes": positions * g * 2 * (d + 4 / BLOCK) + rows * h * d * 4,
            "flops": 4 * d * h * sum(n * p + n * (n + 1) // 2 for p, n in zip(pos0, lens))}


# ------------------------------------------------------------------ 64 bits


def _attend(q, k, v, reach):
    """q [n][d], k and v [p][d] in 64 bits; row i attends to positions 0 .. reach[i]."""
    out = torch.empty_like(q)
    for i in range(0, len(q), 2048):
        at = reach[i:i + 2048, None]
        p = int(at.max()) + 1
        z = (q[i:i + 2048] @ k[:p].T) / math.sqrt(q.shape[1])
        z = z.masked_fill(torch.arange(p, device=q.device)[None, :] > at, -math.inf)
        out[i:i + 2048] = torch.softmax(z, dim=1) @ v[:p]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    h, g, d = (case[n] for n in ("n_heads", "n_kv", "head_dim"))
    x = s.qkv.double().view(s.n_rows, h + 2 * g, d)
    if case["kind"] == "append":
        for b, n in enumerate(s.lens):
            a = int(s.row_start[b])
            pos = torch.arange(n, dtype=torch.float64, device="cuda") + s.pos0_list[b]
            for i in range(d // 2):
                w = pos * ROPE_THETA ** (-2.0 * i / d)
                c, sn = torch.cos(w)[:, None], torch.sin(w)[:, None]
                lo, hi = x[a:a + n, :h + g, i].clone(), x[a:a + n, :h + g, d // 2 + i].clone()
                x[a:a + n, :h + g, i], x[a:a + n, :h + g, d // 2 + i] = lo * c - hi * sn, hi * c + lo * sn
        # codes and scales go by the bf16 values, which have been rounded already
        return {"rows": x.view(s.n_rows, -1), "k": None, "v": None, "k_scale": None, "v_scale": None}
    out = torch.empty((s.n_rows, h, d), dtype=torch.float64, device="cuda")
    for b, n in enumerate(s.lens):
        if not n:
            continue
        a = int(s.row_start[b])
        for j in range(h):
            kv = j // (h // g)
            if case["kind"] == "prompt":
                k, v, first = x[a:a + n, h + kv], x[a:a + n, h + g + kv], 0
            else:
                first = s.pos0_list[b]
                k = s.k[b, kv, :first + n].double() * s.k_scale[b, kv].double().repeat_interleave(BLOCK)[:first + n, None]
                v = s.v[b, kv, :first + n].double() * s.v_scale[b, kv].double().repeat_interleave(BLOCK)[:first + n, None]
            out[a:a + n, j] = _attend(x[a:a + n, j], k, v, first + torch.arange(n, device="cuda"))
    return out.view(s.n_rows, h * d)
