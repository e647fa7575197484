// libsd2 -- the key/value cache in 8 bits (gfx950): what fills it, and attention of new tokens over it.
//
// A block of 32 positions of one head shares a scale, a power of two: a product with it is exact in fp32, bf16 and the matrix
// instructions, so quantising rounds once, a block that is still open is brought to a larger scale by its exponents alone, and
// attention applies scales where they cost nothing (keys: to the score; values: in the conversion to bf16).
#include "sd2_internal.h"
#include "sd2_rows.h"

namespace sd2 {

constexpr int kBlock = kKv8Block;

// ------------------------------------------------------------------ rotary embedding, rounding, storing
//
// Workgroup (block of positions that a sequence's new rows touch, key/value head): the block's new keys and values and the
// group's queries.  A thread owns four pairs of dimensions (i, i + D/2) of a row, so that a rotation needs nothing of another
// lane; D/8 threads are a row, and rows that the workgroup has no use for take further heads.  The angle is position times
// frequency in 64 bits, in revolutions: what is left after the whole ones are dropped has more bits than fp32 keeps.

// smallest e >= -100 with largest <= 448 * 2^e, as 2^e; largest: the magnitude bits of a finite bf16 value
__device__ __forceinline__ float kv8_scale(uint32_t largest) {
    const int exponent = (int)(largest >> 7) - 127, e = exponent - 8 + ((largest & 0x7fu) > 0x60u ? 1 : 0);  // 448 = 1.75 * 2^8
    return __uint_as_float((uint32_t)(max(e, -100) + 127) << 23);
}

// Four values as e4m3, to the nearest, ties to even.  Values beyond the range -- infinities: a scale takes in all that is
// finite -- become NaN, the format has no infinity.
__device__ __forceinline__ uint32_t pack_e4m3(f32x4 x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fabsf(x[i]) <= 448.f ? x[i] : __uint_as_float(0x7fc00000u);
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
}
__device__ __forceinline__ f32x4 unpack_e4m3(uint32_t c) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
}
__device__ __forceinline__ f32x4 bf16x4_to_f32(uint2 p) {
    return f32x4{__uint_as_float(p.x << 16), __uint_as_float(p.x & 0xffff0000u), __uint_as_float(p.y << 16), __uint_as_float(p.y & 0xffff0000u)};
}
// the largest magnitude among four bf16 values and `largest`, those that are not finite left out
__device__ __forceinline__ uint32_t largest_finite(uint2 p, uint32_t largest) {
    const uint32_t m[4] = {p.x & 0x7fffu, (p.x >> 16) & 0x7fffu, p.y & 0x7fffu, (p.y >> 16) & 0x7fffu};
#pragma unroll
    for (int i = 0; i < 4; ++i) largest = max(largest, m[i] < 0x7f80u ? m[i] : 0u);
    return largest;
}

struct AppendArgs {
    Kv8Args c;
    const float* qkv;
    const int32_t* row_start;
    const int32_t* pos0;
    int n_seq, n_rows, rep;
    double log2_theta;
    uint16_t* rows;
};

// blocks that the rows of a sequence touch, positions first .. first + n - 1
__device__ __forceinline__ uint32_t touched_blocks(int64_t first, int n) {
    return n ? (uint32_t)(((first + n - 1) >> 5) - (first >> 5) + 1) : 0u;
}

// P: passes of the workgroup over a full block's rows
template <int P>
__global__ __launch_bounds__(256) void kv8_append_kernel(AppendArgs a) {
    static_assert(kBlock == 32, "shifts by 5");
    __shared__ uint32_t largest[2];
    const int tid = threadIdx.x, grp = blockIdx.y, D = a.c.head_dim, half = D / 2;
    const SeqUnit u = find_unit(blockIdx.x, a.n_seq, [&](int b) { return touched_blocks(a.pos0[b], seq_rows(a.row_start, b, a.n_rows).count); });
    if (u.seq < 0) return;
    const SeqRows sr = seq_rows(a.row_start, u.seq, a.n_rows);
    const int64_t p0 = a.pos0[u.seq], block = (p0 >> 5) + u.index, lo_pos = block * kBlock;
    const int64_t first = max(p0, lo_pos);
    const int n_here = (int)(min(p0 + sr.count, lo_pos + kBlock) - first);
    const int row0 = sr.start + (int)(first - p0);
    const bool stored = block >= 0 && block < a.c.max_pos / kBlock;
    const int n_old = (int)min(max(p0 - lo_pos, (int64_t)0), (int64_t)kBlock);  // positions of the block that were there before
    const size_t head = (size_t)u.seq * a.c.n_kv + grp, at = head * (size_t)(a.c.max_pos / kBlock) + (size_t)block;
    if (tid < 2) largest[tid] = 0;
    float old_scale[2] = {0.f, 0.f};
    if (stored && n_old) {
        old_scale[0] = a.c.k_scale[at];
        old_scale[1] = a.c.v_scale[at];
    }
    const int lanes = D / 8, per_pass = 256 / lanes;             // threads of a row, rows of a pass
    const int rows_at_once = min(n_here, per_pass), others = per_pass / rows_at_once;  // threads of a row for different heads
    const int sub = tid / lanes, j = tid - sub * lanes, other = sub / rows_at_once, row_slot = sub - other * rows_at_once;
    const bool active = sub < per_pass && other < others;
    const int n_heads = a.c.n_kv * a.rep;
    const size_t width = (size_t)(n_heads + 2 * a.c.n_kv) * D;
    const int k_col = (n_heads + grp) * D + 4 * j, v_col = k_col + a.c.n_kv * D;
    double freq[4];  // revolutions a position
#pragma unroll
    for (int i = 0; i < 4; ++i) freq[i] = exp2(-2.0 * (4 * j + i) / D * a.log2_theta) * 0.15915494309189535;
    __syncthreads();

    uint2 kept[2][P][2];  // the rounded keys and values of the thread's rows, low and high dimensions
    uint32_t most[2] = {0u, 0u};
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int r = row_slot + p * rows_at_once;
        kept[0][p][0] = kept[0][p][1] = kept[1][p][0] = kept[1][p][1] = make_uint2(0u, 0u);
        if (!active || r >= n_here) continue;
        f32x4 c, s;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double turns = (double)(first + r) * freq[i];
            float sn, cs;
            sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
            c[i] = cs;
            s[i] = sn;
        }
        const float* src = a.qkv + (size_t)(row0 + r) * width;
        uint16_t* dst = a.rows + (size_t)(row0 + r) * width;
        auto put = [&](int col, uint2 lo, uint2 hi) {
            *reinterpret_cast<uint2*>(dst + col) = lo;
            *reinterpret_cast<uint2*>(dst + col + half) = hi;
        };
        auto rotated = [&](int col, uint2& lo, uint2& hi) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(src + col), y = *reinterpret_cast<const f32x4*>(src + col + half);
            const f32x4 l = x * c - y * s, h = y * c + x * s;
            lo = make_uint2(pack_bf16(l[0], l[1]), pack_bf16(l[2], l[3]));
            hi = make_uint2(pack_bf16(h[0], h[1]), pack_bf16(h[2], h[3]));
        };
        if (other == 0) {
            rotated(k_col, kept[0][p][0], kept[0][p][1]);
            put(k_col, kept[0][p][0], kept[0][p][1]);
            most[0] = largest_finite(kept[0][p][1], largest_finite(kept[0][p][0], most[0]));
        }
        if (other == (others > 1 ? 1 : 0)) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(src + v_col), y = *reinterpret_cast<const f32x4*>(src + v_col + half);
            kept[1][p][0] = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
            kept[1][p][1] = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            put(v_col, kept[1][p][0], kept[1][p][1]);
            most[1] = largest_finite(kept[1][p][1], largest_finite(kept[1][p][0], most[1]));
        }
        // the queries begin with the threads that have neither keys nor values
        for (int q = others > 2 ? (other + others - 2) % others : other; q < a.rep; q += others) {
            const int col = (grp * a.rep + q) * D + 4 * j;
            uint2 lo, hi;
            rotated(col, lo, hi);
            put(col, lo, hi);
        }
    }
    if (!stored) return;
#pragma unroll
    for (int w = 0; w < 2; ++w)
        if (most[w]) atomicMax(&largest[w], most[w]);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const float scale = fmaxf(kv8_scale(largest[w]), old_scale[w]), inv = 1.0f / scale;
        uint8_t* codes = (w ? a.c.v : a.c.k) + (head * a.c.max_pos + (size_t)lo_pos) * D;
        if (n_old && scale != old_scale[w]) {
            const float ratio = old_scale[w] * inv;
            uint32_t* word = reinterpret_cast<uint32_t*>(codes);
            for (int i = tid; i < n_old * D / 4; i += 256) word[i] = pack_e4m3(unpack_e4m3(word[i]) * ratio);
        }
        if (tid == 0) (w ? a.c.v_scale : a.c.k_scale)[at] = scale;
        if (!active || other != (w && others > 1 ? 1 : 0)) continue;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int r = row_slot + p * rows_at_once;
            if (r >= n_here) continue;
            uint8_t* dst = codes + (size_t)((int)(first - lo_pos) + r) * D + 4 * j;
            *reinterpret_cast<uint32_t*>(dst) = pack_e4m3(bf16x4_to_f32(kept[w][p][0]) * inv);
            *reinterpret_cast<uint32_t*>(dst + half) = pack_e4m3(bf16x4_to_f32(kept[w][p][1]) * inv);
        }
    }
}

hipError_t launch_kv8_append(const Kv8Args& c, const float* qkv, int n_heads, const int32_t* row_start, const int32_t* pos0, int n_seq,
                             int n_rows, double theta, uint16_t* rows, hipStream_t s) {
    if (c.head_dim < 16 || c.head_dim > 256 || c.head_dim % 16) return hipErrorInvalidValue;
    if (n_rows == 0 || n_seq == 0) return hipSuccess;
    const AppendArgs a = {c, qkv, row_start, pos0, n_seq, n_rows, n_heads / c.n_kv, log2(theta), rows};
    // n rows touch at most (n + 62) / 32 blocks
    const dim3 grid((unsigned)(n_rows / kBlock + 2 * (n_seq < n_rows ? n_seq : n_rows)), (unsigned)c.n_kv);
    const int per_pass = 256 / (c.head_dim / 8);
    if (per_pass >= 32) hipLaunchKernelGGL(kv8_append_kernel<1>, grid, dim3(256), 0, s, a);
    else if (per_pass >= 16) hipLaunchKernelGGL(kv8_append_kernel<2>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(kv8_append_kernel<4>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------ attention over the cache
//
// o = sum_j exp(q k_j / sqrt(D) - m) v_j / sum_j exp(q k_j / sqrt(D) - m), in one pass over the positions with a running maximum.
//
// The rows of a workgroup are (token, query head of the group) pairs in that order, up to 16 NR of them, so that a cached position
// is read and converted once for all of them.  A workgroup takes a stretch of positions, its four wavefronts every fourth tile of
// 32 -- one block, so a tile has one scale.  Scores come out transposed (positions by rows): a lane then holds eight positions of one
// row, which is how the next product wants its operand, so weights never leave the registers.  Positions are dealt to the rows of the
// first product such that those eight follow one another.  Values pass through LDS for the transposing read.
constexpr int kAttWaves = 4;
constexpr int kAttSpan = 32 * kAttWaves;  // positions of the workgroup's tiles side by side

struct Kv8AttArgs {
    Kv8Args c;
    const uint16_t* q;
    int64_t q_stride;
    const int32_t* row_start;
    const int32_t* pos0;
    int n_seq, n_rows, max_new, rep;
    int want;        // workgroups to aim for, for each key/value head
    uint32_t bound;  // units that the launch and the workspace have room for, for each key/value head
    float scale;     // log2(e) / sqrt(D)
    uint16_t* out;
    float* part;   // [units][key/value heads][16 NR][D]
    float2* stat;  // [units][key/value heads][16 NR]: running maximum (of scores times log2 e) and sum
};

// How a sequence is cut: row tiles and stretches of positions.  The stretch is the same for all sequences, so that workgroups are
// about equally long; a sequence's units are its row tiles times its stretches.
struct SeqCut {
    int start, count;  // rows
    int64_t pos0;
    int n_pos;         // positions that the last of them attends to
    uint32_t tiles, spans;
};
template <int ROWS>
__device__ __forceinline__ SeqCut seq_cut(const Kv8AttArgs& a, int b) {
    const SeqRows sr = seq_rows(a.row_start, b, a.n_rows);
    SeqCut s;
    s.start = sr.start;
    s.count = min(sr.count, a.max_new);
    s.pos0 = a.pos0[b];
    s.n_pos = (int)min(max(s.pos0 + s.count, (int64_t)0), (int64_t)a.c.max_pos);
    s.tiles = (uint32_t)(s.count * a.rep + ROWS - 1) / ROWS;
    s.spans = s.count ? (uint32_t)max((s.n_pos + kAttSpan - 1) / kAttSpan, 1) : 0u;
    return s;
}
// spans of a stretch
template <int ROWS>
__device__ __forceinline__ uint32_t stretch_of(const Kv8AttArgs& a) {
    const uint64_t all = total_units(a.n_seq, [&](int b) {
        const SeqCut s = seq_cut<ROWS>(a, b);
        return s.tiles * s.spans;
    });
    return max((uint32_t)((all + (uint32_t)a.want - 1) / (uint32_t)a.want), 1u);
}

typedef int i32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t e4m3x2_to_bf16(uint32_t codes, float scale, bool high) {
    const bf16x2 v = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
    return __builtin_bit_cast(uint32_t, v);
}
// eight codes as a matrix operand
__device__ __forceinline__ bf16x8 e4m3x8_to_bf16(uint32_t c0, uint32_t c1, float scale) {
    Frag f;
    f.u[0] = e4m3x2_to_bf16(c0, scale, false);
    f.u[1] = e4m3x2_to_bf16(c0, scale, true);
    f.u[2] = e4m3x2_to_bf16(c1, scale, false);
    f.u[3] = e4m3x2_to_bf16(c1, scale, true);
    return f.v;
}

// place of 16-byte piece c of row r in a tile of values: eight rows of a transposing read side by side fall into different banks
template <int D>
__device__ __forceinline__ int value_place(int r, int c) {
    constexpr int kPieces = D / 16;
    const int turn = D == 64 ? (r >> 2) & 3 : D == 128 ? (r >> 1) & 7 : r & 15;
    return 16 * (r * kPieces + (c ^ turn));
}

// wavefronts that share a SIMD's registers
constexpr int kv8_waves(int dim, int nr) { return dim == 256 ? 1 : dim * nr <= 64 ? 4 : dim * nr <= 128 ? 3 : 2; }

template <int D, int NR>
__global__ __launch_bounds__(64 * kAttWaves, kv8_waves(D, NR)) void kv8_attention_kernel(Kv8AttArgs a) {
    constexpr int kRows = 16 * NR, kDb = D / 16, kJ = D / 64, kPieces = D / 16, kTile = 32 * D, kLoads = kTile / 1024;
    constexpr int kORow = D + 4;  // floats
    constexpr int kMerge = kAttWaves * (16 * kORow + 32) * 4, kLds = kAttWaves * kTile > kMerge ? kAttWaves * kTile : kMerge;
    __shared__ __attribute__((aligned(16))) uint8_t smem[kLds];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int grp = blockIdx.x % a.c.n_kv;
    const uint32_t unit = blockIdx.x / a.c.n_kv;
    const uint32_t stretch = stretch_of<kRows>(a);
    const SeqUnit u = find_unit(unit, a.n_seq, [&](int b) {
        const SeqCut s = seq_cut<kRows>(a, b);
        return s.tiles * ((s.spans + stretch - 1) / stretch);
    });
    if (u.seq < 0) return;
    const SeqCut sc = seq_cut<kRows>(a, u.seq);
    const uint32_t cuts = (sc.spans + stretch - 1) / stretch;
    const int tile = (int)(u.index / cuts), cut = (int)(u.index % cuts);
    const int D_used = a.c.head_dim, rep = a.rep, n_used = sc.count * rep;  // rows of the sequence
    const int first = kRows * tile;
    // positions of this workgroup, up to the last that its last row attends to
    const int reach_last = (int)min(sc.pos0 + (min(first + kRows, n_used) - 1) / rep, (int64_t)a.c.max_pos - 1);
    const int from = cut * (int)stretch * kAttSpan, to = min(from + (int)stretch * kAttSpan, reach_last + 1);
    const int reach_first = (int)min(max(sc.pos0 + first / rep, (int64_t)-1), (int64_t)a.c.max_pos);  // of the tile's first row
    const size_t head = (size_t)u.seq * a.c.n_kv + grp;
    const uint8_t* kg = a.c.k + head * a.c.max_pos * D_used;
    const uint8_t* vg = a.c.v + head * a.c.max_pos * D_used;
    const float* ks = a.c.k_scale + head * (a.c.max_pos / kBlock);
    const float* vs = a.c.v_scale + head * (a.c.max_pos / kBlock);
    uint8_t* vt = smem + wave * kTile;

    u32x4 kr[2][kJ], vr[kLoads];
    float kscale = 0.f, vscale = 0.f;
    // K: lane (n, g) brings dimensions 64 j + 16 g .. + 15 of position 8 (n / 4) + 4 b + n % 4; V: pieces in memory's order
    auto request = [&](int base) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int jj = 0; jj < kJ; ++jj) {
                const int d = 64 * jj + 16 * g;
                kr[b][jj] = u32x4{0, 0, 0, 0};
                if (d < D_used)
                    kr[b][jj] = *reinterpret_cast<const u32x4*>(kg + (size_t)(base + 8 * (n >> 2) + 4 * b + (n & 3)) * D_used + d);
            }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int piece = 64 * i + lane, r = piece / kPieces, d = 16 * (piece % kPieces);
            vr[i] = u32x4{0, 0, 0, 0};
            if (d < D_used) vr[i] = *reinterpret_cast<const u32x4*>(vg + (size_t)(base + r) * D_used + d);
        }
        kscale = ks[base / kBlock];
        vscale = vs[base / kBlock];
    };
    int base = from + 32 * wave;
    if (base < to) request(base);

    bf16x8 q[NR][2 * kJ];  // in the order of the keys' dimensions
    int reach[NR];         // last position of row n
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        const int row = min(first + 16 * t + n, n_used - 1), token = row / rep, r = row - token * rep;
        reach[t] = (int)min(max(sc.pos0 + token, (int64_t)-1), (int64_t)a.c.max_pos - 1);
        const uint16_t* src = a.q + (size_t)(sc.start + token) * a.q_stride + (size_t)(grp * rep + r) * D_used;
#pragma unroll
        for (int jj = 0; jj < kJ; ++jj) {
            const int d = 64 * jj + 16 * g;
            Frag f0, f1;
            f0.q = f1.q = u32x4{0, 0, 0, 0};
            if (d < D_used) {
                f0.q = *reinterpret_cast<const u32x4*>(src + d);
                f1.q = *reinterpret_cast<const u32x4*>(src + d + 8);
            }
            q[t][2 * jj] = f0.v;
            q[t][2 * jj + 1] = f1.v;
        }
    }
    float m[NR], l[NR];
    f32x4 o[NR][kDb];  // [dimension block]: dimensions 16 db + 4 g + i of row n
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        m[t] = -3.0e38f;
        l[t] = 0.f;
#pragma unroll
        for (int d = 0; d < kDb; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (; base < to; base += kAttSpan) {
        f32x4 s[NR][2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            bf16x8 kf[2 * kJ];
#pragma unroll
            for (int jj = 0; jj < kJ; ++jj) {
                kf[2 * jj] = e4m3x8_to_bf16(kr[b][jj][0], kr[b][jj][1], 1.0f);
                kf[2 * jj + 1] = e4m3x8_to_bf16(kr[b][jj][2], kr[b][jj][3], 1.0f);
            }
#pragma unroll
            for (int t = 0; t < NR; ++t) {
                s[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int jj = 0; jj < 2 * kJ; ++jj) s[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[jj], q[t][jj], s[t][b], 0, 0, 0);
            }
        }
        const float c = kscale * a.scale, v_scale = vscale;
        const bool masked = base + 31 > reach_first;
        bool odd_values = false;  // a value of a position that not every row attends to is NaN
        if (masked) {
            const int n_here = to - base;  // positions past the last are whatever the memory held
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if ((64 * i + lane) / kPieces >= n_here) vr[i] = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 4; ++e) odd_values |= ((((vr[i][e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0);
            }
            odd_values = __any(odd_values);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int piece = 64 * i + lane;
            *reinterpret_cast<u32x4*>(vt + value_place<D>(piece / kPieces, piece % kPieces)) = vr[i];
        }
        if (base + kAttSpan < to) request(base + kAttSpan);
        bf16x8 p[NR];
#pragma unroll
        for (int t = 0; t < NR; ++t) {
            float w[8], mx = -3.0e38f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = s[t][e >> 2][e & 3] * c;
                if (masked && base + 8 * g + e > reach[t]) w[e] = -__builtin_inff();
                mx = fmaxf(mx, w[e]);
            }
            // The maximum follows only where a weight could grow past 2^8: sums of weights up to that are as exact as those below 1.
            if (__any(mx > m[t] + 8.f)) {
                const float top = fmaxf(m[t], max_quarters(max_halves(mx))), f = __builtin_amdgcn_exp2f(m[t] - top);
                m[t] = top;
                l[t] *= f;
#pragma unroll
                for (int d = 0; d < kDb; ++d) o[t][d] *= f;
            }
            Frag pair;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(w[e] - m[t]);
                l[t] += w[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) pair.u[e] = pack_bf16(w[2 * e], w[2 * e + 1]);
            p[t] = pair.v;
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        // sixteen lanes read eight rows of sixteen dimensions; each gets eight positions of its own dimension
        auto values = [&](int d) __attribute__((always_inline)) {
            const auto* src = (const __attribute__((address_space(3))) uint8_t*)vt + value_place<D>(8 * g + (n >> 1), d) + 8 * (n & 1);
            return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)src);
        };
        if (!odd_values) {
#pragma unroll
            for (int d = 0; d < kDb; ++d) {
                const i32x2 codes = values(d);
                const bf16x8 v = e4m3x8_to_bf16((uint32_t)codes[0], (uint32_t)codes[1], v_scale);
#pragma unroll
                for (int t = 0; t < NR; ++t) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[t], o[t][d], 0, 0, 0);
            }
        } else {
            // A weight of zero times NaN is NaN, also where the row does not attend to the position: NaN goes in as zero, and where a row
            // attends to one -- a product of two masks of ones tells -- its result becomes NaN.
            bf16x8 attends[NR];
#pragma unroll
            for (int t = 0; t < NR; ++t) {
                Frag f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    f.u[e] = (base + 8 * g + 2 * e <= reach[t] ? 0x3f80u : 0u) | (base + 8 * g + 2 * e + 1 <= reach[t] ? 0x3f800000u : 0u);
                attends[t] = f.v;
            }
#pragma unroll
            for (int d = 0; d < kDb; ++d) {
                const i32x2 codes = values(d);
                const uint32_t c0 = (uint32_t)codes[0], c1 = (uint32_t)codes[1];
                const uint32_t n0 = (((c0 & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u, n1 = (((c1 & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u;
                const bf16x8 v = e4m3x8_to_bf16(c0 & ~(n0 * 0xffu), c1 & ~(n1 * 0xffu), v_scale);
                const bf16x8 nan = e4m3x8_to_bf16(n0 * 0x38u, n1 * 0x38u, 1.0f);
#pragma unroll
                for (int t = 0; t < NR; ++t) {
                    const f32x4 hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(nan, attends[t], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                    o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[t], o[t][d], 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[t][d][i] = hits[i] > 0.f ? __builtin_nanf("") : o[t][d][i];
                }
            }
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();  // the next tile overwrites the values
    }

    // the wavefronts' results meet in LDS, sixteen rows at a time
    float* mo = reinterpret_cast<float*>(smem);                     // [wave][16][kORow]
    float2* mstat = reinterpret_cast<float2*>(mo + kAttWaves * 16 * kORow);  // [wave][16]
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        const float sum = sum_quarters(sum_halves(l[t]));
        __syncthreads();
#pragma unroll
        for (int d = 0; d < kDb; ++d) *reinterpret_cast<f32x4*>(mo + (16 * wave + n) * kORow + 16 * d + 4 * g) = o[t][d];
        if (g == 0) mstat[16 * wave + n] = make_float2(m[t], sum);
        __syncthreads();
        const int r16 = tid >> 4, row = first + 16 * t + r16;  // sixteen threads a row
        if (row < n_used) {
            float w[kAttWaves], top = -3.0e38f, all = 0.f;
#pragma unroll
            for (int i = 0; i < kAttWaves; ++i) top = fmaxf(top, mstat[16 * i + r16].x);
#pragma unroll
            for (int i = 0; i < kAttWaves; ++i) {
                const float2 st = mstat[16 * i + r16];
                w[i] = __builtin_amdgcn_exp2f(st.x - top);
                all += w[i] * st.y;
            }
            const int token = row / rep;
            // a row that attends to nothing is zero
            const float inv = sc.pos0 + token < 0 ? 0.f : 1.0f / all;
            const size_t slot = ((size_t)unit * a.c.n_kv + grp) * kRows + 16 * t + r16;
            if (cuts > 1 && (tid & 15) == 0) a.stat[slot] = make_float2(top, all);
#pragma unroll
            for (int d = 4 * (tid & 15); d < D; d += 64) {
                if (d >= D_used) break;
                f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < kAttWaves; ++i) x += *reinterpret_cast<const f32x4*>(mo + (16 * i + r16) * kORow + d) * w[i];
                if (cuts > 1) {
                    *reinterpret_cast<f32x4*>(a.part + slot * D + d) = x;
                } else {
                    x *= inv;
                    uint16_t* dst = a.out + ((size_t)(sc.start + token) * a.c.n_kv * rep + (size_t)grp * rep + (row - token * rep)) * D_used + d;
                    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
                }
            }
        }
    }
}

// Joins the stretches of a sequence that was cut: a wavefront for each (row, query head), a lane for D / 64 dimensions.
template <int D, int NR>
__global__ __launch_bounds__(256) void kv8_combine_kernel(Kv8AttArgs a) {
    constexpr int kRows = 16 * NR, kPer = D / 64;
    const int lane = threadIdx.x & 63, n_heads = a.c.n_kv * a.rep;
    const uint32_t item = blockIdx.x * 4 + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int row = (int)(item / (uint32_t)n_heads), h = (int)(item % (uint32_t)n_heads);
    if (row >= a.n_rows) return;
    const SeqUnit by_row = find_unit((uint32_t)row, a.n_seq, [&](int b) { return (uint32_t)seq_rows(a.row_start, b, a.n_rows).count; });
    if (by_row.seq < 0) return;
    const SeqCut sc = seq_cut<kRows>(a, by_row.seq);
    const int token = row - sc.start;
    if (token < 0 || token >= sc.count) return;
    const uint32_t stretch = stretch_of<kRows>(a), cuts = (sc.spans + stretch - 1) / stretch;
    if (cuts <= 1) return;
    const uint32_t before = (uint32_t)total_units(by_row.seq, [&](int b) {
        const SeqCut s = seq_cut<kRows>(a, b);
        return s.tiles * ((s.spans + stretch - 1) / stretch);
    });
    const int grp = h / a.rep, local = token * a.rep + (h - grp * a.rep), tile = local / kRows;
    const uint32_t unit0 = before + (uint32_t)tile * cuts;
    if (unit0 + cuts > a.bound) return;
    const size_t slot0 = ((size_t)unit0 * a.c.n_kv + grp) * kRows + local % kRows, step = (size_t)a.c.n_kv * kRows;
    float top = -3.0e38f;
    for (uint32_t i = lane; i < cuts; i += 64) top = fmaxf(top, a.stat[slot0 + i * step].x);
    top = max_quarters(max_halves(top));
#pragma unroll
    for (int i = 1; i < 16; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
    float all = 0.f, x[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = 0.f;
#pragma unroll 4
    for (uint32_t i = 0; i < cuts; ++i) {
        const float2 st = a.stat[slot0 + i * step];
        const float w = __builtin_amdgcn_exp2f(st.x - top);
        all += w * st.y;
        const float* src = a.part + (slot0 + i * step) * D + kPer * lane;
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] += w * (kPer * lane + e < a.c.head_dim ? src[e] : 0.f);
    }
    const float inv = sc.pos0 + token < 0 ? 0.f : 1.0f / all;
    uint16_t* dst = a.out + ((size_t)row * n_heads + h) * a.c.head_dim + kPer * lane;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (kPer * lane + e < a.c.head_dim) dst[e] = f32_to_bf16(x[e] * inv);
}

// Rows of a workgroup: as many of a sequence's as there can be, up to what the registers hold.
Kv8Plan kv8_plan(int n_heads, int n_kv, int head_dim, int n_seq, int max_new) {
    Kv8Plan p;
    const int rows = max_new * (n_heads / n_kv);
    p.dim = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256;
    p.nr = rows <= 16 || p.dim == 256 ? 1 : rows <= 32 || p.dim == 128 ? 2 : 4;
    const int kv = n_kv;
    p.want = (2 * device_cu_count() + kv - 1) / kv;
    p.tiles = (rows + 16 * p.nr - 1) / (16 * p.nr);
    // units: sum of tiles * ceil(spans / stretch) <= sum of tiles * spans / stretch + sum of tiles
    p.bound = (uint32_t)p.want + (uint32_t)n_seq * (uint32_t)p.tiles;
    const size_t slots = (size_t)p.bound * kv * 16 * p.nr;
    p.stat_off = slots * p.dim * sizeof(float);
    p.bytes = p.stat_off + slots * sizeof(float2);
    return p;
}

hipError_t launch_kv8_attention(const Kv8Args& c, const uint16_t* q, int64_t q_stride, int n_heads, const int32_t* row_start,
                                const int32_t* pos0, int n_seq, int n_rows, int max_new, uint16_t* out, void* ws, hipStream_t s) {
    if (c.head_dim < 16 || c.head_dim > 256 || c.head_dim % 16) return hipErrorInvalidValue;
    if (n_rows == 0 || n_seq == 0) return hipSuccess;
    const Kv8Plan p = kv8_plan(n_heads, c.n_kv, c.head_dim, n_seq, max_new);
    const int rep = n_heads / c.n_kv;
    Kv8AttArgs a = {c, q, q_stride, row_start, pos0, n_seq, n_rows, max_new, rep, p.want, p.bound,
                    (float)(1.4426950408889634 / sqrt((double)c.head_dim)), out, static_cast<float*>(ws),
                    reinterpret_cast<float2*>(static_cast<uint8_t*>(ws) + p.stat_off)};
    // row tiles that these rows can have
    const uint64_t tiles = (uint64_t)n_rows * rep / (16 * p.nr) + (uint64_t)(n_seq < n_rows ? n_seq : n_rows);
    const uint64_t most = (uint64_t)n_seq * p.tiles;
    const dim3 grid((unsigned)((p.want + (tiles < most ? tiles : most)) * c.n_kv)), join((unsigned)(((uint64_t)n_rows * n_heads + 3) / 4));
#define SD2_KV8(DIM, R)                                                                              \
    if (p.dim == DIM && p.nr == R) {                                                                 \
        hipLaunchKernelGGL((kv8_attention_kernel<DIM, R>), grid, dim3(64 * kAttWaves), 0, s, a);      \
        if (c.max_pos > kAttSpan) hipLaunchKernelGGL((kv8_combine_kernel<DIM, R>), join, dim3(256), 0, s, a); \
    }
    SD2_KV8(64, 1) SD2_KV8(64, 2) SD2_KV8(64, 4)
    SD2_KV8(128, 1) SD2_KV8(128, 2)
    SD2_KV8(256, 1)
#undef SD2_KV8
    return hipGetLastError();
}

}  // namespace sd2
