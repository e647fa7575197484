// libsd2 -- the key/value cache in 8 bits (gfx950): what fills it, and attention of new tokens over it.
//
// A block of 32 positions of one head shares a scale, a power of two: a product with it is exact in fp32, bf16 and the matrix
// instructions, so quantising rounds once, a block that is still open is brought to a larger scale by its exponents alone, and
// attention applies scales where they cost nothing (keys: to the score; values: in the conversion to bf16).
#include <algorithm>

#include "sd2_internal.h"
#include "sd2_rows.h"

namespace sd2 {

constexpr int kBlock = kKv8Block;

// ------------------------------------------------------------------ rotary embedding, rounding, storing
//
// Workgroup (block of positions that a sequence's new rows touch, key/value head): the block's new keys and values and the
// group's queries.  A thread owns eight pairs of dimensions (i, i + D/2) of a row, so that a rotation needs nothing of another
// lane; D/16 threads are a row, and threads that have no row of their own take further heads of the others'.  The angle is position
// times frequency in 64 bits, in revolutions: what is left after the whole ones are dropped has more bits than fp32 keeps.
// Bound by bytes: 9557 rows of 40 heads of 128 (fp32 in, bf16 and codes out, 313 MB) in 70 us, 4.5 TB/s, where a copy has 4.9; a single
// token by its chain of loads, 5.3 us.  (Four pairs a thread and no head ahead: 75 and 5.7 us.)

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
__device__ __forceinline__ f32x4 bf16x4_to_f32(uint32_t a, uint32_t b) {
    return f32x4{__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)};
}
// the largest magnitude among two bf16 values and `largest`, those that are not finite left out
__device__ __forceinline__ uint32_t largest_finite(uint32_t pair, uint32_t largest) {
    const uint32_t lo = pair & 0x7fffu, hi = (pair >> 16) & 0x7fffu;
    return max(largest, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
}

struct AppendArgs {
    Kv8Args c;
    const int32_t* row_start;
    const int32_t* pos0;
    int n_seq, n_rows, rep;
    double log2_theta, step;  // step: ratio of the frequencies of neighbouring dimensions
};

// blocks that the rows of a sequence touch, positions first .. first + n - 1
__device__ __forceinline__ uint32_t touched_blocks(int64_t first, int n) {
    return n ? (uint32_t)(((first + n - 1) >> 5) - (first >> 5) + 1) : 0u;
}

// P: passes of the workgroup over a full block's rows
template <int P>
__global__ __launch_bounds__(256) void kv8_append_kernel(AppendArgs a, const float* __restrict__ qkv, uint16_t* __restrict__ out) {
    static_assert(kBlock == 32, "shifts by 5");
    __shared__ uint32_t largest[2];
    const int tid = threadIdx.x, grp = blockIdx.y, D = a.c.head_dim, half = D / 2;
    const Sequences seqs(a.row_start, a.pos0, a.n_seq, a.n_rows);
    const int lanes = D / 16, per_pass = 256 / lanes, sub = tid / lanes, j = tid - sub * lanes;  // threads of a row, rows of a pass
    double freq[8];  // revolutions a position, while the lengths are on their way
    freq[0] = exp2((double)(-16 * j) / D * a.log2_theta) * 0.15915494309189535;
#pragma unroll
    for (int i = 1; i < 8; ++i) freq[i] = freq[i - 1] * a.step;
    const SeqUnit u = seqs.find(blockIdx.x, [](const SeqRows& r) { return touched_blocks(r.pos0, r.count); });
    if (u.seq < 0) return;
    const SeqRows sr = u.rows;
    const int64_t p0 = sr.pos0, block = (p0 >> 5) + u.index, lo_pos = block * kBlock;
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
    const int rows_at_once = min(n_here, per_pass), others = per_pass / rows_at_once;  // threads of a row for different heads
    const int other = sub / rows_at_once, row_slot = sub - other * rows_at_once;
    const bool active = sub < per_pass && other < others;
    const bool has_k = other == 0, has_v = other == (others > 1 ? 1 : 0);
    const int n_heads = a.c.n_kv * a.rep;
    const size_t width = (size_t)(n_heads + 2 * a.c.n_kv) * D;
    const int k_col = (n_heads + grp) * D + 8 * j, v_col = k_col + a.c.n_kv * D, q_col = grp * a.rep * D + 8 * j;
    __syncthreads();

    u32x4 kept[2][P][2];  // the rounded keys and values of the thread's rows, low and high dimensions
    uint32_t most[2] = {0u, 0u};
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int r = row_slot + p * rows_at_once;
#pragma unroll
        for (int w = 0; w < 4; ++w) kept[w >> 1][p][w & 1] = u32x4{0, 0, 0, 0};
        if (!active || r >= n_here) continue;
        const float* src = qkv + (size_t)(row0 + r) * width;
        uint16_t* dst = out + (size_t)(row0 + r) * width;
        struct Pairs {
            f32x4 x[2], y[2];
        };
        auto load = [&](int col) __attribute__((always_inline)) {
            const f32x4 *lo = reinterpret_cast<const f32x4*>(src + col), *hi = reinterpret_cast<const f32x4*>(src + col + half);
            return Pairs{{lo[0], lo[1]}, {hi[0], hi[1]}};
        };
        auto pack = [](const f32x4& u, const f32x4& v) __attribute__((always_inline)) {
            return u32x4{pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        };
        auto put = [&](int col, const u32x4& lo, const u32x4& hi) __attribute__((always_inline)) {
            *reinterpret_cast<u32x4*>(dst + col) = lo;
            *reinterpret_cast<u32x4*>(dst + col + half) = hi;
        };
        // the queries begin with the threads that have neither keys nor values; a head's rows are asked for a head ahead
        int q = others > 2 ? (other + others - 2) % others : other;
        Pairs kx, vx, qx;
        if (has_k) kx = load(k_col);
        if (has_v) vx = load(v_col);
        if (q < a.rep) qx = load(q_col + q * D);
        f32x4 c[2], s[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double turns = (double)(first + r) * freq[i];
            float sn, cs;
            sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
            c[i >> 2][i & 3] = cs;
            s[i >> 2][i & 3] = sn;
        }
        auto rotate = [&](const Pairs& v, u32x4& lo, u32x4& hi) __attribute__((always_inline)) {
            lo = pack(v.x[0] * c[0] - v.y[0] * s[0], v.x[1] * c[1] - v.y[1] * s[1]);
            hi = pack(v.y[0] * c[0] + v.x[0] * s[0], v.y[1] * c[1] + v.x[1] * s[1]);
        };
        if (has_k) {
            rotate(kx, kept[0][p][0], kept[0][p][1]);
            put(k_col, kept[0][p][0], kept[0][p][1]);
        }
        if (has_v) {
            kept[1][p][0] = pack(vx.x[0], vx.x[1]);
            kept[1][p][1] = pack(vx.y[0], vx.y[1]);
            put(v_col, kept[1][p][0], kept[1][p][1]);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int e = 0; e < 4; ++e) most[w >> 1] = largest_finite(kept[w >> 1][p][w & 1][e], most[w >> 1]);
        while (q < a.rep) {
            const int col = q_col + q * D;
            const Pairs now = qx;
            q += others;
            if (q < a.rep) qx = load(q_col + q * D);
            u32x4 lo, hi;
            rotate(now, lo, hi);
            put(col, lo, hi);
        }
    }
    if (!stored) return;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const uint32_t all = wave_max(most[w]);
        if ((tid & 63) == 0) atomicMax(&largest[w], all);
    }
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
        if (!active || !(w ? has_v : has_k)) continue;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int r = row_slot + p * rows_at_once;
            if (r >= n_here) continue;
            uint8_t* dst = codes + (size_t)((int)(first - lo_pos) + r) * D + 8 * j;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const u32x4 x = kept[w][p][e];
                *reinterpret_cast<uint2*>(dst + e * half) = make_uint2(pack_e4m3(bf16x4_to_f32(x[0], x[1]) * inv), pack_e4m3(bf16x4_to_f32(x[2], x[3]) * inv));
            }
        }
    }
}

hipError_t launch_kv8_append(const Kv8Args& c, const float* qkv, int n_heads, const int32_t* row_start, const int32_t* pos0, int n_seq,
                             int n_rows, double theta, uint16_t* rows, hipStream_t s) {
    if (c.head_dim < 16 || c.head_dim > 256 || c.head_dim % 16) return hipErrorInvalidValue;
    if (n_rows == 0 || n_seq == 0) return hipSuccess;
    const AppendArgs a = {c, row_start, pos0, n_seq, n_rows, n_heads / c.n_kv, log2(theta), exp2(-2.0 / c.head_dim * log2(theta))};
    // n rows touch at most (n + 62) / 32 blocks
    const dim3 grid((unsigned)(n_rows / kBlock + 2 * (n_seq < n_rows ? n_seq : n_rows)), (unsigned)c.n_kv);
    if (c.head_dim <= 128) hipLaunchKernelGGL(kv8_append_kernel<1>, grid, dim3(256), 0, s, a, qkv, rows);
    else hipLaunchKernelGGL(kv8_append_kernel<2>, grid, dim3(256), 0, s, a, qkv, rows);
    return hipGetLastError();
}

// ------------------------------------------------------------------ attention over the cache
//
// o = sum_j exp(q k_j / sqrt(D) - m) v_j / sum_j exp(q k_j / sqrt(D) - m), in one pass over the positions with a running maximum.
//
// The rows of a workgroup are (token, query head of the group) pairs in that order, up to 16 NR of them, so that a cached position
// is read and converted once for all of them.  A workgroup takes a stretch of positions, its four wavefronts every fourth tile of
// 32 -- one block, so a tile has one scale; short caches are not cut, and eight wavefronts take all of one.  Scores come out transposed
// (positions by rows): a lane then holds eight positions of one row, which is how the next product wants its operand, so weights never
// leave the registers.  Positions are dealt to the rows of the first product such that those eight follow one another.  Tiles go from
// memory straight into LDS, one ahead of the one at work, and values leave it by the transposing read.  Weights are rounded to bf16 for
// the second product, at most 2^-8 of a weight.
//
// Bound by bytes where there are many positions: 60 requests with 224 802 positions in 16 heads of keys and values of 128 (464 MB) 95 us,
// 4.9 TB/s, where a pure read has 5.35 (and 5 us to join); by the chain plan - first tile - scores - meeting (- join) where there are few:
// one token against 429 positions 6.7 us (8.1 in a cache of 8192, which is cut), five against 30016 15 us.  64 tokens with four query heads a
// group: 1.9 us for 128 positions of 64 rows, softmax and conversions on the vector ALU.
constexpr int kCutWaves = 4, kWholeWaves = 8;  // wavefronts of a workgroup that takes a stretch, and of one that takes all positions
constexpr int kAttSpan = 32 * kCutWaves;        // positions of four tiles side by side: what stretches are made of

constexpr uint32_t kRest = 0x80000000u;

// Values enter the second product at 2^-8 of their size, and results are multiplied by 2^8 at the end.  The largest that is stored is
// 256 * 2^120, more than bf16 and fp32 have: as an infinity, it would be NaN in the rows whose weight for it is zero.  The smallest,
// 2^-109, stays a normal number.
constexpr float kValuesIn = 0x1p-8f, kResultsOut = 0x1p8f;

struct Kv8AttArgs {
    Kv8Args c;
    const uint16_t* q;
    int64_t q_stride;
    const int32_t* row_start;
    const int32_t* pos0;
    int n_seq, n_rows, max_new, rep;
    int places;      // workgroups that run at the same time, for each key/value head
    uint32_t bound;  // units that the launch and the workspace have room for, for each key/value head
    float scale;     // log2(e) / sqrt(D)
    uint16_t* out;
    float* part;   // [units][key/value heads][16 NR][D]
    float2* stat;  // [units][key/value heads][16 NR]: running maximum (of scores times log2 e) and sum
    uint4* join;   // [sequences][max_new][query heads]: first unit of a row, its whole stretches (kRest: and a shorter one), the unit of that
};

// How a sequence is cut: row tiles and stretches of positions.  The stretch is the same for all sequences, so that workgroups are
// about equally long; a sequence's units are its row tiles times its stretches.
struct SeqCut {
    int count, n_pos;  // rows; positions that the last of them attends to
    uint32_t tiles, spans;
};
template <int ROWS>
__device__ __forceinline__ SeqCut seq_cut(const Kv8AttArgs& a, const SeqRows& r) {
    SeqCut s;
    s.count = min(r.count, a.max_new);
    s.n_pos = (int)min(max((int64_t)r.pos0 + s.count, (int64_t)0), (int64_t)a.c.max_pos);
    s.tiles = (uint32_t)(s.count * a.rep + ROWS - 1) / ROWS;
    s.spans = s.count ? (uint32_t)max((s.n_pos + kAttSpan - 1) / kAttSpan, 1) : 0u;
    return s;
}

// Spans of a stretch, the same for all sequences.  With few row tiles: as few spans as let all stretches run side by side (64 rows against
// 500 to 4000 positions, four sequences: 24 us with 512 stretches for 512 places, 26 with 448, 32 with 320 and with 832).  With many, twice
// as many stretches as places, whole ones first and what is left of each sequence behind them: sequences differ in length, and the short
// ones fill the gaps (60 sequences of 19 to 16005 positions: 101 us; 114 with a stretch a place, 103 with three; 103 with two in the
// sequences' order).  A sequence of more than 128 spans is not cut into single ones, as what they leave has to be joined (30000
// positions: 17.6 us cut into single spans, 14.8 into pairs).
template <int ROWS>
__device__ __forceinline__ uint32_t stretch_of(const Kv8AttArgs& a, const Sequences& seqs, bool& many) {
    const uint64_t all = seqs.total([&](const SeqRows& r) {
        const SeqCut s = seq_cut<ROWS>(a, r);
        return s.tiles * s.spans;
    });
    const uint32_t tiles = (uint32_t)seqs.total([&](const SeqRows& r) { return seq_cut<ROWS>(a, r).tiles; });
    const uint32_t places = (uint32_t)a.places;
    auto share = [&](uint32_t n) { return (uint32_t)((all + n - 1) / n); };
    many = 2 * tiles > places;
    if (many) return max(share(2 * places), 1u);
    uint32_t stretch = max(share(places), all > 128 * (uint64_t)tiles ? 2u : 1u);
    const uint32_t enough = share(places - tiles);  // a sequence's last stretch may be short: no more than one for each row tile
    while (stretch < enough && seqs.total([&](const SeqRows& r) {
               const SeqCut s = seq_cut<ROWS>(a, r);
               return s.tiles * ((s.spans + stretch - 1) / stretch);
           }) > places)
        stretch = min(stretch + max(stretch / 16, 1u), enough);
    return stretch;
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

// Byte offset of 16-byte piece c of row r in a tile of keys or values: the pieces of a row are turned by its number, which spreads the
// reads over the banks -- keys: sixteen rows side by side, values: eight rows of a transposing read, sixteen lanes each.
template <int D>
__device__ __forceinline__ int turned(int r, int c) {
    return c ^ (D == 64 ? (r >> 2) & 3 : D == 128 ? (r >> 1) & 7 : r & 15);
}
template <int D>
__device__ __forceinline__ int tile_place(int r, int c) {
    return 16 * (r * (D / 16) + turned<D>(r, c));
}

// Eight positions of one dimension in every lane, for 16 N dimensions: sixteen lanes read eight rows of sixteen dimensions.  The wait
// is inside, as the compiler would wait for the tile under way as well: it cannot tell the two buffers apart.
template <int N>
__device__ __forceinline__ void read_values(i32x2 (&v)[N], const uint32_t (&at)[N]) {
    static_assert(N % 4 == 0, "read four at a time");
#pragma unroll
    for (int i = 0; i < N; i += 4)
        asm volatile(
            "ds_read_b64_tr_b8 %0, %4\n\tds_read_b64_tr_b8 %1, %5\n\tds_read_b64_tr_b8 %2, %6\n\tds_read_b64_tr_b8 %3, %7\n\ts_waitcnt lgkmcnt(0)"
            : "=&v"(v[i]), "=&v"(v[i + 1]), "=&v"(v[i + 2]), "=&v"(v[i + 3])
            : "v"(at[i]), "v"(at[i + 1]), "v"(at[i + 2]), "v"(at[i + 3])
            : "memory");
}

// the wavefronts' tiles, and afterwards their results: rows of dim + 4 sums, maxima and sums of weights
constexpr int kv8_lds(int dim, int nr, int waves) {
    const int tiles = waves * 2 * 2 * 32 * dim, results = waves * 16 * nr * (dim + 4 + 2) * 4;
    return tiles > results ? tiles : results;
}
// wavefronts that share a SIMD's registers
constexpr int kv8_waves(int dim, int nr, int waves) { return waves == kWholeWaves ? 2 : dim == 256 ? 1 : dim * nr <= 64 ? 4 : dim * nr <= 128 ? 3 : 2; }

// W: kCutWaves or kWholeWaves
template <int D, int NR, int W>
__global__ __launch_bounds__(64 * W, kv8_waves(D, NR, W)) void kv8_attention_kernel(Kv8AttArgs a) {
    constexpr int kRows = 16 * NR, kDb = D / 16, kJ = D / 64, kPieces = D / 16, kTile = 32 * D, kLoads = kTile / 1024;
    constexpr int kORow = D + 4;  // floats
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];  // [wave][buffer][keys, values][32][D]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const uint32_t block = folded_block(), n_kv = (uint32_t)a.c.n_kv, unit = block / n_kv;
    const int grp = (int)(block - unit * n_kv);
    if (unit >= a.bound) return;  // offsets that break the rules can have more units than the workspace has room for
    const Sequences seqs(a.row_start, a.pos0, a.n_seq, a.n_rows);
    bool many = false;
    uint32_t stretch = 1u << 13, n_whole = ~0u;  // as many spans as the longest cache has
    SeqUnit u;
    if constexpr (W == kWholeWaves) {
        u = seqs.find(unit, [&](const SeqRows& r) { return seq_cut<kRows>(a, r).tiles; });
    } else {
        stretch = stretch_of<kRows>(a, seqs, many);
        // with many, whole stretches first, then what is left of each sequence
        auto whole = [&](const SeqRows& r) {
            const SeqCut s = seq_cut<kRows>(a, r);
            return s.tiles * ((many ? s.spans : s.spans + stretch - 1) / stretch);
        };
        if (many) n_whole = (uint32_t)seqs.total(whole);
        u = unit < n_whole ? seqs.find(unit, whole) : seqs.find(unit - n_whole, [&](const SeqRows& r) {
            const SeqCut s = seq_cut<kRows>(a, r);
            return s.spans % stretch ? s.tiles : 0u;
        });
    }
    if (u.seq < 0) return;
    const SeqCut sc = seq_cut<kRows>(a, u.rows);
    const int64_t pos0 = u.rows.pos0;
    const uint32_t cuts = (sc.spans + stretch - 1) / stretch, cuts_whole = many ? sc.spans / stretch : cuts;
    const int tile = (int)(unit < n_whole ? u.index / cuts_whole : u.index), cut = (int)(unit < n_whole ? u.index % cuts_whole : cuts_whole);
    const int D_used = a.c.head_dim, rep = a.rep, n_used = sc.count * rep;  // rows of the sequence
    const int first = kRows * tile;
    // positions of this workgroup, up to the last that its last row attends to
    const int reach_last = (int)min(pos0 + (min(first + kRows, n_used) - 1) / rep, (int64_t)a.c.max_pos - 1);
    const int from = cut * (int)stretch * kAttSpan, to = min(from + (int)stretch * kAttSpan, reach_last + 1);
    const int reach_first = (int)min(max(pos0 + first / rep, (int64_t)-1), (int64_t)a.c.max_pos);  // of the tile's first row
    const int rows_here = min(n_used - first, kRows);  // row tiles past these are left out
    const size_t head = (size_t)u.seq * a.c.n_kv + grp;
    const uint8_t* kg = a.c.k + head * a.c.max_pos * D_used;
    const uint8_t* vg = a.c.v + head * a.c.max_pos * D_used;
    const float* ks = a.c.k_scale + head * (a.c.max_pos / kBlock);
    const float* vs = a.c.v_scale + head * (a.c.max_pos / kBlock);
    uint8_t* ring = smem + wave * 4 * kTile;

    if (D_used < D) {  // dimensions that the heads do not have: zero, and never written again
        for (int i = lane; i < 4 * kTile / 16; i += 64) reinterpret_cast<u32x4*>(ring)[i] = u32x4{0, 0, 0, 0};
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): in front of what follows
        asm volatile("" ::: "memory");
    }
    // A tile straight into LDS: 2 kLoads requests of 1 KiB, rows lane / kPieces + 64 / kPieces i.
    const int r0 = lane / kPieces, c0 = lane % kPieces;
    auto request = [&](int base, int buf) __attribute__((always_inline)) {
        const uint8_t* kb = kg + (size_t)base * D_used;
        const uint8_t* vb = vg + (size_t)base * D_used;
        auto* to_lds = (__attribute__((address_space(3))) uint8_t*)(ring + 2 * buf * kTile);
        auto piece = [&](int i) __attribute__((always_inline)) {
            const int r = r0 + 64 / kPieces * i, d = 16 * turned<D>(r, c0);
            if (D_used == D || d < D_used) {
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(kb + (uint32_t)(r * D_used + d)), to_lds + 1024 * i, 16, 0, 0);
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(vb + (uint32_t)(r * D_used + d)), to_lds + kTile + 1024 * i, 16, 0, 0);
            }
        };
        if (D_used == D) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) piece(i);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) piece(i);
        }
    };
    int base = from + 32 * wave;
    if (base < to) request(base, 0);

    bf16x8 q[NR][2 * kJ];  // in the order of the keys' dimensions
    int reach[NR];         // last position of row n
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        const int row = min(first + 16 * t + n, n_used - 1), token = row / rep, r = row - token * rep;
        reach[t] = (int)min(max(pos0 + token, (int64_t)-1), (int64_t)a.c.max_pos - 1);
        const uint16_t* src = a.q + (size_t)(u.rows.start + token) * a.q_stride + (size_t)(grp * rep + r) * D_used;
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
    const int key_row = 8 * (n >> 2) + (n & 3);
    uint32_t value_at[kDb];
#pragma unroll
    for (int d = 0; d < kDb; ++d)
        value_at[d] = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)ring + kTile + tile_place<D>(8 * g + (n >> 1), d) + 8 * (n & 1);
    // Waits for vector memory are written out: one that the compiler puts where a value is used would be one for the requests as well.
    float k_scales = 0.f, v_scales = 0.f;  // of the wavefront's next 64 tiles, one in each lane
    auto load_scales = [&]() __attribute__((always_inline)) {
        const int block = min(base / kBlock + W * lane, a.c.max_pos / kBlock - 1);
        k_scales = ks[block];
        v_scales = vs[block];
    };
    if (base < to) load_scales();
    __builtin_amdgcn_s_waitcnt(0x0F70);  // the scales, the queries and the first tile
    asm volatile("" : "+v"(k_scales), "+v"(v_scales)::"memory");
    for (int buf = 0, i = 0; base < to; base += 32 * W, buf ^= 1, ++i) {
        if (i && (i & 63) == 0) {
            load_scales();
            __builtin_amdgcn_s_waitcnt(0x0F70);
            asm volatile("" : "+v"(k_scales), "+v"(v_scales)::"memory");
        }
        const float c = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(k_scales), i & 63)) * a.scale;
        const float v_scale = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v_scales), i & 63)) * kValuesIn;
        if (base + 32 * W < to) {
            request(base + 32 * W, buf ^ 1);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0x0F70 | ((2 * kLoads) & 15) | ((2 * kLoads) >> 4 << 14));  // all but the requests just made
        } else {
            __builtin_amdgcn_s_waitcnt(0x0F70);
        }
        asm volatile("" ::: "memory");
        const uint8_t* kt = ring + 2 * buf * kTile;
        f32x4 s[NR][2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            // lane (n, g): dimensions 64 j + 16 g .. + 15 of position 8 (n / 4) + 4 b + n % 4
            bf16x8 kf[2 * kJ];
#pragma unroll
            for (int jj = 0; jj < kJ; ++jj) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(kt + tile_place<D>(key_row + 4 * b, 4 * jj + g));
                kf[2 * jj] = e4m3x8_to_bf16(x[0], x[1], 1.0f);
                kf[2 * jj + 1] = e4m3x8_to_bf16(x[2], x[3], 1.0f);
            }
#pragma unroll
            for (int t = 0; t < NR; ++t) {
                s[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int jj = 0; jj < 2 * kJ; ++jj) s[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[jj], q[t][jj], s[t][b], 0, 0, 0);
            }
        }
        const bool masked = base + 31 > reach_first;
        bf16x8 p[NR];
#pragma unroll
        for (int t = 0; t < NR; ++t) {
            Frag zero;
            zero.q = u32x4{0, 0, 0, 0};
            p[t] = zero.v;
            if (t && 16 * t >= rows_here) continue;
            float w[8], mx = -__builtin_inff();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = s[t][e >> 2][e & 3];
                if (masked && base + 8 * g + e > reach[t]) w[e] = -__builtin_inff();
                mx = fmaxf(mx, w[e]);
            }
            mx = fmaxf(mx * c, -3.0e38f);
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
                w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(w[e], c, -m[t]));
                l[t] += w[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) pair.u[e] = pack_bf16(w[2 * e], w[2 * e + 1]);
            p[t] = pair.v;
        }
        i32x2 codes[kDb];
        {
            uint32_t at[kDb];
#pragma unroll
            for (int d = 0; d < kDb; ++d) at[d] = value_at[d] + 2 * buf * kTile;
            read_values(codes, at);
        }
        bool odd = false;  // a value of a position that not every row attends to is NaN
        if (masked) {
            uint32_t nan = 0;
#pragma unroll
            for (int d = 0; d < kDb; ++d) nan |= (((uint32_t)codes[d][0] & 0x7f7f7f7fu) + 0x01010101u) | (((uint32_t)codes[d][1] & 0x7f7f7f7fu) + 0x01010101u);
            odd = __any((nan & 0x80808080u) != 0);
        }
        if (!odd) {
#pragma unroll
            for (int d = 0; d < kDb; ++d) {
                const bf16x8 v = e4m3x8_to_bf16((uint32_t)codes[d][0], (uint32_t)codes[d][1], v_scale);
#pragma unroll
                for (int t = 0; t < NR; ++t) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[t], o[t][d], 0, 0, 0);
            }
        } else {
            // A weight of zero times NaN is NaN, also where the row does not attend to the position -- a later token's, or one that nothing
            // has been stored in: NaN goes in as zero, and where a row attends to one -- a product of two masks of ones tells -- its result
            // becomes NaN.
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
                const uint32_t c0 = (uint32_t)codes[d][0], c1 = (uint32_t)codes[d][1];
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
    }

    // the wavefronts' results meet in LDS
    float* mo = reinterpret_cast<float*>(smem);                                  // [wave][kRows][kORow]
    float2* mstat = reinterpret_cast<float2*>(mo + W * kRows * kORow);  // [wave][kRows]
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        if (t && 16 * t >= rows_here) break;
        const int at = kRows * wave + 16 * t + n;
        const float sum = sum_quarters(sum_halves(l[t]));
#pragma unroll
        for (int d = 0; d < kDb; ++d) *reinterpret_cast<f32x4*>(mo + at * kORow + 16 * d + 4 * g) = o[t][d];
        if (g == 0) mstat[at] = make_float2(m[t], sum);
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kRows; t += 4 * W) {
        const int mine = t + (tid >> 4), row = first + mine;  // sixteen threads a row
        if (mine < kRows && row < n_used) {
            float w[W], top = -3.0e38f, all = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) top = fmaxf(top, mstat[kRows * i + mine].x);
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float2 st = mstat[kRows * i + mine];
                w[i] = __builtin_amdgcn_exp2f(st.x - top);
                all += w[i] * st.y;
            }
            const int token = row / rep;
            // a row that attends to nothing is zero
            const float inv = pos0 + token < 0 ? 0.f : kResultsOut / all;
            const size_t slot = ((size_t)unit * a.c.n_kv + grp) * kRows + mine;
            if (W == kCutWaves && (tid & 15) == 0) {
                if (cuts > 1) a.stat[slot] = make_float2(top, all);
                uint4* join = a.join + ((size_t)u.seq * a.max_new + token) * (a.c.n_kv * rep) + grp * rep + (row - token * rep);
                if (cut == 0) *reinterpret_cast<uint2*>(join) = make_uint2(unit, cuts_whole | (cuts > cuts_whole ? kRest : 0u));
                if (unit >= n_whole) join->z = unit;
            }
#pragma unroll
            for (int d = 4 * (tid & 15); d < D; d += 64) {
                if (d >= D_used) break;
                f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < W; ++i) x += *reinterpret_cast<const f32x4*>(mo + (kRows * i + mine) * kORow + d) * w[i];
                if (cuts > 1) {
                    *reinterpret_cast<f32x4*>(a.part + slot * D + d) = x;
                } else {
                    x *= inv;
                    uint16_t* dst = a.out + ((size_t)(u.rows.start + token) * a.c.n_kv * rep + (size_t)grp * rep + (row - token * rep)) * D_used + d;
                    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
                }
            }
        }
    }
}

// Joins the stretches of the rows that were cut: W wavefronts for each (row, query head), D / 4 lanes a stretch, eight stretches under way in
// each.  (60 rows of 118 stretches: 4.3 us; a wavefront for all of a row's, four under way: 235 of them took 32.)
template <int D, int NR, int W>
__global__ __launch_bounds__(256) void kv8_combine_kernel(Kv8AttArgs a) {
    constexpr int kRows = 16 * NR, kLanes = D / 4, kSide = 64 * W / kLanes;  // stretches side by side
    __shared__ __attribute__((aligned(16))) float sums[W > 1 ? kSide : 1][W > 1 ? D : 1];
    __shared__ float2 stats[W > 1 ? kSide : 1];
    const int n_heads = a.c.n_kv * a.rep, tid = threadIdx.x & (64 * W - 1);
    const uint32_t item = folded_block() * (4 / W) + (W > 1 ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6));
    const uint32_t h = item % (uint32_t)n_heads, row = item / (uint32_t)n_heads;  // row: sequence times max_new + token
    if (row >= (uint32_t)a.n_seq * (uint32_t)a.max_new) return;
    const uint4 join = a.join[(size_t)row * n_heads + h];
    const int seq = (int)(row / (uint32_t)a.max_new), token = (int)(row % (uint32_t)a.max_new);
    const SeqRows sr = seq_rows(a.row_start, a.pos0, seq, a.n_rows);
    if (token >= sr.count) return;  // nobody wrote the entry
    const uint32_t unit0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)join.x), wholes = (uint32_t)__builtin_amdgcn_readfirstlane((int)(join.y & ~kRest));
    const uint32_t has_rest = (uint32_t)__builtin_amdgcn_readfirstlane((int)(join.y >> 31)), rest = (uint32_t)__builtin_amdgcn_readfirstlane((int)join.z);
    const uint32_t cuts = wholes + has_rest;
    if (cuts <= 1 || unit0 >= a.bound || wholes > a.bound - unit0 || (has_rest && rest >= a.bound)) return;
    const int grp = (int)h / a.rep, local = (token * a.rep + ((int)h - grp * a.rep)) % kRows;
    auto slot_of = [&](uint32_t i) { return ((size_t)(i < wholes ? unit0 + i : rest) * a.c.n_kv + grp) * kRows + local; };
    const int side = tid / kLanes, d = 4 * (tid % kLanes);
    const bool used = d < a.c.head_dim;
    float top = -3.0e38f, all = 0.f;
    f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
    // a running maximum over eight stretches at a time, so that eight loads are under way
    for (uint32_t i = side; i < cuts; i += 8 * kSide) {
        float2 st[8];
        f32x4 v[8];
        float most = top;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t at = i + e * kSide;
            st[e] = make_float2(-3.0e38f, 0.f);
            v[e] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (at < cuts) {
                st[e] = a.stat[slot_of(at)];
                if (used) v[e] = *reinterpret_cast<const f32x4*>(a.part + slot_of(at) * D + d);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, st[e].x);
        const float f = __builtin_amdgcn_exp2f(top - most);
        top = most;
        all *= f;
        x *= f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float w = __builtin_amdgcn_exp2f(st[e].x - top);
            all += w * st[e].y;
            x += v[e] * w;
        }
    }
    if constexpr (W > 1) {
        *reinterpret_cast<f32x4*>(&sums[side][d]) = x;
        if (d == 0) stats[side] = make_float2(top, all);
        __syncthreads();
        if (side) return;
        const float own = top;
#pragma unroll
        for (int e = 1; e < kSide; ++e) top = fmaxf(top, stats[e].x);
        const float f = __builtin_amdgcn_exp2f(own - top);
        all *= f;
        x *= f;
#pragma unroll
        for (int e = 1; e < kSide; ++e) {
            const float w = __builtin_amdgcn_exp2f(stats[e].x - top);
            all += w * stats[e].y;
            x += *reinterpret_cast<const f32x4*>(&sums[e][d]) * w;
        }
    } else {
#pragma unroll
        for (int o = kLanes; o < 64; o <<= 1) {
            const float other = __shfl_xor(top, o), most = fmaxf(top, other), f = __builtin_amdgcn_exp2f(top - most);
            all *= f;
            all += __shfl_xor(all, o);
            x *= f;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], o);
            top = most;
        }
        if (side) return;
    }
    if (!used) return;
    // a row that attends to nothing is zero
    x *= (int64_t)sr.pos0 + token < 0 ? 0.f : kResultsOut / all;
    *reinterpret_cast<uint2*>(a.out + ((size_t)(sr.start + token) * n_heads + h) * a.c.head_dim + d) =
        make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
}

// Rows of a workgroup: as many of a sequence's as there can be, up to what the registers hold.
Kv8Plan kv8_plan(int n_heads, int n_kv, int head_dim, int n_seq, int max_new) {
    Kv8Plan p;
    const int rows = max_new * (n_heads / n_kv);
    p.dim = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256;
    p.nr = rows <= 16 || p.dim == 256 ? 1 : rows <= 32 || p.dim == 128 ? 2 : 4;
    const int kv = n_kv;
    const int by_lds = 163840 / kv8_lds(p.dim, p.nr, kCutWaves), by_registers = kv8_waves(p.dim, p.nr, kCutWaves);
    p.places = (std::min(by_lds, by_registers) * device_cu_count() + kv - 1) / kv;
    p.tiles = (rows + 16 * p.nr - 1) / (16 * p.nr);
    // units: sum of tiles * ceil(spans / stretch) <= sum of tiles * spans / stretch + sum of tiles
    p.bound = 2 * (uint32_t)p.places + (uint32_t)n_seq * (uint32_t)p.tiles;
    const size_t slots = (size_t)p.bound * kv * 16 * p.nr;
    p.stat_off = slots * p.dim * sizeof(float);
    p.join_off = (p.stat_off + slots * sizeof(float2) + 15) & ~(size_t)15;
    p.bytes = p.join_off + (size_t)n_seq * max_new * n_heads * sizeof(uint4);
    return p;
}

hipError_t launch_kv8_attention(const Kv8Args& c, const uint16_t* q, int64_t q_stride, int n_heads, const int32_t* row_start,
                                const int32_t* pos0, int n_seq, int n_rows, int max_new, uint16_t* out, void* ws, hipStream_t s) {
    if (c.head_dim < 16 || c.head_dim > 256 || c.head_dim % 16) return hipErrorInvalidValue;
    if (n_rows == 0 || n_seq == 0) return hipSuccess;
    const Kv8Plan p = kv8_plan(n_heads, c.n_kv, c.head_dim, n_seq, max_new);
    const int rep = n_heads / c.n_kv;
    Kv8AttArgs a = {c, q, q_stride, row_start, pos0, n_seq, n_rows, max_new, rep, p.places, p.bound,
                    (float)(1.4426950408889634 / sqrt((double)c.head_dim)), out, static_cast<float*>(ws),
                    reinterpret_cast<float2*>(static_cast<uint8_t*>(ws) + p.stat_off),
                    reinterpret_cast<uint4*>(static_cast<uint8_t*>(ws) + p.join_off)};
    // Units that these rows can have (a workgroup that finds nothing to do is not free: a thousand of them are 3 us): their row tiles, each
    // in no more stretches than the cache has spans; no more than run at once where stretches are made for that.
    const uint64_t by_rows = (uint64_t)n_rows * rep / (16 * p.nr) + (uint64_t)(n_seq < n_rows ? n_seq : n_rows), by_seq = (uint64_t)n_seq * p.tiles;
    const uint64_t tiles = by_rows < by_seq ? by_rows : by_seq, spans = (uint64_t)((c.max_pos + kAttSpan - 1) / kAttSpan);
    const uint64_t most = 2 * tiles <= (uint64_t)p.places ? (uint64_t)p.places : 2 * (uint64_t)p.places + tiles;
    // A cache of up to 1024 positions is four steps of eight wavefronts at most, less than the second launch that joins what was cut; up to 2048
    // it is where the workgroups fill a quarter of the chip.  (Whole / cut, us: 24 query heads over 8, one token against 429 positions
    // 6.8 / 8.3, against 1000 9.0 / 8.4, against 1900 12.5 / 8.5; 32 drafts of five against 500 10.1 / 15.4, against 1800 25 / 31; 64 against 0 to
    // 1900 23 / 30; eight chunks of 64 against 1800 35 / 45.  Far more workgroups than places: 32 chunks against 500 59 / 51.)
    const uint64_t wholes = tiles * (uint64_t)c.n_kv, cus = (uint64_t)device_cu_count();
    const bool whole = p.dim <= 128 && wholes <= 4 * cus && (c.max_pos <= 1024 || (c.max_pos <= 2048 && 4 * wholes >= cus));
    const dim3 grid = folded_grid((whole ? tiles : tiles * spans < most ? tiles * spans : most) * c.n_kv);
    // (row, query head) pairs; few of them have many stretches each: four wavefronts
    const uint64_t pairs = (uint64_t)n_seq * max_new * n_heads;
    const bool wide = pairs <= 8 * cus;
    const dim3 join = folded_grid(wide ? pairs : (pairs + 3) / 4);
#define SD2_KV8_ATTEND(DIM, R, W)                                                                                                \
    do {                                                                                                                         \
        static std::atomic<uint64_t> done{0};                                                                                    \
        const hipError_t e = allow_lds(reinterpret_cast<const void*>(&kv8_attention_kernel<DIM, R, W>), kv8_lds(DIM, R, W), done); \
        if (e != hipSuccess) return e;                                                                                           \
        hipLaunchKernelGGL((kv8_attention_kernel<DIM, R, W>), grid, dim3(64 * W), kv8_lds(DIM, R, W), s, a);                     \
    } while (0)
#define SD2_KV8_CUT(DIM, R)                                                                                               \
    do {                                                                                                                  \
        SD2_KV8_ATTEND(DIM, R, kCutWaves);                                                                                \
        if (c.max_pos > kAttSpan && wide) hipLaunchKernelGGL((kv8_combine_kernel<DIM, R, 4>), join, dim3(256), 0, s, a);  \
        if (c.max_pos > kAttSpan && !wide) hipLaunchKernelGGL((kv8_combine_kernel<DIM, R, 1>), join, dim3(256), 0, s, a); \
    } while (0)
#define SD2_KV8(DIM, R)                                            \
    if (p.dim == DIM && p.nr == R) {                               \
        if (whole) SD2_KV8_ATTEND(DIM, R, kWholeWaves);            \
        else SD2_KV8_CUT(DIM, R);                                  \
    }
    SD2_KV8(64, 1) SD2_KV8(64, 2) SD2_KV8(64, 4)
    SD2_KV8(128, 1) SD2_KV8(128, 2)
    if (p.dim == 256) SD2_KV8_CUT(256, 1);
#undef SD2_KV8
#undef SD2_KV8_CUT
#undef SD2_KV8_ATTEND
    return hipGetLastError();
}

}  // namespace sd2
