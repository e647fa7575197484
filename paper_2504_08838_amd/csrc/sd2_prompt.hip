// libsd2 -- causal attention over whole prompts, packed one behind the other (gfx950).
//
// o_i = sum_{j <= i} exp(q_i k_j / sqrt(D) - m_i) v_j / sum_{j <= i} exp(q_i k_j / sqrt(D) - m_i), in one pass over the positions with
// a running maximum m_i; products on the matrix cores (bf16 in, fp32 sums), maxima and sums in fp32.  Weights are rounded to bf16 for
// the second product: at most 2^-8 of a weight, as for the result itself (against 64 bits 0.0021 of the result's norm, where the rounding
// of the result alone is 0.0016).
//
// The rows of a workgroup are (token, query head of the group) pairs in that order: what is read of keys and values serves the whole
// group, and the diagonal that is computed and masked is a third as wide with three heads a group.  Scores come out transposed
// (positions by rows), so that a lane holds runs of eight positions of one row -- positions are dealt to the rows of the first product
// such that they follow one another -- and these are the second product's operand as they stand: weights never leave the registers.
// Keys and values go from memory into LDS without passing through registers, a tile ahead; their 16-byte pieces are turned within a row
// by the row's number, which spreads the reads over the banks (no conflicts counted).
//
// What bounds it: on long prompts matrix cores and vector ALU in turn, at a clock that the power they draw sets -- 8192 tokens, 24 query heads
// over 8 of 128 dimensions: 396 us, 1040 TFLOP/s, where a library product of 8192^3 reaches 1245; the matrix cores are busy 52 % of 768 000
// cycles, the vector ALU about as long, at 1.9 of 2.4 GHz.  Scores of the next tile made beside the weights of this one: 8 % fewer cycles at a
// clock 5 % lower, 3 % less time here and 2 to 5 % more for shorter prompts; not kept.  With heads of 64 dimensions the vector instructions
// count twice (3001 + 1 + 2500 + 777 tokens, 32 heads: 80 us, 805 TFLOP/s): of six a score, one is the exponential.  Other head sizes do the
// work of 128 or 256 (3000 tokens, 24 heads over 8: 65 us with heads of 80, 70 with 128; 301 with 144, 234 with 256, where a SIMD has one
// wavefront and a tile serves 32 rows).  On short prompts the chain of steps of the last rows, 1.1 us for 64 positions: 300 tokens 8.2 us,
// 37 tokens 5.9 us, of which a launch that does nothing has 2.
#include <type_traits>

#include "sd2_internal.h"
#include "sd2_rows.h"

namespace sd2 {

// A workgroup is G groups of 32 rows times T teams: a team is a wavefront for each group, and the teams take turns with the tiles of
// positions.  T teams take a T-th of the steps one after the other, and their results meet in LDS.  Where rows alone do not fill the chip,
// what counts is the chain of steps.
constexpr int prompt_tile(int g) { return g == 1 ? 32 : 64; }
// Keys and values of each team's tile.  Teams of several wavefronts have two buffers, as all of them must be through with one before it can
// be filled again; a wavefront alone asks for its next keys when the scores are there and for its next values when these have been read.
constexpr int prompt_tiles(int dim, int g, int t) { return t * (g == 1 ? 1 : 2) * 2 * prompt_tile(g) * dim * 2; }
constexpr int prompt_meeting(int dim, int g, int t) { return t > 1 ? t * 32 * g * (dim + 4 + 2) * 4 : 0; }  // rows of dim + 4 sums, maxima and sums of weights
constexpr int prompt_lds(int dim, int g, int t) {
    return prompt_tiles(dim, g, t) > prompt_meeting(dim, g, t) ? prompt_tiles(dim, g, t) : prompt_meeting(dim, g, t);
}

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t q_stride, kv_stride;
    const int32_t* row_start;
    int n_seq, n_rows, n_kv, rep, head_dim;
    float scale;  // log2(e) / sqrt(D)
    uint16_t* out;
};

// byte offset of 16-byte piece c of row r in a tile: keys are read sixteen rows at a time, values four rows of four pieces
template <int D>
__device__ __forceinline__ int key_place(int r, int c) {
    return 16 * (r * (D / 8) + (c ^ (D == 64 ? (r >> 1) & 7 : r & 15)));
}
template <int D>
__device__ __forceinline__ int val_place(int r, int c) {
    return 16 * (r * (D / 8) + (c ^ (D == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3))));
}

// 16 bytes from base + offset of every lane to lds + 16 * lane.  As assembly, because the compiler waits for all such requests in front of
// every transposing read of LDS: it cannot tell the buffers apart.  Nothing returns to registers; whoever reads the bytes waits first.
// (m0 is never allocated, of which the compiler warns; named, it is known to be written.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits for all but the last N vector memory operations, and for all operations on LDS; nothing moves across them.
template <int N>
__device__ __forceinline__ void wait_memory() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4 << 14));
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" ::: "memory");
}

template <int D, int G, int T>
__global__ __launch_bounds__(64 * G * T, D < 256 ? 2 : 1) void prompt_attention_kernel(PromptArgs a) {
    constexpr int kTile = prompt_tile(G), kRb = kTile / 32, kSteps = D / 16, kDb = D / 32, kBytes = kTile * D * 2, kRows = 32 * G;
    constexpr int kCalls = kBytes / (1024 * G);  // requests of a wavefront for a tile of keys (and of values)
    constexpr int kAhead = kTile * T;            // positions from a team's tile to its next
    extern __shared__ __attribute__((aligned(16))) uint8_t whole[];  // [team][kBuffers][keys, values][kBytes]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const uint32_t block = folded_block(), n_kv = (uint32_t)a.n_kv, unit = block / n_kv;
    const int grp = (int)(block - unit * n_kv), rep = a.rep, hd = a.head_dim;
    auto tiles_of = [&](const SeqRows& r) { return (uint32_t)(r.count * rep + kRows - 1) / kRows; };
    const SeqUnit u = Sequences(a.row_start, nullptr, a.n_seq, a.n_rows).find_largest_first(unit, tiles_of);
    if (u.seq < 0) return;
    const SeqRows sr = u.rows;
    const int n_used = sr.count * rep;
    const int team = wave / G, member = wave % G;
    constexpr int kBuffers = G == 1 ? 1 : 2;
    uint8_t* smem = whole + team * kBuffers * 2 * kBytes;
    const int first = kRows * (int)u.index, wave_first = first + 32 * member;
    const int n_pos = min(first + kRows - 1, n_used - 1) / rep + 1;               // positions that the workgroup's rows attend to
    // positions that the last of the wavefront's own rows attends to (no rows: none)
    const int wave_pos = wave_first < n_used ? min(wave_first + 31, n_used - 1) / rep + 1 : 0;
    // Last position of the team's tiles in the steps that no mask touches, steps in which all rows attend to all positions.  Where steps have
    // barriers, these are steps of all teams: the workgroup's wavefronts go from the one loop into the other together.
    const int low = first / rep - (G == 1 ? 0 : kTile * (T - 1 - team));
    const uint16_t* kg = a.k + (size_t)sr.start * a.kv_stride + (size_t)grp * hd;
    const uint16_t* vg = a.v + (size_t)sr.start * a.kv_stride + (size_t)grp * hd;

    if (hd < D) {  // dimensions that the heads do not have: zero, and never written again
        for (int i = tid; i < prompt_tiles(D, G, T) / 16; i += 64 * G * T) reinterpret_cast<u32x4*>(whole)[i] = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
    // A tile's requests of this lane: rows r0, r0 + kStep, ..., the turned piece of each, as byte offsets from the tile's first row.
    constexpr int kStep = 64 * G / (D / 8);
    const int r0 = (64 * member + lane) / (D / 8), c0 = lane % (D / 8);
    const uint32_t row_bytes = 2 * (uint32_t)a.kv_stride;
    auto request = [&](int base, int buf, auto which) __attribute__((always_inline)) {  // 1: keys, 2: values, 3: both
        constexpr bool keys = decltype(which)::value & 1, values = decltype(which)::value & 2;
        const uint16_t* kb = kg + (size_t)base * a.kv_stride;
        const uint16_t* vb = vg + (size_t)base * a.kv_stride;
        const uint32_t to_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)(smem + 2 * buf * kBytes + 1024 * member);
        auto pieces = [&](bool inside, bool all) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kCalls; ++i) {
                const int r = r0 + kStep * i;
                const uint32_t kc = (uint32_t)key_place<D>(r, c0) % (2 * D), vc = (uint32_t)val_place<D>(r, c0) % (2 * D);
                const uint32_t at = (inside ? (uint32_t)r : (uint32_t)min(r, sr.count - 1 - base)) * row_bytes;  // no row past the sequence's last
                if (keys && (all || kc < 2u * hd)) load_to_lds(kb, at + kc, to_lds + 1024 * G * i);
                if (values && (all || vc < 2u * hd)) load_to_lds(vb, at + vc, to_lds + kBytes + 1024 * G * i);
            }
        };
        if (hd == D && base + kTile <= sr.count) pieces(true, true);
        else pieces(false, false);
    };
    using Keys = std::integral_constant<int, 1>;
    using Values = std::integral_constant<int, 2>;
    using Both = std::integral_constant<int, 3>;
    int base = kTile * team;
    if (T == 1 || base < n_pos) {
        if (G == 1) {
            request(base, 0, Keys());
            request(base, 0, Values());
        } else {
            request(base, 0, Both());
        }
    }

    // operand of the scores: row n, dimensions 16 step + 8 h .. + 7 (rows past the last repeat it; never written)
    const int row = min(wave_first + n, n_used - 1), token = row / rep, head = grp * rep + (row - token * rep);
    bf16x8 q[kSteps];
    {
        const uint16_t* src = a.q + (size_t)(sr.start + token) * a.q_stride + (size_t)head * hd + 8 * h;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            Frag f;
            f.q = u32x4{0, 0, 0, 0};
            if (16 * i < hd) f.q = *reinterpret_cast<const u32x4*>(src + 16 * i);
            q[i] = f.v;
        }
    }
    float m = -3.0e38f, l = 0.f;
    f32x16 o[kDb];  // dimension 32 db + 8 (i / 4) + 4 h + i % 4 of row n
#pragma unroll
    for (int d = 0; d < kDb; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

    // where in a tile the lane reads
    const int key_row = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);
    const int val_row = 8 * h + ((lane & 15) >> 2), val_piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), val_byte = 8 * (lane & 1);

    int buf = 0, odd_from = 0x7fffffff;
    auto tile = [&](int base, auto is_masked) __attribute__((always_inline)) {
        constexpr bool masked = decltype(is_masked)::value;
        const uint8_t* kt = smem + 2 * buf * kBytes;
        const uint8_t* vt = kt + kBytes;
        f32x16 s[kRb];
#pragma unroll
        for (int rb = 0; rb < kRb; ++rb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[rb][i] = 0.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int rb = 0; rb < kRb; ++rb) {
                const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kt + key_place<D>(32 * rb + key_row, 2 * i + h));
                s[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[i], s[rb], 0, 0, 0);
            }
        // six reads of LDS under way in front of each product (8192 tokens: 399 us; as the compiler orders them, two: 409)
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int i = 0; i < kSteps * kRb; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        if constexpr (G == 1) {
            if (base + kAhead < n_pos) {
                wait_lds();  // the keys have been read
                request(base + kAhead, 0, Keys());
            }
        }
        if (masked) {
#pragma unroll
            for (int rb = 0; rb < kRb; ++rb)
#pragma unroll
                for (int i = 0; i < 16; ++i)  // position 32 rb + 16 (i / 8) + 8 h + i % 8
                    if (base + 32 * rb + 16 * (i >> 3) + 8 * h + (i & 7) > token) s[rb][i] = -__builtin_inff();
        }
        float mx = s[0][0];
#pragma unroll
        for (int rb = 0; rb < kRb; ++rb)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[rb][i]);
        mx *= a.scale;
        // The maximum follows only where a weight could grow past 2^8: sums of weights up to that are as exact as those below 1.
        if (__any(mx > m + 8.f)) {
            const float top = fmaxf(m, max_halves(mx)), f = __builtin_amdgcn_exp2f(m - top);
            m = top;
            l *= f;
#pragma unroll
            for (int d = 0; d < kDb; ++d) o[d] *= f;
        }
        if constexpr (G == 1) {  // this tile's values: all but the keys just asked for
            if (base + kAhead < n_pos) wait_memory<kCalls>();
            else wait_memory<0>();
        }
        if (masked) {
            // A weight of zero times an infinity or NaN is NaN, also where the row does not attend to the position: from the first tile
            // on that holds such a value and is not attended to by all rows, values are added at the end, one position after the other.
            uint32_t largest = 0;
#pragma unroll
            for (int i = 0; i < kBytes / 1024; ++i) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(vt + 1024 * i + 16 * lane);
#pragma unroll
                for (int e = 0; e < 4; ++e) largest = max(largest, max((x[e] << 1) & 0xfffe0000u, (x[e] & 0x7fffu) << 17));
            }
            if (__any(largest >= 0xff000000u)) odd_from = min(odd_from, base);
        }
        // operand of eight positions (32 rb + 16 j + 8 h ..) of dimension 32 db + n: two transposing reads of four rows
        auto values = [&](int d, int rb, int j) __attribute__((always_inline)) {
            Frag f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 32 * rb + 16 * j + 4 * e + val_row;
                const auto* src = (const __attribute__((address_space(3))) uint8_t*)vt + val_place<D>(r, 4 * d + val_piece) + val_byte;
                const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)src);
                reinterpret_cast<s16x4*>(&f)[e] = x;
            }
            return f;
        };
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int rb = 0; rb < kRb; ++rb)
#pragma unroll
            for (int j = 0; j < 2; ++j) {  // positions 32 rb + 16 j + 8 h .. + 7
                float w[8];
                Frag f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][8 * j + e], a.scale, -m));
                    sum[e & 1] += w[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) f.u[e] = pack_bf16(w[2 * e], w[2 * e + 1]);
                if (masked && odd_from <= base) continue;
#pragma unroll
                for (int d = 0; d < kDb; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values(d, rb, j).v, f.v, o[d], 0, 0, 0);
            }
        l += sum[0] + sum[1];
        if constexpr (G == 1) {
            if (base + kAhead < n_pos) {
                wait_lds();  // the values have been read
                request(base + kAhead, 0, Values());
            }
        }
    };
    auto next = [&]() __attribute__((always_inline)) {
        if constexpr (G == 1) {
            wait_memory<kCalls>();  // the keys: all but the values behind them
        } else {
            wait_memory<0>();  // this wavefront's requests
            __syncthreads();  // everybody's: the tile is there, and nobody reads the other buffer
            if (base + kAhead < n_pos) request(base + kAhead, buf ^ 1, Both());
        }
    };
    // the queries with the first tile: a wait of the compiler's for them would be one for what is asked for behind them as well
    if (G == 1) wait_memory<0>();
    const int last = n_pos + kTile * team;           // as many steps for every team
    for (; base < last && base + kTile - 1 <= low; base += kAhead, buf ^= kBuffers - 1) {
        next();
        if (G == 1 || wave_pos > 0) tile(base, std::false_type());
    }
    for (; base < last; base += kAhead, buf ^= kBuffers - 1) {
        next();
        if (base < wave_pos) tile(base, std::true_type());
    }
#pragma unroll 1
    for (int pos = odd_from; pos <= token; ++pos) {
        if (T > 1 && pos / kTile % T != team) continue;
        const uint16_t* key = kg + (size_t)pos * a.kv_stride;
        const uint16_t* query = a.q + (size_t)(sr.start + token) * a.q_stride + (size_t)head * hd;
        float dot = 0.f;
#pragma unroll 1
        for (int d = 0; d < hd; ++d) dot += bf16_to_f32(query[d]) * bf16_to_f32(key[d]);
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(dot, a.scale, -m));
        const uint16_t* src = vg + (size_t)pos * a.kv_stride + 4 * h;
#pragma unroll
        for (int d = 0; d < kDb; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (32 * d + 8 * i >= hd) continue;
                const uint2 x = *reinterpret_cast<const uint2*>(src + 32 * d + 8 * i);
                o[d][4 * i] += w * __uint_as_float(x.x << 16);
                o[d][4 * i + 1] += w * __uint_as_float(x.x & 0xffff0000u);
                o[d][4 * i + 2] += w * __uint_as_float(x.y << 16);
                o[d][4 * i + 3] += w * __uint_as_float(x.y & 0xffff0000u);
            }
    }
    l = sum_halves(l);
    if constexpr (T > 1) {  // the teams' results meet in LDS, 2 T threads a row
        constexpr int kORow = D + 4;
        float* sums = reinterpret_cast<float*>(whole);                        // [team][kRows][kORow]
        float2* stats = reinterpret_cast<float2*>(sums + T * kRows * kORow);  // [team][kRows]
        __syncthreads();
        const int at = team * kRows + 32 * member + n;
#pragma unroll
        for (int d = 0; d < kDb; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(sums + at * kORow + 32 * d + 8 * i + 4 * h) = f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
        if (h == 0) stats[at] = make_float2(m, l);
        __syncthreads();
        const int mine = tid / (2 * T), part = tid % (2 * T), row_of = first + mine;
        if (row_of >= n_used) return;
        float w[T], top = -3.0e38f, all = 0.f;
#pragma unroll
        for (int t = 0; t < T; ++t) top = fmaxf(top, stats[t * kRows + mine].x);
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const float2 st = stats[t * kRows + mine];
            w[t] = __builtin_amdgcn_exp2f(st.x - top);
            all += w[t] * st.y;
        }
        const float inv = 1.0f / all;
        const int own = row_of / rep;
        uint16_t* dst = a.out + ((size_t)(sr.start + own) * a.n_kv * rep + grp * rep + (row_of - own * rep)) * hd;
#pragma unroll
        for (int d = 4 * part; d < D; d += 8 * T) {
            if (d >= hd) break;
            f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < T; ++t) x += *reinterpret_cast<const f32x4*>(sums + (t * kRows + mine) * kORow + d) * w[t];
            x *= inv;
            *reinterpret_cast<uint2*>(dst + d) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
        }
        return;
    }
    if (wave_first + n >= n_used) return;
    const float inv = 1.0f / l;
    uint16_t* dst = a.out + ((size_t)(sr.start + token) * a.n_kv * rep + head) * hd + 4 * h;
#pragma unroll
    for (int d = 0; d < kDb; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (32 * d + 8 * i < hd)
                *reinterpret_cast<uint2*>(dst + 32 * d + 8 * i) = make_uint2(pack_bf16(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                                                                              pack_bf16(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv));
}

hipError_t launch_prompt_attention(const uint16_t* q, const uint16_t* k, const uint16_t* v, int64_t q_stride, int64_t kv_stride,
                                   const int32_t* row_start, int n_seq, int n_rows, int n_heads, int n_kv, int head_dim, uint16_t* out,
                                   hipStream_t s) {
    if (head_dim < 16 || head_dim > 256 || head_dim % 16) return hipErrorInvalidValue;
    if (n_rows == 0 || n_seq == 0) return hipSuccess;
    const int rep = n_heads / n_kv;
    const PromptArgs a = {q, k, v, q_stride, kv_stride, row_start, n_seq, n_rows, n_kv, rep, head_dim,
                          (float)(1.4426950408889634 / sqrt((double)head_dim)), out};
    const int64_t seqs = n_seq < n_rows ? n_seq : n_rows, cus = device_cu_count();
    auto units = [&](int g) { return ((int64_t)n_rows * rep / (32 * g) + seqs) * n_kv; };  // each of up to 512 threads
#define SD2_PROMPT(DIM, G, T)                                                                                                        \
    do {                                                                                                                             \
        static std::atomic<uint64_t> done{0};                                                                                        \
        const hipError_t e = allow_lds(reinterpret_cast<const void*>(&prompt_attention_kernel<DIM, G, T>), prompt_lds(DIM, G, T), done); \
        if (e != hipSuccess) return e;                                                                                               \
        hipLaunchKernelGGL((prompt_attention_kernel<DIM, G, T>), folded_grid(units(G)), dim3(64 * G * T), prompt_lds(DIM, G, T), s, a); \
    } while (0)
    // Which kernel, by what the host knows (us, 24 query heads over 8 of 128 dimensions unless said otherwise; 32 rows a workgroup and four
    // teams / 128 rows and two teams / 128 rows and one team):
    //   300 tokens 8.1 / 10.9 / 11.5, 600 tokens 10.9 / 15.7 / 16.9, 2000 tokens with 12 heads over 2 28.3 / 33.4 / 39.0,
    //   1024 tokens 21.6 / 21.6 / 23.9, 1500 tokens - / 29.0 / 34.1, eight prompts of 60 to 120 tokens 12.3 / 9.7 / 9.5: short prompts
    //   have few steps to share, and more workgroups than run at once are not worth it there.
    const bool few = units(1) <= 2 * cus || (units(1) <= 4 * cus && n_rows / seqs >= 256), some = units(4) <= 2 * cus;
    if (head_dim <= 64 && few) SD2_PROMPT(64, 1, 4);
    else if (head_dim <= 64 && some) SD2_PROMPT(64, 4, 2);
    else if (head_dim <= 64) SD2_PROMPT(64, 4, 1);
    else if (head_dim <= 128 && few) SD2_PROMPT(128, 1, 4);
    else if (head_dim <= 128 && some) SD2_PROMPT(128, 4, 2);
    else if (head_dim <= 128) SD2_PROMPT(128, 4, 1);
    else SD2_PROMPT(256, 1, 4);  // one tile of 128 rows leaves the registers no room for a second wavefront (6000 tokens: 256 / 281 us)
#undef SD2_PROMPT
    return hipGetLastError();
}

}  // namespace sd2
