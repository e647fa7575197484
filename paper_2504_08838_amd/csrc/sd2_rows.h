// Packed rows of several sequences: which sequence a unit of work belongs to (device side, not part of the C ABI).
//
// Row offsets and positions live on the device, so that a captured call serves requests of any length: every wavefront
// finds its own work by a prefix sum over the sequences.  Offsets are clamped to the rows that the call has, and whatever
// they hold, no kernel reads or writes outside its buffers.
#pragma once
#include <atomic>

#include "sd2_device.h"

namespace sd2 {

// Lets a kernel have more than 64 KiB of LDS.  `done`: the devices (bit by number) that have been told so for this kernel.
inline hipError_t allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
    if (bytes <= 65536) return hipSuccess;
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = (uint64_t)1 << (device & 63);
    if (done.load(std::memory_order_acquire) & bit) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

// Grids of any number of workgroups: HIP launches fewer than 2^32 threads in a dimension, so those past 2^22 go into a second one.  The
// last row of a folded grid may be longer than what is left: kernels end workgroups without work by themselves.
constexpr int kGridFold = 22;
inline dim3 folded_grid(uint64_t workgroups) {
    const uint64_t row = (uint64_t)1 << kGridFold;
    return workgroups <= row ? dim3((unsigned)workgroups) : dim3((unsigned)row, (unsigned)((workgroups + row - 1) >> kGridFold));
}
__device__ __forceinline__ uint32_t folded_block() { return blockIdx.y << kGridFold | blockIdx.x; }

struct SeqRows {
    int start, count, pos0;  // first row, rows, position of the first row
};

// pos0 may be null: prompts
__device__ __forceinline__ SeqRows seq_rows(const int32_t* __restrict__ row_start, const int32_t* __restrict__ pos0, int b, int n_rows) {
    const int from = row_start[b], to = row_start[b + 1], first = pos0 ? pos0[b] : 0;
    const int lo = min(max(from, 0), n_rows), hi = min(max(to, lo), n_rows);
    return {lo, hi - lo, first};
}

struct SeqUnit {
    int seq;         // -1: past the last unit
    uint32_t index;  // unit inside the sequence
    SeqRows rows;
};

// The sequences as a wavefront goes through them, 64 a step, one in each lane; the first 64 are loaded once.  All lanes take part, and
// what the functions return is the same in all of them.
struct Sequences {
    const int32_t *row_start, *pos0;
    int n_seq, n_rows;
    SeqRows first;

    __device__ __forceinline__ Sequences(const int32_t* rs, const int32_t* p0, int n, int rows)
        : row_start(rs), pos0(p0), n_seq(n), n_rows(rows), first(at(0)) {}

    __device__ __forceinline__ SeqRows at(int base) const {
        const int b = base + (threadIdx.x & 63);
        return b < n_seq ? seq_rows(row_start, pos0, b, n_rows) : SeqRows{0, 0, 0};
    }

    // the sum of count(sequence) over all sequences; count of no rows is zero
    template <typename F>
    __device__ __forceinline__ uint64_t total(F&& count) const {
        uint64_t sum = 0;
        for (int base = 0; base < n_seq; base += 64)
            sum += (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_scan(count(base ? at(base) : first)), 63);
        return sum;
    }

    // the sequence that owns `unit`
    template <typename F>
    __device__ __forceinline__ SeqUnit find(uint32_t unit, F&& count) const {
        uint32_t before = 0;
        for (int base = 0; base < n_seq; base += 64) {
            const SeqRows own = base ? at(base) : first;
            const uint32_t n = count(own), incl = wave_incl_scan(n);
            const uint64_t past = __ballot(before + incl > unit);
            if (past) {
                const int lane = __builtin_ctzll(past);
                const SeqRows rows = {__builtin_amdgcn_readlane(own.start, lane), __builtin_amdgcn_readlane(own.count, lane),
                                      __builtin_amdgcn_readlane(own.pos0, lane)};
                return {__builtin_amdgcn_readfirstlane(base + lane), unit - before - (uint32_t)__builtin_amdgcn_readlane((int)(incl - n), lane), rows};
            }
            before += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
        }
        return {-1, 0, {0, 0, 0}};
    }

    // The same units in another order: by their number inside their sequence, the largest first, so that what lasts longest starts first.
    // (For up to 64 sequences; with more, sequence by sequence, as find has them, the largest first in each.)
    template <typename F>
    __device__ __forceinline__ SeqUnit find_largest_first(uint32_t unit, F&& count) const {
        if (n_seq == 1 || n_seq > 64) {
            SeqUnit u = find(unit, count);
            u.index = count(u.rows) - 1 - u.index;
            return u;
        }
        const uint32_t own = count(first);
        // units whose number is at least `level`
        auto from = [&](uint32_t level) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_scan(own > level ? own - level : 0u), 63); };
        if (unit >= from(0)) return {-1, 0, {0, 0, 0}};
        uint32_t level = 0, past = 1;
        while (from(past) > unit) {
            level = past;
            past *= 2;
        }
        while (past - level > 1) {  // from(level) > unit >= from(past)
            const uint32_t mid = (level + past) / 2;
            if (from(mid) > unit) level = mid;
            else past = mid;
        }
        const uint32_t incl = wave_incl_scan(own > level ? 1u : 0u);
        const int lane = __builtin_ctzll(__ballot(incl > unit - from(past)));
        return {lane, level, {__builtin_amdgcn_readlane(first.start, lane), __builtin_amdgcn_readlane(first.count, lane), 0}};
    }
};

// the larger (the sum) of two lanes 32 apart, in both
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// of two lanes 16 apart
__device__ __forceinline__ float max_quarters(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_quarters(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// the largest over all lanes, in all of them
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#define SD2_ROW_MAX(ctrl) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xf, 0xf, true))
    SD2_ROW_MAX(0x121);  // row_ror:1
    SD2_ROW_MAX(0x122);  // row_ror:2
    SD2_ROW_MAX(0x124);  // row_ror:4
    SD2_ROW_MAX(0x128);  // row_ror:8
#undef SD2_ROW_MAX
    const auto r16 = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(r16[0], r16[1]);
    const auto r32 = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max(r32[0], r32[1]);
}

}  // namespace sd2
