// Packed rows of several sequences: which sequence a unit of work belongs to (device side, not part of the C ABI).
//
// Row offsets and positions live on the device, so that a captured call serves requests of any length: every wavefront
// finds its own work by a prefix sum over the sequences.  Offsets are clamped to the rows that the call has, and whatever
// they hold, no kernel reads or writes outside its buffers.
#pragma once
#include "sd2_device.h"

namespace sd2 {

struct SeqRows {
    int start, count;
};

__device__ __forceinline__ SeqRows seq_rows(const int32_t* __restrict__ row_start, int b, int n_rows) {
    const int lo = min(max(row_start[b], 0), n_rows), hi = min(max(row_start[b + 1], lo), n_rows);
    return {lo, hi - lo};
}

struct SeqUnit {
    int seq;         // -1: past the last unit
    uint32_t index;  // unit inside the sequence
    uint32_t before; // units of the sequences in front of it
};

// The sequence that owns `unit`, where sequence b has count(b) units: 64 sequences a step, one in each lane.  All lanes of
// the wavefront take part; the result is the same in all of them.
template <typename F>
__device__ __forceinline__ SeqUnit find_unit(uint32_t unit, int n_seq, F&& count) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int base = 0; base < n_seq; base += 64) {
        const int b = base + lane;
        const uint32_t own = b < n_seq ? count(b) : 0u, incl = wave_incl_scan(own);
        const uint64_t past = __ballot(before + incl > unit);
        if (past) {
            const int at = __builtin_ctzll(past);
            const uint32_t first = before + (uint32_t)__builtin_amdgcn_readlane((int)(incl - own), at);
            return {__builtin_amdgcn_readfirstlane(base + at), unit - first, first};
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
    }
    return {-1, 0, before};
}

// the sum of count(b) over all sequences
template <typename F>
__device__ __forceinline__ uint64_t total_units(int n_seq, F&& count) {
    uint64_t sum = 0;
    for (int base = 0; base < n_seq; base += 64) {
        const int b = base + (threadIdx.x & 63);
        sum += (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_scan(b < n_seq ? count(b) : 0u), 63);
    }
    return sum;
}

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

}  // namespace sd2
