// Lane moves, wave reductions and the register form of the rotation, shared by the attention kernels.
#pragma once

#include "common.hpp"
#include "plan.hpp"

namespace kvarn {
namespace {

__device__ __forceinline__ int dpp_x1(int v) { return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true); }
__device__ __forceinline__ int dpp_x2(int v) { return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true); }
__device__ __forceinline__ int dpp_half_mirror(int v) { return __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true); }
__device__ __forceinline__ int dpp_mirror(int v) { return __builtin_amdgcn_mov_dpp(v, 0x140, 0xF, 0xF, true); }
__device__ __forceinline__ float fdpp_x1(float v) { return __int_as_float(dpp_x1(__float_as_int(v))); }
__device__ __forceinline__ float fdpp_x2(float v) { return __int_as_float(dpp_x2(__float_as_int(v))); }
__device__ __forceinline__ float fdpp_half_mirror(float v) { return __int_as_float(dpp_half_mirror(__float_as_int(v))); }
__device__ __forceinline__ float fdpp_mirror(float v) { return __int_as_float(dpp_mirror(__float_as_int(v))); }
// The 128-point butterflies (unnormalized) over a wave's lanes, lane l holding channels 2l, 2l + 1:
// stride 1 in the lane, then lane partners l ^ 1, 2, 4, ..., 32, all by lane moves (partner ^4 is
// the half-row mirror of the quad-reversed value, ^8 a rotation of the row by 8).
template <int M>
__device__ __forceinline__ float lane_xor(float v, int l) {
    if constexpr (M == 1) return fdpp_x1(v);
    else if constexpr (M == 2) return fdpp_x2(v);
    else if constexpr (M == 4) return fdpp_half_mirror(__int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x1B, 0xF, 0xF, true)));
    else if constexpr (M == 8) return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128, 0xF, 0xF, true));
    else if constexpr (M == 16) {
        const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return __uint_as_float(((l >> 4) & 1) ? x[0] : x[1]);
    } else {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return __uint_as_float(l < 32 ? x[1] : x[0]);
    }
}
template <int M>
__device__ __forceinline__ void fwht_stage(float (&x)[2], int l) {
    const bool upper = (l & M) != 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const float p = lane_xor<M>(x[e], l);
        x[e] = upper ? p - x[e] : x[e] + p;
    }
}
__device__ __forceinline__ void fwht128(float (&x)[2], int l) {
    const float t = x[0];
    x[0] = t + x[1];
    x[1] = t - x[1];
    fwht_stage<1>(x, l);
    fwht_stage<2>(x, l);
    fwht_stage<4>(x, l);
    fwht_stage<8>(x, l);
    fwht_stage<16>(x, l);
    fwht_stage<32>(x, l);
}

// One stage of the butterflies on a register bit: x[r], x[r + step] to their sum and difference.
template <int N>
__device__ __forceinline__ void stage(float (&x)[N], int step) {
#pragma unroll
    for (int r = 0; r < N; ++r)
        if (!(r & step)) {
            const float u = x[r], v = x[r + step];
            x[r] = u + v;
            x[r + step] = u - v;
        }
}

template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_or_0(double x) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xF, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Running sum over the lanes, this one included: inside rows of 16 by shifts, then the last lanes of the rows before.
__device__ __forceinline__ double running(double x) {
    x += dpp_or_0<0x111, 0xF>(x);
    x += dpp_or_0<0x112, 0xF>(x);
    x += dpp_or_0<0x114, 0xF>(x);
    x += dpp_or_0<0x118, 0xF>(x);
    x += dpp_or_0<0x142, 0xA>(x);
    return x + dpp_or_0<0x143, 0xC>(x);
}

// The sequence with the given rank by length, the longest first (equal ones in order of index).
// Every wave ranks the whole batch, two sequences per lane; where all are equally long, rank is index.
__device__ __forceinline__ int sequence_of_rank(const int32_t* seq_len, int batch, int rank, int l) {
    const int i0 = min(l, batch - 1), i1 = min(64 + l, batch - 1);
    const int len0 = seq_len[i0], len1 = seq_len[i1];
    const int first = __builtin_amdgcn_readfirstlane(len0);
    if (!__any(len0 != first || len1 != first)) return rank;
    // unique keys: the length (capped, an order is all that is asked), then the smaller index
    const uint32_t k0 = (uint32_t)min(max(len0, 0), 0xFFFFFF) << 7 | (uint32_t)(kOrderBatch - 1 - i0);
    const uint32_t k1 = (uint32_t)min(max(len1, 0), 0xFFFFFF) << 7 | (uint32_t)(kOrderBatch - 1 - i1);
    int r0 = 0, r1 = 0;
    for (int i = 0; i < min(batch, 64); ++i) {
        const uint32_t k = __builtin_amdgcn_readlane(k0, i);
        r0 += k > k0;
        r1 += k > k1;
    }
    for (int i = 64; i < batch; ++i) {
        const uint32_t k = __builtin_amdgcn_readlane(k1, i - 64);
        r0 += k > k0;
        r1 += k > k1;
    }
    // (clamped lanes repeat the last sequence; the first lane that holds the rank is taken)
    const uint64_t m0 = __ballot(r0 == rank), m1 = __ballot(r1 == rank);
    return min(m0 ? __builtin_ctzll(m0) : 64 + __builtin_ctzll(m1), batch - 1);
}

// Orders this wave's accesses to its own LDS: a wave's LDS operations execute in issue order,
// so no wait is needed, only a point that the compiler does not move memory operations across.
// (Each wave of a decode workgroup has an LDS block of its own.)
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

}  // namespace
}  // namespace kvarn
