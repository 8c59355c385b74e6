// Packed tiles as operands of the 16-bit matrix cores (v_mfma_f32_16x16x32_f16): tiles as buffers, their codes as halves,
// values as pairs of halves.
#pragma once

#include "common.hpp"
#include "lanes.hpp"

namespace kvarn {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4f mfma_f16(v4u a, v4u b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}
__device__ __forceinline__ v4f mfma_bf16(v4u a, v4u b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// Over the four lanes of a column (lanes n, 16 + n, 32 + n, 48 + n).
template <class F>
__device__ __forceinline__ float across_groups(float v, F f) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(x[0]), __uint_as_float(x[1]));
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float add2(float x, float y) { return x + y; }
__device__ __forceinline__ float max2(float x, float y) { return fmaxf(x, y); }
// Largest of values >= 0 over the wave: their bit patterns order as integers (and a NaN's is the largest).
__device__ __forceinline__ float max_over_wave(float v) {
    int b = __float_as_int(v);
    b = max(b, dpp_x1(b));
    b = max(b, dpp_x2(b));
    b = max(b, dpp_half_mirror(b));
    b = max(b, dpp_mirror(b));
    return across_groups(__int_as_float(b), [](float x, float y) { return __int_as_float(max(__float_as_int(x), __float_as_int(y))); });
}

// log2 of the factor that code_operand leaves at position s of a unit.
template <int BITS, int PREC, int KIND>
__device__ constexpr int plane_shift(int s) {
    return PREC == 2 ? 0 : KIND == KVARN_KEYS && BITS == 2 ? 2 * s : BITS * (s & 1);
}
// 1 / the factor of all positions
template <int BITS, int PREC, int KIND>
constexpr float kCodeUnit = PREC == 2 ? 1.f : KIND == KVARN_KEYS ? 0x1p24f : BITS == 2 ? 0x1p17f : 0x1p21f;

// Codes as halves: positions s = 2 half, 2 half + 1 of a unit, two dwords each (codes 4 s, 4 s + 2 and
// 4 s + 1, 4 s + 3).  PREC 1: times 2^plane_shift / kCodeUnit.  PREC 2: less 2^(bits - 1), without a factor,
// for which the other operand's lower half has no bits to spare.
template <int BITS, int PREC, int KIND>
__device__ __forceinline__ v4u code_operand(const uint32_t* unit, int half) {
    const uint32_t w0 = BITS == 2 ? unit[0] : unit[half];
    const int d = BITS == 2 && half ? 4 : 0;
    const uint32_t m = BITS == 2 ? 0x00030003u : 0x000F000Fu;
    if constexpr (PREC == 1 && KIND == KVARN_KEYS) {
        const uint32_t y = w0 >> 8;
        return v4u{w0 & (m << d), y & (m << d), w0 & (m << (d + BITS)), y & (m << (d + BITS))};
    } else if constexpr (PREC == 1) {
        const int up = BITS == 2 ? 7 : 3, by = up - d;
        const uint32_t x = w0 << by, y = w0 >> (8 - by);
        return v4u{x & (m << up), y & (m << up), x & (m << (up + BITS)), y & (m << (up + BITS))};
    } else {
        v4u w{(w0 >> d) & m, (w0 >> (8 + d)) & m, (w0 >> (d + BITS)) & m, (w0 >> (8 + d + BITS)) & m};
        constexpr _Float16 less = (_Float16)(float)(1024 + (1 << (BITS - 1)));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, w[i] | 0x64006400u) - v2h{less, less});
        return w;
    }
}

__device__ __forceinline__ uint32_t half_pair(float x, float y) {
    return __builtin_bit_cast(uint32_t, v2h{(_Float16)x, (_Float16)y});
}
// x, y as PREC pairs of halves that add up to them
template <int PREC>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&w)[PREC]) {
    w[0] = half_pair(x, y);
    if constexpr (PREC == 2) {
        // The rest is taken from the halves as they are: formed anew from a product, the compiler may round them
        // in another way than the first time (a fused multiply and conversion), one step apart near a tie.
        asm("" : "+v"(w[0]));
        const v2h h = __builtin_bit_cast(v2h, w[0]);
        w[1] = half_pair(x - (float)h[0], y - (float)h[1]);
    }
}
// A packed tile as a buffer: its address stays in scalar registers, a lane's part of an address is one 32-bit offset.
struct Tile {
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ Tile(const uint8_t* p, uint32_t bytes)
        : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, (int)bytes, 0x00027000)) {}
    __device__ __forceinline__ v4u load16(uint32_t at, int off) const { return __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, off, 0); }
    __device__ __forceinline__ float2 load8(uint32_t at, int off) const {
        typedef uint32_t v2u __attribute__((ext_vector_type(2)));
        const v2u x = __builtin_amdgcn_raw_buffer_load_b64(r, (int)at, off, 0);
        return make_float2(__uint_as_float(x[0]), __uint_as_float(x[1]));
    }
    __device__ __forceinline__ uint32_t load4(uint32_t at, int off) const { return __builtin_amdgcn_raw_buffer_load_b32(r, (int)at, off, 0); }
    __device__ __forceinline__ uint16_t load2(uint32_t at, int off) const { return __builtin_amdgcn_raw_buffer_load_b16(r, (int)at, off, 0); }
};

// A tile's aux as it lies in memory, at byte `off`: lane l holds entries 2 l and 2 l + 1 of a, b and s2.
template <int CMP>
struct RawAux {
    float2 a, b, s;
    __device__ __forceinline__ void load(const Tile& t, int off, int l) {
        a = t.load8(8u * l, off);
        b = t.load8(8u * l, off + 512);
        s = t.load8(8u * l, off + 1024);
    }
    __device__ __forceinline__ void get(float2& va, float2& vb, float2& vs) const { va = a, vb = b, vs = s; }
};
template <>
struct RawAux<1> {
    uint32_t b;
    uint16_t a, s;
    __device__ __forceinline__ void load(const Tile& t, int off, int l) {
        b = t.load4(4u * l, off);
        a = t.load2(2u * l, off + 256);
        s = t.load2(2u * l, off + 384);
    }
    __device__ __forceinline__ void get(float2& va, float2& vb, float2& vs) const {
        const v2h h = __builtin_bit_cast(v2h, b);
        const auto fa = __builtin_amdgcn_cvt_pk_f32_fp8((int)a, false), fs = __builtin_amdgcn_cvt_pk_f32_fp8((int)s, false);
        va = make_float2(fa[0], fa[1]);
        vb = make_float2((float)h[0], (float)h[1]);
        vs = make_float2(fs[0], fs[1]);
    }
};

__device__ __forceinline__ float inverse(float power) { return __uint_as_float((254u << 23) - __float_as_uint(power)); }

// A value that is the same in every lane, in a scalar register: so are then the addresses formed from it.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ size_t uniform(size_t v) { return (size_t)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v); }
__device__ __forceinline__ float uniform(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }

}  // namespace
}  // namespace kvarn
