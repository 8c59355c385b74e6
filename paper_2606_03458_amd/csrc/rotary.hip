// Rotary positions of queries and keys (include/kvarn.h, kvarn_rotary).
#include "common.hpp"

namespace kvarn {
namespace {

// cos and sin of position m at one frequency, times the amplitude.  The angle is reduced to half turns in
// 64 bits with the product's and 2 pi's rounding carried along (an fp32 angle at position 10^6 is off by
// up to 0.03, a plain fp64 one at 2^31 by 5e-7); the rest is small and exact enough in 32.
__device__ __forceinline__ void turn(const RotaryArgs& a, int64_t m, int i, float& c, float& s) {
    constexpr double kTwoPiHi = 6.283185307179586232, kTwoPiLo = 2.4492935982947064e-16;
    const double d = (double)m, f = a.rope.freq[i];
    const double hi = d * f, lo = fma(d, f, -hi);
    const double n = rint(hi * 0.15915494309189534561);
    const double r = fma(-n, kTwoPiLo, fma(-n, kTwoPiHi, hi) + lo);
    float sn, cs;
    sincospif((float)(r * 0.31830988618379069122), &sn, &cs);
    c = cs * a.rope.amplitude;
    s = (a.inverse ? -sn : sn) * a.rope.amplitude;
}

__device__ __forceinline__ int64_t position(const RotaryArgs& a, int64_t token) {
    const int64_t seq = a.tokens_per_seq == 1 ? token : token / a.tokens_per_seq;
    int64_t m = a.positions ? a.positions[token] : token - seq * a.tokens_per_seq;
    if (a.seq_start) m += a.seq_start[seq];
    return m;
}

__device__ __forceinline__ float load1(const void* p, int64_t i, int bf16) {
    return bf16 ? bf16_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store1(void* p, int64_t i, int bf16, float v) {
    if (bf16) static_cast<uint16_t*>(p)[i] = f32_to_bf16(v);
    else static_cast<float*>(p)[i] = v;
}

// Any alignment, any even rot_dim: one wave per token, lane i a pair (or two of the channels behind
// rot_dim) of each of its heads.
__global__ __launch_bounds__(256) void k_rotary_pairs(RotaryArgs a) {
    const int64_t token = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int i = threadIdx.x & 63, h = a.rope.rot_dim / 2;
    if (token >= a.n_tokens) return;
    const bool rot = i < h;
    float c = 1.f, s = 0.f;
    if (rot) turn(a, position(a, token), i, c, s);
    const bool half = a.rope.layout == KVARN_ROPE_HALF;
    const int c0 = rot && half ? i : 2 * i, c1 = rot && half ? i + h : 2 * i + 1;
    for (int head = 0; head < a.n_q + a.n_kv; ++head) {
        const bool key = head >= a.n_q;
        const int hh = key ? head - a.n_q : head;
        const void* x = key ? a.k : a.q;
        void* y = key ? a.k_out : a.q_out;
        const int64_t xi = token * (key ? a.k_stride : a.q_stride) + hh * kD;
        const int64_t yi = token * (key ? a.k_out_stride : a.q_out_stride) + hh * kD;
        const float u = load1(x, xi + c0, a.bf16), v = load1(x, xi + c1, a.bf16);
        store1(y, yi + c0, a.bf16, rot ? u * c - v * s : u);
        store1(y, yi + c1, a.bf16, rot ? u * s + v * c : v);
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
    const int64_t groups = (a.n_tokens + 3) / 4;
    hipLaunchKernelGGL(k_rotary_pairs, dim3((unsigned)groups), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace kvarn
