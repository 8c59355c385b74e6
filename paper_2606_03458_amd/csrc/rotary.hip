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
// rot_dim) of each of its heads, one head after the other in 2 or 4 bytes a lane.  Bound by the latency of a head's loads and
// stores: 16407 tokens of 32 / 8 heads, 40 channels turned, take 149 us in bf16 (2.3 TB/s), 160 in fp32 (4.2).
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

// A 16-byte piece: 8 channels of bf16 or 4 of fp32.
template <int BF16>
struct Piece {
    static constexpr int N = BF16 ? 8 : 4;
    uint4 w;
    __device__ __forceinline__ float get(int e) const {
        const int k = BF16 ? e / 2 : e;
        const uint32_t x = k == 0 ? w.x : k == 1 ? w.y : k == 2 ? w.z : w.w;
        return __uint_as_float(!BF16 ? x : e % 2 ? x & 0xFFFF0000u : x << 16);
    }
    __device__ __forceinline__ void set(const float (&x)[N]) {
        if constexpr (BF16) w = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
        else w = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};

// Rows 16 bytes at a time: 8 threads per head, each with 16 channels in pieces that lie 8 pieces apart (so that
// the threads of a head, and of the next one, read and write whole lines together), over HEADS heads of a
// token, whose cos and sin it forms once.  Bound by memory: 16407 tokens of 32 / 8 heads in bf16 take
// 60 us, 5.6 TB/s, by stores past the caches (which rows that fill no whole lines do not take), and 67 through them; 5003 of 40 / 8 in fp32, half of the channels turned, 39 and 52.  (With one
// head per thread, for a few tokens, either way makes the same time.)
template <int BF16, int HALF, int HEADS>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a, int slices) {
    const int64_t id = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
    const int64_t token = id / slices;
    const int slice = (int)(id - token * slices), j = threadIdx.x & 7;
    if (token >= a.n_tokens) return;
    using P = Piece<BF16>;
    constexpr int es = BF16 ? 2 : 4, N = P::N, NP = 16 / N;  // channels of a piece, pieces of a thread and head
    const int rd = a.rope.rot_dim, h = rd / 2;
    int at[NP];      // first channel of each piece
    bool rot[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        if constexpr (HALF) {
            // pieces 2 q and 2 q + 1: the two channels of N pairs each, or two pieces behind rot_dim
            const int q = j + 8 * (i / 2), turned = h / N;
            rot[i] = q < turned;
            at[i] = rot[i] ? N * q + (i % 2) * h : rd + N * (q - turned) + (i % 2) * (64 - h);
        } else {
            at[i] = N * (j + 8 * i);
            rot[i] = at[i] < rd;
        }
    }
    const int heads = a.n_q + a.n_kv;
    P x[HEADS][NP];
    char* to[HEADS];
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int head = min(slice * HEADS + k, heads - 1);
        const bool key = head >= a.n_q;
        const int hh = key ? head - a.n_q : head;
        const char* from = static_cast<const char*>(key ? a.k : a.q) + (token * (key ? a.k_stride : a.q_stride) + hh * kD) * es;
        to[k] = static_cast<char*>(key ? a.k_out : a.q_out) + (token * (key ? a.k_out_stride : a.q_out_stride) + hh * kD) * es;
#pragma unroll
        for (int i = 0; i < NP; ++i) x[k][i].w = *reinterpret_cast<const uint4*>(from + at[i] * es);
    }
    const int64_t m = position(a, token);
#pragma unroll
    for (int i = 0; i < NP; i += HALF ? 2 : 1) {
        if (!rot[i]) continue;
        constexpr int PAIRS = HALF ? N : N / 2;
        float c[PAIRS], s[PAIRS];
#pragma unroll
        for (int e = 0; e < PAIRS; ++e) turn(a, m, (HALF ? at[i] : at[i] / 2) + e, c[e], s[e]);
#pragma unroll
        for (int k = 0; k < HEADS; ++k) {
            float lo[N], hi[N];
#pragma unroll
            for (int e = 0; e < PAIRS; ++e) {
                const float u = HALF ? x[k][i].get(e) : x[k][i].get(2 * e), v = HALF ? x[k][i + HALF].get(e) : x[k][i].get(2 * e + 1);
                const float p = u * c[e] - v * s[e], q = u * s[e] + v * c[e];
                if constexpr (HALF) lo[e] = p, hi[e] = q;
                else lo[2 * e] = p, lo[2 * e + 1] = q;
            }
            x[k][i].set(lo);
            if constexpr (HALF) x[k][i + 1].set(hi);
        }
    }
#pragma unroll
    for (int k = 0; k < HEADS; ++k)
        if (slice * HEADS + k < heads)
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                if constexpr (HEADS > 1) store_row(to[k] + at[i] * es, x[k][i].w, a.lines);
                else *reinterpret_cast<uint4*>(to[k] + at[i] * es) = x[k][i].w;
            }
}

template <int BF16>
hipError_t launch_wide(const RotaryArgs& a, hipStream_t stream) {
    const int heads = a.n_q + a.n_kv;
    // One head per thread as long as that fills the card (256 CUs with 8 workgroups of 32 heads each), else four,
    // so that a token's angles are formed a quarter as often.
    const int per = a.n_tokens * heads <= 65536 ? 1 : 4, slices = (heads + per - 1) / per;
    const int64_t groups = (a.n_tokens * slices + 31) / 32;
    if (groups > 0xFFFFFFFFll / 256) return hipErrorInvalidValue;
    const dim3 grid((unsigned)groups), block(256);
    if (a.rope.layout == KVARN_ROPE_HALF) {
        if (per == 1) hipLaunchKernelGGL((k_rotary<BF16, 1, 1>), grid, block, 0, stream, a, slices);
        else hipLaunchKernelGGL((k_rotary<BF16, 1, 4>), grid, block, 0, stream, a, slices);
    } else {
        if (per == 1) hipLaunchKernelGGL((k_rotary<BF16, 0, 1>), grid, block, 0, stream, a, slices);
        else hipLaunchKernelGGL((k_rotary<BF16, 0, 4>), grid, block, 0, stream, a, slices);
    }
    return hipGetLastError();
}

// Whether the rows of a side can go 16 bytes at a time.
bool wide_rows(const void* p, int64_t stride, int heads, int es) {
    return heads == 0 || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * es % 16 == 0);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a0, hipStream_t stream) {
    RotaryArgs a = a0;
    const int es = a.bf16 ? 2 : 4;
    a.lines = (a.n_q == 0 || fills_lines(a.q_out, a.q_out_stride * es)) && (a.n_kv == 0 || fills_lines(a.k_out, a.k_out_stride * es));
    if (a.rope.rot_dim % 16 == 0 && wide_rows(a.q, a.q_stride, a.n_q, es) && wide_rows(a.q_out, a.q_out_stride, a.n_q, es) &&
        wide_rows(a.k, a.k_stride, a.n_kv, es) && wide_rows(a.k_out, a.k_out_stride, a.n_kv, es))
        return a.bf16 ? launch_wide<1>(a, stream) : launch_wide<0>(a, stream);
    const int64_t groups = (a.n_tokens + 3) / 4;
    if (groups > 0xFFFFFFFFll / 256) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_rotary_pairs, dim3((unsigned)groups), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace kvarn
