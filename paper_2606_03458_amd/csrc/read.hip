// Cached tokens back as rows (include/kvarn.h, kvarn_read_tokens): sink and residual rows as stored, body
// tiles dequantized, (code a + b) s2, and rotated back.
#include "common.hpp"

namespace kvarn {
namespace {

// Code of (token t, channel c) of a packed tile (layout: include/kvarn.h).
__device__ __forceinline__ int code_at(const uint32_t* w, int kind, int bits, int t, int c) {
    const int p = 8 / bits;
    int u, e;
    if (kind == KVARN_KEYS) {
        u = ((t >> 6) * 64 + 16 * ((c & 63) >> 4) + (t & 15)) * 8 + 2 * ((t & 63) >> 4) + (c >> 6);
        e = c & 15;
    } else {
        u = ((t >> 6) * 64 + 16 * ((t & 15) >> 2) + (c & 15)) * 8 + (c >> 4);
        e = 4 * ((t & 63) >> 4) + (t & 3);
    }
    const int sigma = u >> 9, L = (u >> 3) & 63, wi = u & 7, s = e >> 2, q = e & 3;
    const uint32_t word = w[512 * (bits / 2) * sigma + 256 * (wi / p) + 4 * L + (bits / 2) * (wi % p) + s / p];
    return (int)(word >> (8 * q + bits * (s % p))) & ((1 << bits) - 1);
}

template <int CMP>
__device__ __forceinline__ void aux_at(const uint8_t* x, int i, float& a, float& b, float& s2) {
    if constexpr (CMP) {
        b = (float)reinterpret_cast<const _Float16*>(x)[i];
        a = __builtin_amdgcn_cvt_f32_fp8(x[256 + i], 0);
        s2 = __builtin_amdgcn_cvt_f32_fp8(x[384 + i], 0);
    } else {
        const float* f = reinterpret_cast<const float*>(x);
        a = f[i];
        b = f[kD + i];
        s2 = f[2 * kD + i];
    }
}

__device__ __forceinline__ void store_row(void* out, int64_t at, int bf16, int c, float v) {
    if (bf16) static_cast<uint16_t*>(out)[at + c] = f32_to_bf16(v);
    else static_cast<float*>(out)[at + c] = v;
}

// Workgroup (stream, kind, part): part 0 the sink and residual rows of the range, part 1 + j the j-th of
// the body tiles that the range touches.  One thread per token.
template <int CMP>
__global__ __launch_bounds__(128) void k_read(ReadArgs a) {
    const int64_t id = blockIdx.x;
    const int part = (int)(id % a.parts);
    const int64_t rest = id / a.parts;
    const int kind = a.kinds == 2 ? (int)(rest & 1) : a.kind0;
    const int64_t stream = a.kinds == 2 ? rest >> 1 : rest;
    const int b = (int)(stream / a.c.n_kv), kh = (int)(stream % a.c.n_kv);
    const int len = a.c.seq_len[b];
    const int64_t first = a.first ? a.first[b] : 0, last = min(first + a.n_tokens, (int64_t)len);
    const int body = len > a.n_sink ? min((len - a.n_sink) / kG, a.c.max_blocks) : 0;
    void* out = kind == KVARN_KEYS ? a.k_out : a.v_out;
    const int64_t base = b * a.seq_stride + kh * a.head_stride;
    if (part == 0) {
        const int64_t body_end = (int64_t)a.n_sink + (len > a.n_sink ? (len - a.n_sink) / kG : 0) * (int64_t)kG;
        for (int64_t t = max(first, (int64_t)0) + threadIdx.x; t < last; t += 128) {
            const uint16_t* row;
            if (t < a.n_sink)
                row = static_cast<const uint16_t*>(kind == KVARN_KEYS ? a.c.k_sink : a.c.v_sink) + (stream * a.n_sink + t) * kD;
            else if (t >= body_end)
                row = static_cast<const uint16_t*>(kind == KVARN_KEYS ? a.c.k_resid : a.c.v_resid) + (stream * kG + (t - body_end)) * kD;
            else
                continue;
            for (int c = 0; c < kD; ++c) store_row(out, base + (t - first) * a.token_stride, a.bf16, c, bf16_to_f32(row[c]));
        }
        return;
    }
    const int64_t from = max(first - a.n_sink, (int64_t)0);
    const int64_t blk = from / kG + part - 1;
    const int64_t t = a.n_sink + blk * kG + threadIdx.x;
    if (blk >= body || t - threadIdx.x >= last) return;
    const int64_t ti = body_tile(a.c, b, kh, (int)blk);
    if (ti < 0 || t < first || t >= last) return;
    const uint8_t* tile = static_cast<const uint8_t*>(kind == KVARN_KEYS ? a.c.k_body : a.c.v_body) +
                          (size_t)ti * tile_bytes(a.bits, CMP);
    const uint8_t* aux = tile + code_bytes(a.bits);
    const int r = threadIdx.x;
    float x[kD];
    float at, bt, st;
    aux_at<CMP>(aux, r, at, bt, st);
#pragma unroll
    for (int c = 0; c < kD; ++c) {
        float ac, bc, sc;
        aux_at<CMP>(aux, c, ac, bc, sc);
        const float z = (float)code_at(reinterpret_cast<const uint32_t*>(tile), kind, a.bits, r, c);
        x[c] = kind == KVARN_KEYS ? (z * ac + bc) * st : (z * at + bt) * sc;
    }
    if (a.rotate) {
#pragma unroll
        for (int m = 1; m < kD; m *= 2)
#pragma unroll
            for (int c = 0; c < kD; ++c)
                if (!(c & m)) {
                    const float u = x[c], v = x[c + m];
                    x[c] = u + v;
                    x[c + m] = u - v;
                }
    }
#pragma unroll
    for (int c = 0; c < kD; ++c)
        store_row(out, base + (t - first) * a.token_stride, a.bf16, c, a.rotate ? x[c] * kInvSqrt128 : x[c]);
}

}  // namespace

hipError_t launch_read(const ReadArgs& a0, hipStream_t stream) {
    ReadArgs a = a0;
    // a range of n tokens touches at most (n - 2) / 128 + 2 tiles
    a.parts = 1 + std::min(a.c.max_blocks, (a.n_tokens + kG - 2) / kG + 1);
    const int64_t grid = (int64_t)a.c.batch * a.c.n_kv * a.kinds * a.parts;
    if (grid * 128 > 0xFFFFFFFFll) return hipErrorInvalidValue;
    if (a.compact) hipLaunchKernelGGL(k_read<1>, dim3((unsigned)grid), dim3(128), 0, stream, a);
    else hipLaunchKernelGGL(k_read<0>, dim3((unsigned)grid), dim3(128), 0, stream, a);
    return hipGetLastError();
}

}  // namespace kvarn
