// Attention of drafted tokens over the packed cache and over the drafts that their masks name
// (include/kvarn.h, kvarn_tree_attention).  One wave per (draft, query head): body tiles are attended in
// the rotated domain with both scales applied to every element, sink, residual and draft rows as they
// are, with the running maximum and sum of the softmax over both.
#include "common.hpp"

namespace kvarn {
namespace {

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

__device__ __forceinline__ void aux_at(const TreeArgs& a, const uint8_t* x, int i, float& va, float& vb, float& vs) {
    if (a.compact) {
        vb = (float)reinterpret_cast<const _Float16*>(x)[i];
        va = __builtin_amdgcn_cvt_f32_fp8(x[256 + i], 0);
        vs = __builtin_amdgcn_cvt_f32_fp8(x[384 + i], 0);
    } else {
        const float* f = reinterpret_cast<const float*>(x);
        va = f[i];
        vb = f[kD + i];
        vs = f[2 * kD + i];
    }
}

__device__ __forceinline__ float load1(const void* p, int64_t i, int bf16) {
    return bf16 ? bf16_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

struct Row {
    float q[kD], p[kD];
};

// H x / sqrt(128) of a row in LDS, by the wave that owns it.
__device__ void rotate_row(float* x, int l) {
    for (int m = 1; m < kD; m *= 2) {
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");
        __builtin_amdgcn_wave_barrier();
        const int c = (l & (m - 1)) | (l & ~(m - 1)) << 1;
        const float u = x[c], v = x[c + m];
        x[c] = u + v;
        x[c + m] = u - v;
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");
    __builtin_amdgcn_wave_barrier();
    x[l] *= kInvSqrt128;
    x[l + 64] *= kInvSqrt128;
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float wave_reduce_max(float v) {
    for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}
__device__ __forceinline__ float wave_reduce_sum(float v) {
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

__global__ __launch_bounds__(64) void k_tree_rows(TreeArgs a) {
    __shared__ Row r;
    const int l = threadIdx.x;
    const int64_t id = blockIdx.x;  // ((batch * n_draft) * n_q)
    const int h = (int)(id % a.n_q);
    const int64_t bi = id / a.n_q;
    const int i = (int)(bi % a.n_draft), b = (int)(bi / a.n_draft);
    const int live = a.n_live ? min(max(a.n_live[b], 0), a.n_draft) : a.n_draft;
    if (i >= live) return;
    const int kh = h / a.g;
    const int64_t stream = (int64_t)b * a.c.n_kv + kh;
    const int64_t qi = bi * a.q_stride + (int64_t)h * kD;
    const float q0 = load1(a.q, qi + l, a.q_bf16), q1 = load1(a.q, qi + l + 64, a.q_bf16);
    const int len = max(a.c.seq_len[b], 0);
    const int ns = min(len, a.n_sink);
    const int nb = min((len - ns) / kG, a.c.max_blocks), nr = (len - ns) % kG;
    float m = -3e38f, sum = 0.f, o0 = 0.f, o1 = 0.f;  // channels l and l + 64
    r.q[l] = q0;
    r.q[l + 64] = q1;
    bool ids_ok = true;
    if (a.c.block_table)
        for (int blk = 0; blk < nb; ++blk) ids_ok &= body_tile(a.c, b, kh, blk) >= 0;
    if (ids_ok && nb > 0) {
        if (a.rotate) rotate_row(r.q, l);
        for (int blk = 0; blk < nb; ++blk) {
            const size_t at = (size_t)body_tile(a.c, b, kh, blk) * tile_bytes(a.bits, a.compact);
            const uint8_t* kt = static_cast<const uint8_t*>(a.c.k_body) + at;
            const uint8_t* vt = static_cast<const uint8_t*>(a.c.v_body) + at;
            float s[2];
            for (int e = 0; e < 2; ++e) {
                const int t = l + 64 * e;
                float sa, sb, ss, dot = 0.f;
                for (int c = 0; c < kD; ++c) {
                    aux_at(a, kt + code_bytes(a.bits), c, sa, sb, ss);
                    dot += r.q[c] * ((float)code_at(reinterpret_cast<const uint32_t*>(kt), 0, a.bits, t, c) * sa + sb);
                }
                aux_at(a, kt + code_bytes(a.bits), t, sa, sb, ss);
                s[e] = dot * ss * a.scale_log2;
            }
            const float mn = fmaxf(m, wave_reduce_max(fmaxf(s[0], s[1])));
            const float al = exp2f(m - mn), p0 = exp2f(s[0] - mn), p1 = exp2f(s[1] - mn);
            m = mn;
            sum = sum * al + wave_reduce_sum(p0 + p1);
            __syncthreads();
            r.p[l] = p0;
            r.p[l + 64] = p1;
            __syncthreads();
            float x[2] = {0.f, 0.f}, sa, sb, ss;
            for (int t = 0; t < kG; ++t) {
                aux_at(a, vt + code_bytes(a.bits), t, sa, sb, ss);
                for (int e = 0; e < 2; ++e)
                    x[e] += r.p[t] * ((float)code_at(reinterpret_cast<const uint32_t*>(vt), 1, a.bits, t, l + 64 * e) * sa + sb);
            }
            aux_at(a, vt + code_bytes(a.bits), l, sa, sb, ss);
            o0 = o0 * al + x[0] * ss;
            aux_at(a, vt + code_bytes(a.bits), l + 64, sa, sb, ss);
            o1 = o1 * al + x[1] * ss;
        }
        if (a.rotate) {
            __syncthreads();
            r.p[l] = o0;
            r.p[l + 64] = o1;
            rotate_row(r.p, l);
            o0 = r.p[l];
            o1 = r.p[l + 64];
        }
    }
    const uint64_t mask = a.mask ? a.mask[bi] : (i == 63 ? ~0ull : (2ull << i) - 1);
    for (int t = 0; t < ns + nr + live; ++t) {
        float k0, k1, v0, v1;
        if (t < ns + nr) {
            const bool sink = t < ns;
            const int64_t at = (sink ? stream * a.n_sink + t : stream * kG + (t - ns)) * kD + l;
            const uint16_t* kp = static_cast<const uint16_t*>(sink ? a.c.k_sink : a.c.k_resid) + at;
            const uint16_t* vp = static_cast<const uint16_t*>(sink ? a.c.v_sink : a.c.v_resid) + at;
            k0 = bf16_to_f32(kp[0]);
            k1 = bf16_to_f32(kp[64]);
            v0 = bf16_to_f32(vp[0]);
            v1 = bf16_to_f32(vp[64]);
        } else {
            const int j = t - ns - nr;
            if (!((mask >> j) & 1)) continue;
            const int64_t at = ((int64_t)b * a.n_draft + j) * a.kv_stride + (int64_t)kh * kD + l;
            k0 = bf16_to_f32(f32_to_bf16(load1(a.k, at, a.kv_bf16)));
            k1 = bf16_to_f32(f32_to_bf16(load1(a.k, at + 64, a.kv_bf16)));
            v0 = bf16_to_f32(f32_to_bf16(load1(a.v, at, a.kv_bf16)));
            v1 = bf16_to_f32(f32_to_bf16(load1(a.v, at + 64, a.kv_bf16)));
        }
        const float s = wave_reduce_sum(q0 * k0 + q1 * k1) * a.scale_log2;
        const float mn = fmaxf(m, s), al = exp2f(m - mn), p = exp2f(s - mn);
        m = mn;
        sum = sum * al + p;
        o0 = o0 * al + p * v0;
        o1 = o1 * al + p * v1;
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const int64_t oi = bi * a.out_stride + (int64_t)h * kD + l;
    if (a.out_bf16) {
        static_cast<uint16_t*>(a.out)[oi] = f32_to_bf16(o0 * inv);
        static_cast<uint16_t*>(a.out)[oi + 64] = f32_to_bf16(o1 * inv);
    } else {
        static_cast<float*>(a.out)[oi] = o0 * inv;
        static_cast<float*>(a.out)[oi + 64] = o1 * inv;
    }
}

}  // namespace

size_t tree_workspace_bytes(const kvarn_cache&, int, int, int, int, int) { return 0; }

hipError_t launch_tree(const TreeArgs& a, hipStream_t stream) {
    const int64_t rows = (int64_t)a.c.batch * a.n_draft * a.n_q;
    if (rows * 64 > 0xFFFFFFFFll) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_tree_rows, dim3((unsigned)rows), dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace kvarn
