// Cached tokens back as rows (include/kvarn.h, kvarn_read_tokens): sink and residual rows as stored, body
// tiles dequantized, (code a + b) s2, and rotated back.
//
// Bound by memory: a tile of 4.5 to 9.5 KB becomes 32 KB of bf16 or 64 KB of fp32.  About 12 vector instructions per
// element stand beside that, which a CU has time for only if no lane idles, so the rotation's stages are
// taken where the format puts the bits of the channel: those that a lane holds in registers first, the row's two
// that keys keep in lanes by row swaps that exchange them with register bits, and the four that values keep in
// lanes on the way through LDS, by which the rows reach the lanes that store them (16 lanes, one row).
#include "common.hpp"
#include "lanes.hpp"

namespace kvarn {
namespace {

constexpr int kReadRow = 132;  // floats of a row in LDS: rows start 4 banks apart

struct ReadSmem {
    float aux[3][kD];               // a, b, s2 / sqrt(128)
    float rows[4][16][kReadRow];    // a wave's 16 tokens
};

// code j (0..3) of the dword of four codes at position s of a unit, as a float
template <int BITS>
__device__ __forceinline__ uint32_t four_codes(const uint32_t* unit, int s) {
    if constexpr (BITS == 2) return (unit[0] >> (2 * s)) & 0x03030303u;
    else return (unit[s >> 1] >> (4 * (s & 1))) & 0x0F0F0F0Fu;
}
__device__ __forceinline__ float byte_of(uint32_t w, int j) { return (float)((w >> (8 * j)) & 0xFFu); }

// Keys of 16 tokens: lane (G, n) has channels 64 kappa + 16 G + e of token n in x[16 kappa + e].  Rotated, it
// has channels 64 (G % 2) + 32 (r / 8 % 2) + 16 (r / 16) + 8 (G / 2) + r % 8 in x[r].
__device__ __forceinline__ void rotate_keys(float (&x)[32], bool rotate) {
    if (rotate) {
#pragma unroll
        for (int step = 1; step < 32; step *= 2) stage(x, step);
    }
#pragma unroll
    for (int r = 0; r < 32; ++r)
        if (!(r & 8)) {
            const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[r]), __float_as_uint(x[r + 8]), false, false);
            x[r] = __uint_as_float(w[0]);
            x[r + 8] = __uint_as_float(w[1]);
        }
    if (rotate) stage(x, 8);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[r]), __float_as_uint(x[r + 16]), false, false);
        x[r] = __uint_as_float(w[0]);
        x[r + 16] = __uint_as_float(w[1]);
    }
    if (rotate) stage(x, 16);
}

// Row t of the range, if it is in it.
struct Range {
    char* out;  // (sequence, kv head)'s first row
    int64_t first, last, token_bytes;
    __device__ __forceinline__ char* row(int64_t t) const { return t >= first && t < last ? out + (t - first) * token_bytes : nullptr; }
};

// Wave (sg, pair): tokens 64 sg + 32 pair .. + 31 of the tile.
template <int BITS, int KIND, int BF16>
__device__ __forceinline__ void read_tile(const ReadArgs& a, const uint8_t* tile, ReadSmem& sm, const Range& to, int64_t t0) {
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63, G = l >> 4, n = l & 15;
    const int sg = wave >> 1, pair = wave & 1;
    const uint32_t* codes = reinterpret_cast<const uint32_t*>(tile) + 256 * BITS * sg;  // of this half tile
    float(&rows)[16][kReadRow] = sm.rows[wave];
    const bool rotate = a.rotate;
    // units of this lane (BITS / 2 words each): keys 4 pair .. + 3, values all 8
    constexpr int W = BITS / 2, UNITS = KIND == KVARN_KEYS ? 4 : 8;
    uint32_t w[UNITS * W];
#pragma unroll
    for (int i = 0; i < UNITS * W / 4; ++i) {
        const int piece = KIND == KVARN_KEYS ? pair * W + i : i;
        const uint4 v = reinterpret_cast<const uint4*>(codes)[64 * piece + l];
        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
    __syncthreads();  // aux is there
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int tau = 2 * pair + h;  // tokens 64 sg + 16 tau + ..
        if constexpr (KIND == KVARN_KEYS) {
            float x[32];
#pragma unroll
            for (int kap = 0; kap < 2; ++kap)
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const uint32_t c = four_codes<BITS>(&w[(2 * h + kap) * W], s);
                    const float4 va = *reinterpret_cast<const float4*>(&sm.aux[0][64 * kap + 16 * G + 4 * s]);
                    const float4 vb = *reinterpret_cast<const float4*>(&sm.aux[1][64 * kap + 16 * G + 4 * s]);
                    x[16 * kap + 4 * s] = byte_of(c, 0) * va.x + vb.x;
                    x[16 * kap + 4 * s + 1] = byte_of(c, 1) * va.y + vb.y;
                    x[16 * kap + 4 * s + 2] = byte_of(c, 2) * va.z + vb.z;
                    x[16 * kap + 4 * s + 3] = byte_of(c, 3) * va.w + vb.w;
                }
            rotate_keys(x, rotate);
            const float s2 = sm.aux[2][64 * sg + 16 * tau + n];
            wave_sync();
#pragma unroll
            for (int g = 0; g < 4; ++g) {  // register bits 4, 3: channels 16, 32
                const int c = 64 * (G & 1) + 32 * (g & 1) + 16 * (g >> 1) + 8 * (G >> 1);
                const float* y = &x[8 * g];
                if constexpr (BF16) {
                    *reinterpret_cast<uint4*>(&rows[n][c / 2]) = make_uint4(bf16_pair(y[0] * s2, y[1] * s2), bf16_pair(y[2] * s2, y[3] * s2),
                                                                           bf16_pair(y[4] * s2, y[5] * s2), bf16_pair(y[6] * s2, y[7] * s2));
                } else {
                    *reinterpret_cast<float4*>(&rows[n][c]) = make_float4(y[0] * s2, y[1] * s2, y[2] * s2, y[3] * s2);
                    *reinterpret_cast<float4*>(&rows[n][c + 4]) = make_float4(y[4] * s2, y[5] * s2, y[6] * s2, y[7] * s2);
                }
            }
            wave_sync();
            constexpr int LANES = BF16 ? 16 : 32;  // of one row, 16 bytes each
#pragma unroll
            for (int i = 0; i < 16 * LANES / 64; ++i) {
                const int r = i * (64 / LANES) + l / LANES;
                const float4 v = *reinterpret_cast<const float4*>(&rows[r][4 * (l % LANES)]);
                char* p = to.row(t0 + 64 * sg + 16 * tau + r);
                if (p) *reinterpret_cast<float4*>(p + 16 * (l % LANES)) = v;
            }
        } else {
            // lane (G, n): channels 16 w + n of tokens 4 G + i
            const float4 va = *reinterpret_cast<const float4*>(&sm.aux[0][64 * sg + 16 * tau + 4 * G]);
            const float4 vb = *reinterpret_cast<const float4*>(&sm.aux[1][64 * sg + 16 * tau + 4 * G]);
            float x[4][8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                // (the unit's position is a wave's own: one of two constants, by a select)
                const uint32_t c0 = four_codes<BITS>(&w[u * W], h), c1 = four_codes<BITS>(&w[u * W], 2 + h);
                const uint32_t c = pair ? c1 : c0;
                const float s2 = sm.aux[2][16 * u + n];
                x[0][u] = (byte_of(c, 0) * va.x + vb.x) * s2;
                x[1][u] = (byte_of(c, 1) * va.y + vb.y) * s2;
                x[2][u] = (byte_of(c, 2) * va.z + vb.z) * s2;
                x[3][u] = (byte_of(c, 3) * va.w + vb.w) * s2;
            }
            if (rotate) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int step = 1; step < 8; step *= 2) stage(x[i], step);
            }
            wave_sync();
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int u = 0; u < 8; ++u) rows[4 * G + i][16 * u + n] = x[i][u];
            wave_sync();
            // 8 channels of a row: the stage across bit 3 on the way in, bits 0, 1, 2 in registers
            const int j = n;
            const float sign = (j & 1) ? -1.f : 1.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 4 * i + G;
                float y[8];
                const float* lo = &rows[r][16 * (j >> 1)];
                if (rotate) {
                    const float4 p0 = *reinterpret_cast<const float4*>(lo), p1 = *reinterpret_cast<const float4*>(lo + 4);
                    const float4 q0 = *reinterpret_cast<const float4*>(lo + 8), q1 = *reinterpret_cast<const float4*>(lo + 12);
                    y[0] = p0.x + sign * q0.x, y[1] = p0.y + sign * q0.y, y[2] = p0.z + sign * q0.z, y[3] = p0.w + sign * q0.w;
                    y[4] = p1.x + sign * q1.x, y[5] = p1.y + sign * q1.y, y[6] = p1.z + sign * q1.z, y[7] = p1.w + sign * q1.w;
#pragma unroll
                    for (int step = 1; step < 8; step *= 2) stage(y, step);
                } else {
                    const float4 p0 = *reinterpret_cast<const float4*>(lo + 8 * (j & 1)), p1 = *reinterpret_cast<const float4*>(lo + 8 * (j & 1) + 4);
                    y[0] = p0.x, y[1] = p0.y, y[2] = p0.z, y[3] = p0.w, y[4] = p1.x, y[5] = p1.y, y[6] = p1.z, y[7] = p1.w;
                }
                char* p = to.row(t0 + 64 * sg + 16 * tau + r);
                if (!p) continue;
                if constexpr (BF16) {
                    *reinterpret_cast<uint4*>(p + 16 * j) = make_uint4(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7]));
                } else {
                    *reinterpret_cast<float4*>(p + 32 * j) = make_float4(y[0], y[1], y[2], y[3]);
                    *reinterpret_cast<float4*>(p + 32 * j + 16) = make_float4(y[4], y[5], y[6], y[7]);
                }
            }
        }
    }
}

// Rows that are stored as bf16: tokens from .. until - 1, row t at src + (t - base) * 128, 16 lanes each.
template <int BF16>
__device__ __forceinline__ void read_rows(const uint16_t* src, int64_t base, int64_t from, int64_t until, const Range& to) {
    const int c = threadIdx.x & 15;
    for (int64_t t = from + (threadIdx.x >> 4); t < until; t += 16) {
        char* p = to.row(t);
        if (!p) continue;
        const uint4 v = reinterpret_cast<const uint4*>(src + (t - base) * kD)[c];
        if constexpr (BF16) {
            reinterpret_cast<uint4*>(p)[c] = v;
        } else {
            float4* f = reinterpret_cast<float4*>(p) + 2 * c;
            f[0] = make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u));
            f[1] = make_float4(__uint_as_float(v.z << 16), __uint_as_float(v.z & 0xFFFF0000u), __uint_as_float(v.w << 16), __uint_as_float(v.w & 0xFFFF0000u));
        }
    }
}

// Workgroup (stream, kind, part): first the parts of 128 sink rows each, then one of residual rows, then the
// body tiles that the range touches.
template <int BITS, int CMP, int BF16>
__global__ __launch_bounds__(256) void k_read(ReadArgs a) {
    __shared__ ReadSmem sm;
    const uint32_t parts = (uint32_t)a.parts;
    const uint32_t rest = blockIdx.x / parts;
    const int part = (int)(blockIdx.x - rest * parts);
    const int kind = a.kinds == 2 ? (int)(rest & 1) : a.kind0;
    const int64_t stream = a.kinds == 2 ? rest >> 1 : rest;
    const int b = (int)(stream / a.c.n_kv), kh = (int)(stream % a.c.n_kv);
    const int len = a.c.seq_len[b];
    const int64_t first = a.first ? a.first[b] : 0, last = min(first + a.n_tokens, (int64_t)len);
    const int64_t held = max(len - a.n_sink, 0) / kG;  // whole groups
    constexpr int esize = BF16 ? 2 : 4;
    const Range to{static_cast<char*>(kind == KVARN_KEYS ? a.k_out : a.v_out) + (b * a.seq_stride + kh * a.head_stride) * esize, first, last,
                   a.token_stride * esize};
    const int sink_parts = (a.n_sink + kG - 1) / kG;
    if (part < sink_parts) {
        const uint16_t* src = static_cast<const uint16_t*>(kind == KVARN_KEYS ? a.c.k_sink : a.c.v_sink) + stream * a.n_sink * kD;
        read_rows<BF16>(src, 0, (int64_t)part * kG, min((int64_t)(part + 1) * kG, (int64_t)min(len, a.n_sink)), to);
        return;
    }
    if (part == sink_parts) {
        const uint16_t* src = static_cast<const uint16_t*>(kind == KVARN_KEYS ? a.c.k_resid : a.c.v_resid) + stream * kG * kD;
        const int64_t base = a.n_sink + held * kG;
        read_rows<BF16>(src, base, base, len, to);
        return;
    }
    const int64_t blk = max(first - a.n_sink, (int64_t)0) / kG + part - sink_parts - 1;
    const int64_t t0 = a.n_sink + blk * kG;
    if (blk >= min(held, (int64_t)a.c.max_blocks) || t0 >= last || t0 + kG <= first) return;
    const int64_t ti = body_tile(a.c, b, kh, (int)blk);
    if (ti < 0) return;
    const uint8_t* tile = static_cast<const uint8_t*>(kind == KVARN_KEYS ? a.c.k_body : a.c.v_body) + (size_t)ti * tile_bytes(BITS, CMP);
    const int i = threadIdx.x;
    if (i < kD) {
        const uint8_t* x = tile + code_bytes(BITS);
        float va, vb, vs;
        if constexpr (CMP) {
            vb = (float)reinterpret_cast<const _Float16*>(x)[i];
            va = __builtin_amdgcn_cvt_f32_fp8(x[256 + i], 0);
            vs = __builtin_amdgcn_cvt_f32_fp8(x[384 + i], 0);
        } else {
            const float* f = reinterpret_cast<const float*>(x);
            va = f[i];
            vb = f[kD + i];
            vs = f[2 * kD + i];
        }
        sm.aux[0][i] = va;
        sm.aux[1][i] = vb;
        sm.aux[2][i] = a.rotate ? vs * kInvSqrt128 : vs;
    }
    if (kind == KVARN_KEYS) read_tile<BITS, KVARN_KEYS, BF16>(a, tile, sm, to, t0);
    else read_tile<BITS, KVARN_VALUES, BF16>(a, tile, sm, to, t0);
}

template <int BITS, int CMP>
void launch_kind(const ReadArgs& a, unsigned grid, hipStream_t stream) {
    if (a.bf16) hipLaunchKernelGGL((k_read<BITS, CMP, 1>), dim3(grid), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((k_read<BITS, CMP, 0>), dim3(grid), dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_read(const ReadArgs& a0, hipStream_t stream) {
    ReadArgs a = a0;
    // a range of n tokens touches at most (n - 2) / 128 + 2 tiles
    const int tiles = (int)std::min<int64_t>(a.c.max_blocks, ((int64_t)a.n_tokens + kG - 2) / kG + 1);
    a.parts = (a.n_sink + kG - 1) / kG + 1 + tiles;
    const int64_t grid = (int64_t)a.c.batch * a.c.n_kv * a.kinds * a.parts;
    if (grid * 256 > 0xFFFFFFFFll) return hipErrorInvalidValue;
    if (a.compact) a.bits == 2 ? launch_kind<2, 1>(a, (unsigned)grid, stream) : launch_kind<4, 1>(a, (unsigned)grid, stream);
    else a.bits == 2 ? launch_kind<2, 0>(a, (unsigned)grid, stream) : launch_kind<4, 0>(a, (unsigned)grid, stream);
    return hipGetLastError();
}

}  // namespace kvarn
