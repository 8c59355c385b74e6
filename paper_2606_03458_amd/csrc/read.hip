// Cached tokens back as rows (include/kvarn.h, kvarn_read_tokens): sink and residual rows as stored, body
// tiles dequantized, (code a + b) s2, and rotated back.
//
// Bound by memory: a tile of 4.5 to 9.5 KB becomes 32 KB of bf16 or 64 KB of fp32.  16384 tokens of 8 sequences and 8 kv
// heads (2 bits, bf16, 616 MB) take 100 us, 19928 of 3 at 4 bits to fp32 (563 MB) 92, 6.1 TB/s both.  Stores decide it: whole
// rows, past the caches where they fill lines (store_row).  Through them the two took 138 and 127 us; 64 bytes of 16 rows at a time in place of
// whole rows, 168 for the first; parts of lines past the caches, 162 for the second.
//
// Rows that come back rotated and as bf16 are matrix products (read_pairs).  The others need more bits than
// those leave, or no product (read_tile): about 12 vector instructions per element, for which a CU has time only if no
// lane idles, so the rotation's stages are taken where the format puts the bits of the channel: those that a lane holds
// in registers first, the row's two that keys keep in lanes by row swaps that exchange them with register bits, and the
// four that values keep in lanes on the way through LDS, by which the rows reach the lanes that store them.  (In bf16
// these took 119 us for the first above.)
#include "common.hpp"
#include "operands.hpp"

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
    const bool rotate = !BF16 && a.rotate;  // (bf16: read_pairs)
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
                if (p) store_row(p + 16 * (l % LANES), v, a.lines);
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
                if constexpr (BF16) {
                    char* p = to.row(t0 + 64 * sg + 16 * tau + r);
                    if (p) store_row(p + 16 * j, make_uint4(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7])), a.lines);
                } else {
                    // once more through LDS, so that a store takes whole rows: parts of lines cost more
                    wave_sync();
                    *reinterpret_cast<float4*>(&rows[r][8 * j]) = make_float4(y[0], y[1], y[2], y[3]);
                    *reinterpret_cast<float4*>(&rows[r][8 * j + 4]) = make_float4(y[4], y[5], y[6], y[7]);
                    wave_sync();
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int rr = 4 * i + 2 * k + (l >> 5);
                        const float4 v = *reinterpret_cast<const float4*>(&rows[rr][4 * (l & 31)]);
                        char* p = to.row(t0 + 64 * sg + 16 * tau + rr);
                        if (p) store_row(p + 16 * (l & 31), v, a.lines);
                    }
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

// Rotated rows as bf16 by the matrix cores: with H the rotation, u = s2 and w = a of keys, u = a and w = s2 of values,
//   keys    row[d] = u[t] (sum_c H[c][d] w[c] code[t][c] + (H b)[d])
//   values  row[d] = u[t] sum_c H[c][d] w[c] code[t][c] + b[t] (H w)[d]
// The codes are the B operand (a column is a token), exactly; H w, a pair of halves that carries 22 bits of w, is A, whose rows
// are in the order that leaves a lane eight channels of its token side by side.  Keys' units are that operand
// as they lie in memory.  Values' units have their tokens where it has channels: a product with the identity,
// exact, turns them round.  Two bits of c (64 and 4 of keys, 64 and 32 of values) are kept out of the products: H is +-1
// there, so sums and differences of four products make the rows for all four values of these bits of d.  With
// that H w takes 64 registers, which a wave holds for all the tokens it reads.
struct ReadWave {
    float w[kD], h[kD], u[kD], b[kD];  // w scaled, H b or H w, u and b of the tokens
    uint32_t rows[16][68];             // 16 tokens, on their way to the lanes that store them (68: 4 pad)
};

// The same rows one at a time in 32 bits, for a tile whose w lie too far apart for the halves: lane l has channels 2 l and
// 2 l + 1, whose a, b, s2 (values: of tokens) are its va, vb, vs.
template <int BITS, int KIND>
__device__ __forceinline__ void read_apart(const Tile& tile, float2 va, float2 vb, float2 vs, ReadWave& sm, const Range& to, int64_t t0, int p0, int p1) {
    const int l = threadIdx.x & 63;
    constexpr int W = BITS / 2;
    constexpr uint32_t kMask = BITS == 2 ? 0x03u : 0x0Fu;
    wave_sync();
    *reinterpret_cast<float2*>(&sm.u[2 * l]) = KIND == KVARN_KEYS ? vs : va;
    *reinterpret_cast<float2*>(&sm.b[2 * l]) = vb;
    wave_sync();
#pragma unroll 1
    for (int t = 32 * p0; t < 32 * p1; ++t) {
        // a dword of codes of this token (keys) or of four (values), 16 bits of place and token apart
        const int pos = KIND == KVARN_KEYS ? (l >> 1) & 3 : (t >> 4) & 3;
        const int unit = KIND == KVARN_KEYS ? 2 * ((t >> 4) & 3) + (l >> 5) : l >> 3;
        const int word = unit * W + (BITS == 4 ? pos >> 1 : 0);
        const int shift = (BITS == 2 ? 2 * pos : 4 * (pos & 1)) + 8 * (KIND == KVARN_KEYS ? 2 * (l & 1) : t & 3);
        const int from = KIND == KVARN_KEYS ? 16 * ((l >> 3) & 3) + (t & 15) : 16 * ((t >> 2) & 3) + 2 * (l & 7);
        const uint32_t at = 16u * from + 1024u * ((t >> 6) * BITS + word / 4) + 4u * (word % 4);
        const uint32_t w0 = tile.load4(at, 0), w1 = KIND == KVARN_KEYS ? w0 >> 8 : tile.load4(at + 16u, 0);
        const float c0 = (float)(w0 >> shift & kMask), c1 = (float)(w1 >> shift & kMask), u = sm.u[t];
        float x[2];
        if constexpr (KIND == KVARN_KEYS) {
            x[0] = c0 * va.x + vb.x, x[1] = c1 * va.y + vb.y;
        } else {
            const float b = sm.b[t];
            x[0] = (c0 * u + b) * vs.x, x[1] = (c1 * u + b) * vs.y;
        }
        fwht128(x, l);
        const float scale = KIND == KVARN_KEYS ? u * kInvSqrt128 : kInvSqrt128;
        char* p = to.row(t0 + t);
        if (p) *reinterpret_cast<uint32_t*>(p + 4 * l) = bf16_pair(x[0] * scale, x[1] * scale);
    }
}

// Parts p0 .. p1 - 1 of a tile, 32 tokens each.
template <int BITS, int CMP, int KIND>
__device__ __forceinline__ void read_pairs(const ReadArgs& a, const uint8_t* at, ReadWave& sm, const Range& to, int64_t t0, int p0, int p1) {
    const int l = threadIdx.x & 63, G = l >> 4, n = l & 15;
    constexpr int W = BITS / 2, WORDS = KIND == KVARN_KEYS ? 4 * W : 8 * W;
    constexpr float kUnit = kCodeUnit<BITS, 1, KVARN_VALUES>;
    const Tile tile(at, (uint32_t)tile_bytes(BITS, CMP));
    RawAux<CMP> aux;
    aux.load(tile, 2048 * BITS, l);
    auto load = [&](int p, v4u(&w)[WORDS / 4]) {
        const int base = 1024 * BITS * (p >> 1);
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) w[i] = tile.load16(16u * l, base + 1024 * (KIND == KVARN_KEYS ? (p & 1) * W + i : i));
    };
    v4u raw[WORDS / 4];
    load(p0, raw);
    // [rows d & 32 (keys) or d & 4 (values)][channels c: 64, 4 (keys) or 32 (values)]
    v4u hi[2][4], lo[2][4];
    {
        float2 va, vb, vs;
        aux.get(va, vb, vs);
        const float2 x = KIND == KVARN_KEYS ? va : vs;
        // A group of zero range has step 1, whatever the others': down to 2^-16 of it they keep the pair's 22 bits.
        if (__any(fminf(fabsf(x.x), fabsf(x.y)) < 0x1p-16f * max_over_wave(fmaxf(fabsf(x.x), fabsf(x.y))))) {
            read_apart<BITS, KIND>(tile, va, vb, vs, sm, to, t0, p0, p1);
            return;
        }
        float f[2] = {KIND == KVARN_KEYS ? vb.x : vs.x, KIND == KVARN_KEYS ? vb.y : vs.y};
        const float top = max_over_wave(fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(f[0]), fabsf(f[1]))));
        // a power of two, kept within 2^-100 .. 2^126: w and b at most 2^14 against halves of up to 2^16
        const float up = __uint_as_float(min(max(__float_as_uint(top) & 0x7F800000u, 27u << 23), 253u << 23));
        const float down = inverse(up) * 0x1p13f, out = 0x1p-13f * kInvSqrt128;
        if constexpr (KIND == KVARN_KEYS) {
            // H b but for the bits 4 and 64 of c, which are those of the products that it is added to
            const float t = f[0];
            f[0] = t + f[1], f[1] = t - f[1];
            fwht_stage<1>(f, l);
            fwht_stage<4>(f, l);
            fwht_stage<8>(f, l);
            fwht_stage<16>(f, l);
            f[0] *= down / kUnit, f[1] *= down / kUnit;
            vs.x = vs.x * (out * kUnit) * up, vs.y = vs.y * (out * kUnit) * up;
            *reinterpret_cast<float2*>(&sm.u[2 * l]) = vs;
        } else {
            fwht128(f, l);
            f[0] *= kInvSqrt128, f[1] *= kInvSqrt128;
            va.x = va.x * (out * kUnit) * up, va.y = va.y * (out * kUnit) * up;
            *reinterpret_cast<float2*>(&sm.u[2 * l]) = va;
            *reinterpret_cast<float2*>(&sm.b[2 * l]) = vb;
        }
        *reinterpret_cast<float2*>(&sm.w[2 * l]) = make_float2(x.x * down, x.y * down);
        *reinterpret_cast<float2*>(&sm.h[2 * l]) = make_float2(f[0], f[1]);
    }
    wave_sync();
    {
        // Lane (G, n) has row n of A: d = 8 (n / 4) + n % 4 and the rest of m.  H's sign is the parity of c & d: per bit of d
        // a mask for the halves whose c has it.
        auto bit = [&](int b) -> uint32_t { return (n >> b) & 1 ? 0x80008000u : 0u; };
        const uint32_t d0 = bit(0), d1 = bit(1) & 0x80000000u, d3 = bit(2), d4 = bit(3);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                // channels c .. c + 3, dwords (c, c + 2) and (c + 1, c + 3)
                const int c = KIND == KVARN_KEYS ? 64 * (k >> 1) + 16 * G + 8 * e + 4 * (k & 1) : 64 * (k >> 1) + 32 * (k & 1) + 16 * e + 4 * G;
                float4 x = *reinterpret_cast<const float4*>(&sm.w[c]);
                if (KIND == KVARN_KEYS && (k & 1)) {
                    // (the factor that the code's place leaves)
                    constexpr float less = 1.f / (1 << plane_shift<BITS, 1, KVARN_VALUES>(1));
                    x.x *= less, x.y *= less, x.z *= less, x.w *= less;
                }
                const uint32_t own = d1 ^ (KIND == KVARN_KEYS ? (e ? d3 : 0u) ^ (G & 1 ? d4 : 0u) : (G & 2 ? d3 : 0u) ^ (e ? d4 : 0u));
                uint32_t w0[2], w1[2];
                split_pair<2>(x.x, x.z, w0);
                split_pair<2>(x.y, x.w, w1);
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    // keys: c & 32 against d & 32; values: c & 4 against d & 4
                    const uint32_t s = m && (KIND == KVARN_KEYS ? G & 2 : G & 1) ? own ^ 0x80008000u : own;
                    hi[m][k][2 * e] = w0[0] ^ s;
                    hi[m][k][2 * e + 1] = w1[0] ^ s ^ d0;
                    lo[m][k][2 * e] = w0[1] ^ s;
                    lo[m][k][2 * e + 1] = w1[1] ^ s ^ d0;
                }
            }
    }
    for (int p = p0; p < p1; ++p) {
        v4u w[WORDS / 4];
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) w[i] = raw[i];
        if (p + 1 < p1) load(p + 1, raw);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = 32 * p + 16 * h + n;
            v4u f[4];
            if constexpr (KIND == KVARN_KEYS) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int u = (2 * h + k) * W;
                    const uint32_t unit[2] = {w[u / 4][u % 4], w[(u + W - 1) / 4][(u + W - 1) % 4]};
                    const v4u x = code_operand<BITS, 1, KVARN_VALUES>(unit, 0), y = code_operand<BITS, 1, KVARN_VALUES>(unit, 1);
                    f[2 * k] = v4u{x[0], x[1], y[0], y[1]};
                    f[2 * k + 1] = v4u{x[2], x[3], y[2], y[3]};
                }
            } else {
                // token 4 G + i of this half in dwords 2 h (i = 0, 2) and 2 h + 1 (i = 1, 3)
                const uint32_t one = BITS * h == 0 ? 0x3C00u : BITS == 2 ? 0x3400u : 0x2C00u;  // 2^-plane_shift(h)
                const uint32_t x = n >> 2 == G ? ((n & 2) ? one << 16 : one) : 0u;
                v4u unity{0u, 0u, 0u, 0u};
                unity[2 * h] = n & 1 ? 0u : x;
                unity[2 * h + 1] = n & 1 ? x : 0u;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t unit[1];
                    if constexpr (BITS == 2) unit[0] = w[c / 4][c % 4] >> (4 * (p & 1));
                    else unit[0] = p & 1 ? w[c / 2][2 * (c % 2) + 1] : w[c / 2][2 * (c % 2)];
                    const v4f r = mfma_f16(code_operand<BITS, 1, KVARN_VALUES>(unit, 0), unity, v4f{0.f, 0.f, 0.f, 0.f});
                    f[c >> 1][2 * (c & 1)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(r[0], r[2]));
                    f[c >> 1][2 * (c & 1) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(r[1], r[3]));
                }
            }
            const float u = sm.u[t], vb = KIND == KVARN_KEYS ? 0.f : sm.b[t];
            uint32_t row[2][2][4];  // [d & 64][d & 32][pair of channels]
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                // where d is for channel bits k of the products: d & 64 in k & 2, d & 4 (keys) or d & 32 (values) in k & 1
                const float* c = &sm.h[8 * G + (KIND == KVARN_KEYS ? 32 : 4) * m];
                constexpr int kNext = KIND == KVARN_KEYS ? 4 : 32;
                v4f s[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v4f z{0.f, 0.f, 0.f, 0.f};
                    if constexpr (KIND == KVARN_KEYS) z = *reinterpret_cast<const v4f*>(c + 64 * (k >> 1) + kNext * (k & 1));
                    s[k] = mfma_f16(lo[m][k], f[k], z);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) s[k] = mfma_f16(hi[m][k], f[k], s[k]);
                const v4f x0 = s[0] + s[1], x1 = s[0] - s[1], y0 = s[2] + s[3], y1 = s[2] - s[3];
                v4f x[4] = {x0 + y0, x1 + y1, x0 - y0, x1 - y1};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    x[k] *= u;
                    if constexpr (KIND == KVARN_VALUES) x[k] += vb * *reinterpret_cast<const v4f*>(c + 64 * (k >> 1) + kNext * (k & 1));
                    uint32_t* r = KIND == KVARN_KEYS ? &row[k >> 1][m][2 * (k & 1)] : &row[k >> 1][k & 1][2 * m];
                    r[0] = bf16_pair(x[k][0], x[k][1]);
                    r[1] = bf16_pair(x[k][2], x[k][3]);
                }
            }
            wave_sync();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t* r = row[i >> 1][i & 1];
                *reinterpret_cast<uint4*>(&sm.rows[n][4 * G + 16 * i]) = make_uint4(r[0], r[1], r[2], r[3]);
            }
            wave_sync();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 4 * i + G;
                const uint4 v = *reinterpret_cast<const uint4*>(&sm.rows[r][4 * n]);
                char* q = to.row(t0 + 32 * p + 16 * h + r);
                if (q) store_row(q + 16 * n, v, a.lines);
            }
        }
    }
}

// A workgroup's (stream, kind, part): first the parts of 128 sink rows each, then one of residual rows, then the
// body tiles that the range touches, `tiles` of them for a workgroup.
struct Job {
    Range to;
    int64_t stream, t0;     // t0: the token that tile blk starts with
    int64_t blk, ends;      // tiles blk .. ends - 1 at most
    int kind, b, kh;
};

// The workgroup's job, or false if it is done: its rows are copied, or it has no tile.
template <int BF16>
__device__ __forceinline__ bool take_job(const ReadArgs& a, int tiles, Job& job) {
    const uint32_t n_kv = (uint32_t)a.c.n_kv, parts = (uint32_t)a.parts;
    const uint32_t all = blockIdx.x / n_kv, rest = all / parts;
    const int kh = (int)(blockIdx.x - all * n_kv), part = (int)(all - rest * parts);
    const int kind = a.kinds == 2 ? (int)(rest & 1) : a.kind0;
    const int b = (int)(a.kinds == 2 ? rest >> 1 : rest);
    const int64_t stream = (int64_t)b * a.c.n_kv + kh;
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
        return false;
    }
    if (part == sink_parts) {
        const uint16_t* src = static_cast<const uint16_t*>(kind == KVARN_KEYS ? a.c.k_resid : a.c.v_resid) + stream * kG * kD;
        const int64_t base = a.n_sink + held * kG;
        read_rows<BF16>(src, base, base, len, to);
        return false;
    }
    const int64_t blk = max(first - a.n_sink, (int64_t)0) / kG + (int64_t)(part - sink_parts - 1) * tiles;
    // (a range that ends within the sink, or before it, ends before tile 0)
    const int64_t ends = min(min(held, (int64_t)a.c.max_blocks), last > a.n_sink && last > first ? (last - a.n_sink + kG - 1) / kG : (int64_t)0);
    job = Job{to, stream, a.n_sink + blk * kG, blk, ends, kind, b, kh};
    return blk < ends;
}

template <int BITS, int CMP, int BF16>
__global__ __launch_bounds__(256) void k_read(ReadArgs a) {
    __shared__ ReadSmem sm;
    Job j;
    if (!take_job<BF16>(a, 1, j)) return;
    const int64_t ti = body_tile(a.c, j.b, j.kh, (int)j.blk);
    if (ti < 0) return;
    const uint8_t* tile = static_cast<const uint8_t*>(j.kind == KVARN_KEYS ? a.c.k_body : a.c.v_body) + (size_t)ti * tile_bytes(BITS, CMP);
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
        sm.aux[2][i] = !BF16 && a.rotate ? vs * kInvSqrt128 : vs;
    }
    if (j.kind == KVARN_KEYS) read_tile<BITS, KVARN_KEYS, BF16>(a, tile, sm, j.to, j.t0);
    else read_tile<BITS, KVARN_VALUES, BF16>(a, tile, sm, j.to, j.t0);
}

// Rotated, as bf16: a wave has a tile of its own (WHOLE), or a quarter of one.
template <int BITS, int CMP, bool WHOLE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_read_rotated(ReadArgs a) {
    __shared__ ReadWave sm[4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Job j;
    if (!take_job<1>(a, WHOLE ? 4 : 1, j)) return;
    if constexpr (WHOLE) {
        j.blk += wave;
        j.t0 += wave * kG;
        if (j.blk >= j.ends) return;
    }
    const int64_t ti = body_tile(a.c, j.b, j.kh, (int)j.blk, threadIdx.x & 63);
    if (ti < 0) return;
    const size_t at = uniform((size_t)ti * tile_bytes(BITS, CMP));
    const int p0 = WHOLE ? 0 : wave, p1 = WHOLE ? 4 : wave + 1;
    if (j.kind == KVARN_KEYS) read_pairs<BITS, CMP, KVARN_KEYS>(a, static_cast<const uint8_t*>(a.c.k_body) + at, sm[wave], j.to, j.t0, p0, p1);
    else read_pairs<BITS, CMP, KVARN_VALUES>(a, static_cast<const uint8_t*>(a.c.v_body) + at, sm[wave], j.to, j.t0, p0, p1);
}

template <int BITS, int CMP>
void launch_kind(const ReadArgs& a, bool whole, unsigned grid, hipStream_t stream) {
    if (a.bf16 && a.rotate && whole) hipLaunchKernelGGL((k_read_rotated<BITS, CMP, true>), dim3(grid), dim3(256), 0, stream, a);
    else if (a.bf16 && a.rotate) hipLaunchKernelGGL((k_read_rotated<BITS, CMP, false>), dim3(grid), dim3(256), 0, stream, a);
    else if (a.bf16) hipLaunchKernelGGL((k_read<BITS, CMP, 1>), dim3(grid), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((k_read<BITS, CMP, 0>), dim3(grid), dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_read(const ReadArgs& a0, hipStream_t stream) {
    ReadArgs a = a0;
    // a range of n tokens touches at most (n - 2) / 128 + 2 tiles
    const int tiles = (int)std::min<int64_t>(a.c.max_blocks, ((int64_t)a.n_tokens + kG - 2) / kG + 1);
    const int64_t streams = (int64_t)a.c.batch * a.c.n_kv * a.kinds;
    // A tile for each wave, which forms H w once for it, where that makes most of the 2048 waves that the card holds; else a
    // workgroup for each tile (8 kv heads, 2 bits: 112 tiles 10.5 and 5.1 us, 960: 15.0 and 12.0, 1984: 16.2 and 18.8,
    // 15872: 108 and 129).
    const bool whole = a.bf16 && a.rotate && streams * tiles >= 1536;
    a.parts = (a.n_sink + kG - 1) / kG + 1 + (whole ? (tiles + 3) / 4 : tiles);
    const int64_t grid = streams * a.parts, es = a.bf16 ? 2 : 4;
    a.lines = fills_lines(a.k_out, a.token_stride * es) && fills_lines(a.v_out, a.head_stride * es) && a.seq_stride * es % 128 == 0;
    if (grid * 256 > 0xFFFFFFFFll) return hipErrorInvalidValue;
    if (a.compact) a.bits == 2 ? launch_kind<2, 1>(a, whole, (unsigned)grid, stream) : launch_kind<4, 1>(a, whole, (unsigned)grid, stream);
    else a.bits == 2 ? launch_kind<2, 0>(a, whole, (unsigned)grid, stream) : launch_kind<4, 0>(a, whole, (unsigned)grid, stream);
    return hipGetLastError();
}

}  // namespace kvarn
