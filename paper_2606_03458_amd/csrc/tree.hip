// Attention of drafted tokens over the packed cache and over the drafts that their masks name
// (include/kvarn.h, kvarn_tree_attention).
//
// The drafts of a sequence and the query heads of a kv head make n_draft * group query rows over the same
// keys: matrix products, on the 16-bit matrix cores (v_mfma_f32_16x16x32_f16).  With q the rotated query and a
// tile's scales (as in the decode)
//   S[t]  = s2K[t] * (sum_c (q a_K)[c] code[t][c] + q . b_K)
//   O[c] += s2V[c] * (sum_t (p a_V)[t] code[t][c] + p . b_V)
// so the codes enter the products as they are, exactly, and only q a_K and p a_V are rounded to 16 bits (for
// an fp32 out to a pair of 16-bit halves).  Both products are taken transposed, keys and values as
// the A operand, rows as columns of B: the tile format's units are then A operands as they lie in
// memory, a row's logits lie in the registers of the four lanes of its column, and they are B operand of
// the second product where the first one leaves them, without a lane move.
//
// A code as an operand costs little more than one instruction per pair: two codes of a 32-bit word, 16 bits
// apart, are masked out where they lie in the word or in one shifted copy of it, which reads as two
// halves, subnormal ones or ones of the lowest exponent, which continue them: the codes times a power of two. The
// other operand's a carries what differs between the places.  The matrix cores keep so many bits of a product from
// its operands' exponents on and cut off the rest, so a subnormal code costs bits of the sum, fewer the
// higher it lies.  Of keys they are taken at bits 0 and up: the products have either sign, and a logit's error is below 1e-5.
// Of values all products are positive and what is lost always goes down (2.5e-4 in the first channel over 33k
// tokens, where the constant part of a rotated row ends up), so theirs lie at bits 7, 8 and 9, 10 (3 to 6
// and 7 to 10 at 4 bits), for a second shift.  The 22 bits of an fp32 out take whole halves, 1024 + code less 1024 +
// 2^(bits - 1).
//
// The probabilities are formed with a in them, but for the power of two of the tile's largest, which goes to s2:
// p a = 2^(logit + log2(a) - reference), largest at 2^kUp whatever the tile's values.  So a tile of values far below or
// above another's keeps its probabilities' bits, and its part of the sum.
//
// For a bf16 out the terms that stand beside the codes go through the matrix cores too, as four more rows of A:
// sum_c (q a)[c] (b / a)[c], sum_t (p a)[t] (b / a)[t] and the softmax's own sum_t (p a)[t] (1 / a)[t], their
// right sides as pairs of halves that add up to 22 bits.  That takes 230 of 1220 vector instructions out of a tile's
// work on 32 rows, and since the same rounded q a and p a meet code + b / a, the key or value itself, their rounding
// weighs no more than a rounding of q or p.  An fp32 out takes these sums in 32 bits, with the codes less their middle; the
// matrix cores cut off what they add to a larger value, so its products start from 0 and the offsets are added behind them.
//
// A tile whose smallest a lies too far below its largest (kApartK, kApartV) is left for a loop of its own, which takes its
// elements in 32 bits: a group of zero range has step 1, so the others may lie as far below as they like.
//
// Bound by vector issue: a tile with 32 rows takes 1019 vector instructions beside 144 matrix products, most of them the softmax's
// (an exponential, a conversion, a maximum per logit) and the codes'.  32 sequences of 32k tokens, 64 drafts, 32 / 8 heads,
// 2 bits: 1.36 ms, 809 TFLOP/s, vector units issuing 80 % of the time, matrix cores busy 36 %.  One sequence of 8k with 16
// drafts: 18 us, the latency of a wave's two or three tiles and of the merge.
//
// Sink, residual and draft rows (bf16, unrotated) take the bf16 matrix cores in chunks of 32, queries and
// probabilities as sums of bf16 pieces.  A wave attends its tiles first, rotates its sums back in registers,
// and goes on with its chunks.
#include "common.hpp"
#include "operands.hpp"

namespace kvarn {
namespace {

constexpr int kRow = 132;        // floats of a row in LDS and of a partial: 128, its reference and sum, 2 pad
constexpr float kUp = 14.f;      // log2 of the largest probability (times a): halves hold up to 2^16
constexpr float kNone = -3e38f;  // the running reference of a row that has seen nothing
// Of a tile's largest step, what its smallest may be for the halves to carry both (keys', values').  Values' would go down to
// 2^-16 by that; but the largest may be that of a token of zeros, whose range is none and whose step is 1, and where such a token
// takes most of a row's weight the others' p a lie further down (values of 1e-3 at 4 bits, of steps 2^-12, beside one with 0.9999 of
// the weight: rows off by 2.5e-2 of themselves; at 2^-5 by 2e-4).
template <int PREC> constexpr float kApartK = PREC == 2 ? 0x1p-6f : 0x1p-13f;
template <int PREC> constexpr float kApartV = PREC == 2 ? 0x1p-6f : 0x1p-5f;
// PREC 2 takes codes less their middle, so that a group of zero range, whose step is 1 and whose elements are none of it, leaves
// the rounding of 2^(BITS - 1) steps (a value token of zeros with 0.9 of a row's weight beside values of 1: rows off by 4e-4 of
// themselves; a channel of zeros that queries of 1000 meet: logits by 1e-3).  So tiles with such a group are left for the
// second loop, too: looking for one costs 1 %.
constexpr float kMostV = 0x1p80f;  // values' steps that s2 and a code's unit still go beside
constexpr float kMost = 0x1p100f, kLeast = 0x1p-55f;  // the powers of two that power_of gives

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// x, y as N pairs of bf16 that add up to them
template <int N>
__device__ __forceinline__ void split_bf16(float x, float y, uint32_t (&w)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        w[i] = bf16_pair(x, y);
        x -= __uint_as_float(w[i] << 16);
        y -= __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// The power of two at or below a value >= 0, kept within 2^-55 .. 2^100 (kLeast, kMost), so that the product of two inverses (of a
// query's and a tile's) is finite, too.
__device__ __forceinline__ float power_of(float v) { return __uint_as_float(min(max(__float_as_uint(v) & 0x7F800000u, 72u << 23), 227u << 23)); }

// Two neighbouring entries x, y as halves into row `type` of `rows` (64 dwords and 4 pad) and what is left of them into the
// row behind it.
__device__ __forceinline__ void put_halves(uint32_t (&rows)[6][68], int type, int at, float x, float y) {
    const _Float16 hx = (_Float16)x, hy = (_Float16)y;
    char* p = reinterpret_cast<char*>(rows[type]) + at;
    *reinterpret_cast<_Float16*>(p) = hx;
    *reinterpret_cast<_Float16*>(p + 4) = hy;
    *reinterpret_cast<_Float16*>(p + 272) = (_Float16)(x - (float)hx);
    *reinterpret_cast<_Float16*>(p + 276) = (_Float16)(y - (float)hy);
}

// A row's reference moves up to 2^-kUp of the new maximum; what it has so far goes down by as much.
__device__ __forceinline__ void raise(float top, float& m, float& sum, v4f (&o)[8]) {
    top = fmaxf(top - kUp, m);
    if (__any(top != m)) {
        const float down = exp2_fast(m - top);
        m = top;
        sum *= down;
#pragma unroll
        for (int w = 0; w < 8; ++w) o[w] *= down;
    }
}

template <int PREC, int NB, int WAVES>
struct TreeSmem {
    union {
        struct {
            float q[16 * NB][kRow];                 // rotated queries
            uint32_t plain[PREC + 1][16 * NB][68];  // queries as given, in pieces of bf16 that add up to them (68: 4 pad)
            float own[WAVES][NB == 1 ? 896 : 1024];  // a wave's: aux rows of its tile, or probabilities of a chunk
        };
        float o[WAVES][16 * NB][kRow];  // the waves' sums (o[..][128]: reference, [129]: sum)
    };
    float top[WAVES], steep[WAVES];
    float low[16 * NB];  // the power of two of a row over that of the largest, where it was taken out of sm.q
    uint32_t more[WAVES][6][68];  // a wave's: b / a of its K tile, 1 / a and b / a of its V tile, in halves and the rest
};

// A sequence's regions: sink tokens, body tiles, residual tokens, live drafts, and chunks of 32 of all but the tiles.
struct Regions {
    int ns, nb, nr, live, cs, cr, ct;
    __device__ __forceinline__ Regions(const TreeArgs& a, int b) {
        live = a.n_live ? min(max(uniform(a.n_live[b]), 0), a.n_draft) : a.n_draft;
        const int len = max(uniform(a.c.seq_len[b]), 0);
        ns = min(len, a.n_sink);
        nr = (len - ns) % kG;
        nb = min((len - ns) / kG, a.c.max_blocks);
        cs = (ns + kRC - 1) / kRC;
        cr = (nr + kRC - 1) / kRC;
        ct = (live + kRC - 1) / kRC;
    }
    __device__ __forceinline__ int units() const { return nb + cs + cr + ct; }
    // workgroups that share the sequence: a shorter one takes fewer, with as much to do for each
    __device__ __forceinline__ int parts(const TreeArgs& a) const { return a.n_wg == 1 ? 1 : min(a.n_wg, uniform((units() + a.share - 1) / a.share)); }
};

// What a wave of a workgroup works on.
struct Place {
    int b, kh, r0, rows;  // first query row of the chunk and rows in all: row r is draft r / g, head kh g + r % g
    int live;
    int64_t stream;
};

__device__ __forceinline__ bool row_of(const TreeArgs& a, const Place& p, int r, int& draft, int& head) {
    r += p.r0;
    draft = r / a.g;
    head = p.kh * a.g + r % a.g;
    return r < p.rows && draft < p.live;
}

// Waves of a workgroup share 16 NB query rows and take even shares of the sequence's tiles and chunks.
// Lane (G, n) = (l / 16, l % 16) holds column n, so query rows n and 16 + n.
template <int BITS, int CMP, int PREC, int NB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, 8))) void k_tree(TreeArgs a) {
    extern __shared__ __align__(16) unsigned char dyn_lds[];
    TreeSmem<PREC, NB, WAVES>& sm = *reinterpret_cast<TreeSmem<PREC, NB, WAVES>*>(dyn_lds);
    constexpr int WORDS = 4 * BITS;      // code words per lane, half tile and K or V
    constexpr float kUnitK = kCodeUnit<BITS, PREC, KVARN_KEYS>, kUnitV = kCodeUnit<BITS, PREC, KVARN_VALUES>;
    constexpr float kMid = (float)(1 << (BITS - 1));  // PREC 2: codes are taken around it
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l = threadIdx.x & 63, G = l >> 4, n = l & 15;
    // Workgroup ids go round the 8 XCDs.  The row chunks of a part of a stream, which read the same tiles, follow
    // one another on one XCD and meet in its L2; the parts of a stream go round the XCDs, since those of a short
    // sequence behind its first few have nothing to do.
    const uint32_t xcd = blockIdx.x & 7, n_kv = (uint32_t)a.c.n_kv, eighth = ((uint32_t)a.c.batch * n_kv + 7) / 8;
    const uint32_t j = blockIdx.x >> 3, part = uniform(j / (uint32_t)a.n_chunk);
    const int chunk = (int)(j - part * (uint32_t)a.n_chunk);
    const int wgi = a.n_wg > 1 ? uniform((int)(part / eighth)) : 0;
    const uint32_t stream = (part - (uint32_t)wgi * eighth) * 8 + ((xcd - (uint32_t)wgi) & 7);
    if (stream >= (uint32_t)a.c.batch * n_kv) return;
    Place pl;
    const int place = uniform((int)(stream / n_kv));
    pl.b = a.order ? uniform(sequence_of_rank(a.c.seq_len, a.c.batch, place, l)) : place;
    pl.kh = (int)(stream - (uint32_t)place * n_kv);
    pl.stream = (int64_t)pl.b * n_kv + pl.kh;
    const Regions rg(a, pl.b);
    pl.live = rg.live;
    pl.r0 = chunk * 16 * NB;
    pl.rows = a.n_draft * a.g;
    const int parts = rg.parts(a);
    if (pl.r0 >= pl.live * a.g || wgi >= parts) return;
    const int ns = rg.ns, nr = rg.nr, nb = rg.nb, cs = rg.cs, cr = rg.cr;
    // (at most 2^24 + 38 units and 128 waves)
    const uint32_t units = (uint32_t)rg.units(), waves = (uint32_t)(parts * WAVES), me = (uint32_t)(wgi * WAVES + wave);
    const int u0 = uniform((int)(units * me / waves)), u1 = uniform((int)(units * (me + 1) / waves));

    // ---- the first tile ---------------------------------------------------------------------------
    // Asked for before the queries are seen to, so that it is there when they are.
    int t0 = min(u0, nb);
    const int t1 = min(u1, nb);
    if (a.c.block_table && t0 < t1) {
        // Every wave looks at all ids of the sequence, so that its body is left out as a whole, whatever the plan.
        bool bad = false;
        for (int i = l; i < nb; i += 64) {
            const int id = a.c.block_table[(size_t)pl.b * a.c.max_blocks + i];
            bad |= id < 0 || id >= a.c.n_phys;
        }
        if (__any(bad)) {
            if (l == 0 && a.c.err_word) __hip_atomic_fetch_or(a.c.err_word, 2u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            t0 = t1;
        }
    }
    const size_t tb = tile_bytes(BITS, CMP);
    auto tile_at = [&](int t) -> size_t {
        const int64_t id = a.c.block_table ? (int64_t)a.c.block_table[(size_t)pl.b * a.c.max_blocks + t] * a.c.n_kv + pl.kh
                                           : pl.stream * a.c.max_blocks + t;
        return uniform((size_t)id * tb);
    };
    auto k_tile = [&](size_t at) { return Tile(static_cast<const uint8_t*>(a.c.k_body) + at, (uint32_t)tb); };
    auto v_tile = [&](size_t at) { return Tile(static_cast<const uint8_t*>(a.c.v_body) + at, (uint32_t)tb); };
    constexpr int kAuxAt = 2048 * BITS;
    // With 32 rows at 4 bits there are registers for one of the two code regions: the values' follow the keys' into
    // the same ones, asked for when the logits are through (else a tile ahead).
    constexpr bool ONE = BITS == 4 && NB == 2;
    uint32_t kw[2][WORDS], vw_[2][ONE ? 1 : WORDS];
    uint32_t(&vw)[2][WORDS] = reinterpret_cast<uint32_t(&)[2][WORDS]>(*(ONE ? &kw[0][0] : &vw_[0][0]));
    auto load_codes = [&](const Tile& t, uint32_t(&w)[2][WORDS]) {
#pragma unroll
        for (int i = 0; i < 2 * BITS; ++i) {
            const v4u x = t.load16(16u * l, 1024 * i);
            uint32_t* d = &w[i / BITS][4 * (i % BITS)];
            d[0] = x[0], d[1] = x[1], d[2] = x[2], d[3] = x[3];
        }
    };
    RawAux<CMP> ka, va;
    if (t0 < t1) {
        const size_t at = tile_at(t0);
        ka.load(k_tile(at), kAuxAt, l);
        load_codes(k_tile(at), kw);
        va.load(v_tile(at), kAuxAt, l);
        if (!ONE) load_codes(v_tile(at), vw);
    }

    // Keys of the next chunk are asked for ahead where there are registers for it.
    constexpr bool AHEAD = NB == 1;
    // ---- chunks: where they lie and how they are loaded ----------------------------------------------
    const int c0 = max(u0, nb) - nb, c1 = max(u1, nb) - nb;
    // A chunk's rows first .. last - 1 of a region whose row r begins at element base + r * stride of k and v.
    struct Chunk {
        const void *k, *v;
        int64_t base;
        uint32_t stride;  // (64 rows fit 32 bits in bytes)
        int first, last;
        bool drafts, f32;
    };
    auto chunk_at = [&](int c) {
        Chunk x;
        x.drafts = c >= cs + cr;
        x.f32 = x.drafts && !a.kv_bf16;
        x.first = (c < cs ? c : x.drafts ? c - cs - cr : c - cs) * kRC;
        x.last = min(x.first + kRC, c < cs ? ns : x.drafts ? pl.live : nr);
        x.base = x.drafts ? (int64_t)pl.b * a.n_draft * a.kv_stride + (int64_t)pl.kh * kD : pl.stream * (c < cs ? a.n_sink : kG) * kD;
        x.stride = x.drafts ? (uint32_t)a.kv_stride : kD;
        x.k = x.drafts ? a.k : c < cs ? a.c.k_sink : a.c.k_resid;
        x.v = x.drafts ? a.v : c < cs ? a.c.v_sink : a.c.v_resid;
        return x;
    };
    // keys of token 16 tau + n, channels 32 k + 8 G ..
    v4u kr[2][4];
    auto key_at = [&](const Chunk& x, int tau, int k) { return min(x.first + 16 * tau + n, x.last - 1) * x.stride + 8u * G + 32u * k; };
    auto load_keys = [&](const Chunk& x) {  // (fp32 rows are loaded where they are used)
        if (x.f32) return;
        const uint16_t* f = static_cast<const uint16_t*>(x.k) + x.base;
#pragma unroll
        for (int tau = 0; tau < 2; ++tau)
#pragma unroll
            for (int k = 0; k < 4; ++k) kr[tau][k] = *reinterpret_cast<const v4u*>(f + key_at(x, tau, k));
    };

    // ---- queries into LDS -----------------------------------------------------------------------
    // Eight lanes a row, 16 channels each: four stages of the rotation in registers, three by lane moves.
    float q_up, q_down;  // the power of two of the largest query value, and its inverse
    bool uneven;         // whether rows far below that largest one are scaled up to it
    float apart_k;       // kApartK, or infinity where that power is not its own: all tiles go by their elements then
    {
        float x[16], top = 0.f;
        const int r = 8 * wave + (l >> 3), part = l & 7;
        int draft, head;
        const bool ok = row_of(a, pl, min(r, 16 * NB - 1), draft, head);
        const int64_t at = ((int64_t)pl.b * a.n_draft + (ok ? draft : 0)) * a.q_stride + (int64_t)(ok ? head : 0) * kD + 16 * part;
        if (a.q_bf16) {
            const uint4* f = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + at);
            const uint4 u[2] = {f[0], f[1]};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t w[4] = {u[e].x, u[e].y, u[e].z, u[e].w};
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    x[8 * e + 2 * d] = __uint_as_float(w[d] << 16);
                    x[8 * e + 2 * d + 1] = __uint_as_float(w[d] & 0xFFFF0000u);
                }
            }
        } else {
            const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 w = f[e];
                x[4 * e] = w.x, x[4 * e + 1] = w.y, x[4 * e + 2] = w.z, x[4 * e + 3] = w.w;
            }
        }
        if (r < 16 * NB) {
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
                uint32_t w[4][PREC + 1];
#pragma unroll
                for (int d = 0; d < 4; ++d) split_bf16<PREC + 1>(ok ? x[e + 2 * d] : 0.f, ok ? x[e + 2 * d + 1] : 0.f, w[d]);
#pragma unroll
                for (int p = 0; p <= PREC; ++p)
                    if (p == 0 || !a.q_bf16) *reinterpret_cast<v4u*>(&sm.plain[p][r][8 * part + e / 2]) = v4u{w[0][p], w[1][p], w[2][p], w[3][p]};
            }
        }
        if (a.rotate) {
#pragma unroll
            for (int step = 1; step < 16; step *= 2) stage(x, step);
            const float s1 = (l & 1) ? -1.f : 1.f, s2 = (l & 2) ? -1.f : 1.f, s4 = ((l & 4) ? -1.f : 1.f) * kInvSqrt128;
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = s1 * x[e] + lane_xor<1>(x[e], l);
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = s2 * x[e] + lane_xor<2>(x[e], l);
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = s4 * x[e] + kInvSqrt128 * lane_xor<4>(x[e], l);
        }
        if (r < 16 * NB) {
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<float4*>(&sm.q[r][16 * part + e]) = ok ? make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(x[e]));
        if (!(ok && top < INFINITY)) top = 0.f;  // (a row with an infinity or a NaN does not count)
        float row = fmaxf(top, fdpp_x1(top));
        row = fmaxf(row, fdpp_x2(row));
        row = fmaxf(row, fdpp_half_mirror(row));
        float steep = max_over_wave(row > 0.f ? inverse(power_of(row)) : 0.f);
        top = max_over_wave(top);
        if (l == 0) sm.top[wave] = top, sm.steep[wave] = steep;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, sm.top[w]), steep = fmaxf(steep, sm.steep[w]);
        q_up = uniform(power_of(top));
        apart_k = uniform(top >= kMost || (top > 0.f && top < kLeast) ? INFINITY : kApartK<PREC>);
        q_down = uniform(inverse(q_up));
        // The halves carry a row with all its bits down to 2^-12 of the largest one; a smaller one goes in at that one's height.
        uneven = uniform((int)(q_up * steep > 0x1p12f));
        if (uneven) {
            const float own = row > 0.f ? power_of(row) : q_up;
            if (r < 16 * NB) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (ok) sm.q[r][16 * part + e] = x[e] * inverse(own) * q_up;
                if (part == 0) sm.low[r] = own * q_down;
            }
            __syncthreads();
        }
    }

    v4f o[NB][8];
    float m[NB], sum[NB];
#pragma unroll
    for (int rb = 0; rb < NB; ++rb) {
        m[rb] = kNone;
        sum[rb] = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) o[rb][w] = v4f{0.f, 0.f, 0.f, 0.f};
    }

    // ---- body tiles --------------------------------------------------------------------------------
    if (t0 < t1) {
        float(&aux)[7][kD] = *reinterpret_cast<float(*)[7][kD]>(sm.own[wave]);  // a' b s2' of K, log2 a, 1 / a, b / a, s2' of V
        // The powers of two of a tile's steps x, and of offsets y of keys (PREC 2: to codes less their middle) beside which they are lost.
        auto power_of_keys = [&](float2 x, float2 y) {
            float top = fmaxf(fabsf(x.x), fabsf(x.y));
            if constexpr (PREC == 2) top = fmaxf(top, 0x1p-12f * fmaxf(fabsf(y.x), fabsf(y.y)));
            return power_of(max_over_wave(top));
        };
        auto power_of_values = [&](float2 x) { return power_of(max_over_wave(fmaxf(fabsf(x.x), fabsf(x.y)))); };
        // Whether a group of the tile whose codes are w has no range: all its codes are 0.
        auto zero_range = [&](const uint32_t(&w)[2][WORDS], bool keys) {
            constexpr int W = BITS / 2;
            bool zero = false;
#pragma unroll
            for (int g = 0; g < 2 * W; ++g) {  // keys' channels by kappa, values' tokens by half tile: 16 per lane group
                const int which = g / W, j = g % W;
                uint32_t x = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) x |= keys ? w[i >> 2][(2 * (i & 3) + which) * W + j] : w[which][i * W + j];
                x |= dpp_x1(x);
                x |= dpp_x2(x);
                x |= dpp_half_mirror(x);
                x |= dpp_mirror(x);
                x |= x >> 1;
                if (BITS == 4) x |= x >> 2;
                constexpr uint32_t kOnes = BITS == 2 ? 0x55555555u : 0x11111111u;
                zero |= (x & kOnes) != kOnes;
            }
            return (bool)__any(zero);
        };
        bool left = false;  // tiles that are left for the loop behind this one
        const float s_scale = uniform(a.scale_log2 * q_up * (0x1p-10f * kUnitK));
#pragma unroll 1
        for (int t = t0; t < t1; ++t) {
            const size_t here = ONE ? tile_at(t) : 0, next = tile_at(min(t + 1, t1 - 1));
            // The scales go to LDS with everything folded in that the sums carry.  Those of keys are brought to
            // [1, 2) by the power of two of the largest |a| (PREC 2: or of 2^-12 of the largest |b|, beside which a
            // smaller a is lost).
            float k_down, r_up, sum_up, b_up;  // that power's inverse; the powers taken out of b / a and 1 / a
            bool far = false;                  // steps too far apart for one power of two
            {
                // What a lane knows of its entries is formed anew for each tile: there are no registers to keep it.
                int e = l;
                asm volatile("" : "+v"(e));
                const int k_plane = plane_shift<BITS, PREC, KVARN_KEYS>((e & 7) >> 1), v_plane = plane_shift<BITS, PREC, KVARN_VALUES>((e & 31) >> 3);
                const float k_part = ldexpf(1.f, k_plane), v_part = ldexpf(1.f, v_plane), k_scale = ldexpf(q_down, 10 - k_plane);
                // Entries 2 l and 2 l + 1 of a row of `more`: one half of two dwords that follow one another.
                const int at_more = 4 * ((((e >> 5) * 2 + ((e >> 2) & 1)) * 4 + ((e >> 3) & 3)) * 4 + ((e >> 1) & 1) * 2) + 2 * (e & 1);
                const int at_more_v = 4 * ((((e >> 5) * 2 + ((e >> 4) & 1)) * 4 + ((e >> 1) & 3)) * 4 + ((e >> 3) & 1) * 2) + 2 * (e & 1);
                float2 x, y, z;
                ka.get(x, y, z);
                if constexpr (PREC == 2) y = make_float2(y.x + kMid * x.x, y.y + kMid * x.y);
                const float k_up = power_of_keys(x, y);
                far = __any(fminf(x.x, x.y) < apart_k * k_up || k_up >= kMost);
                k_down = inverse(k_up);
                const float f = k_down * k_scale, g = k_up * s_scale;
                wave_sync();
                if constexpr (PREC == 1) {
                    const float2 r = make_float2(y.x * __builtin_amdgcn_rcpf(x.x) * k_part, y.y * __builtin_amdgcn_rcpf(x.y) * k_part);
                    r_up = power_of(max_over_wave(fmaxf(fabsf(r.x), fabsf(r.y))));
                    const float down = inverse(r_up) * 0x1p12f;
                    put_halves(sm.more[wave], 0, at_more, r.x * down, r.y * down);
                    r_up *= 0x1p-12f / kUnitK;
                } else {
                    *reinterpret_cast<float2*>(&aux[1][2 * l]) = y;
                }
                *reinterpret_cast<float2*>(&aux[0][2 * l]) = make_float2(x.x * f, x.y * f);
                *reinterpret_cast<float2*>(&aux[2][2 * l]) = make_float2(z.x * g, z.y * g);
                va.get(x, y, z);
                if constexpr (PREC == 2) y = make_float2(y.x + kMid * x.x, y.y + kMid * x.y);
                const float v_up = power_of_values(x);
                far |= __any(fminf(x.x, x.y) < kApartV<PREC> * v_up || v_up > kMostV);
                const float v_down = inverse(v_up);
                const float2 r = make_float2(__builtin_amdgcn_rcpf(x.x) * v_part, __builtin_amdgcn_rcpf(x.y) * v_part);
                const float2 br = make_float2(y.x * r.x, y.y * r.y);
                *reinterpret_cast<float2*>(&aux[3][2 * l]) = make_float2(__builtin_amdgcn_logf(x.x * v_down) - v_plane, __builtin_amdgcn_logf(x.y * v_down) - v_plane);
                if constexpr (PREC == 1) {
                    // 1 / a is up to 2^6 of the largest a's, times the place's 2^BITS
                    constexpr float kDown = 0.5f / (1 << BITS);
                    const float s_down = v_up * kDown;
                    put_halves(sm.more[wave], 2, at_more_v, r.x * s_down, r.y * s_down);
                    sum_up = 1.f / kDown;
                    b_up = power_of(max_over_wave(fmaxf(fabsf(br.x), fabsf(br.y))));
                    const float down = inverse(b_up) * 0x1p12f;
                    put_halves(sm.more[wave], 4, at_more_v, br.x * down, br.y * down);
                    b_up *= 0x1p-12f / kUnitV;
                } else {
                    *reinterpret_cast<float2*>(&aux[4][2 * l]) = make_float2(r.x * v_up, r.y * v_up);
                    *reinterpret_cast<float2*>(&aux[5][2 * l]) = br;
                }
                *reinterpret_cast<float2*>(&aux[6][2 * l]) = make_float2(z.x * kUnitV * v_up, z.y * kUnitV * v_up);
                wave_sync();
            }
            if constexpr (PREC == 2) far = far || zero_range(kw, true) || zero_range(vw, false);
            if (far) {
                left = true;
                load_codes(k_tile(next), kw);
                ka.load(k_tile(next), kAuxAt, l);
                va.load(v_tile(next), kAuxAt, l);
                if (!ONE) load_codes(v_tile(next), vw);
                continue;
            }

            // logits: token 64 sg + 16 tau + 4 G + i, rows 16 rb + n, in s[rb][4 sg + tau][i]
            v4f s[NB][8];
            float beta[NB];
            v4u qa[NB][2][2][PREC];  // (q a) operands [rb][kappa][half]
#pragma unroll
            for (int rb = 0; rb < NB; ++rb) beta[rb] = 0.f;
#pragma unroll
            for (int kap = 0; kap < 2; ++kap)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float4 fa[2], fb[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int c = 64 * kap + 16 * G + 8 * half + 4 * e;
                        fa[e] = *reinterpret_cast<const float4*>(&aux[0][c]);
                        if (PREC == 2) fb[e] = *reinterpret_cast<const float4*>(&aux[1][c]);
                    }
#pragma unroll
                    for (int rb = 0; rb < NB; ++rb)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float4 q = *reinterpret_cast<const float4*>(&sm.q[16 * rb + n][64 * kap + 16 * G + 8 * half + 4 * e]);
                            if (PREC == 2) beta[rb] += q.x * fb[e].x + q.y * fb[e].y + q.z * fb[e].z + q.w * fb[e].w;
                            uint32_t w0[PREC], w1[PREC];
                            split_pair<PREC>(q.x * fa[e].x, q.z * fa[e].z, w0);
                            split_pair<PREC>(q.y * fa[e].y, q.w * fa[e].w, w1);
#pragma unroll
                            for (int p = 0; p < PREC; ++p) {
                                qa[rb][kap][half][p][2 * e] = w0[p];
                                qa[rb][kap][half][p][2 * e + 1] = w1[p];
                            }
                        }
                }
#pragma unroll
            for (int rb = 0; rb < NB; ++rb) {
                float x = 0.f;
                if constexpr (PREC == 1) {  // rows n of A: b / a (n even) and the rest of it (n odd)
                    v4f y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kap = 0; kap < 2; ++kap)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
                            y = mfma_f16(*reinterpret_cast<const v4u*>(&sm.more[wave][n & 1][16 * (2 * kap + half) + 4 * G]), qa[rb][kap][half][0], y);
                    x = (y[0] + y[1]) * r_up;
                } else {
                    beta[rb] = across_groups(beta[rb], add2) * (k_down * q_down * (0x1p10f / kUnitK));
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) s[rb][k] = v4f{x, x, x, x};
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int kap = 0; kap < 2; ++kap)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const v4u c = code_operand<BITS, PREC, KVARN_KEYS>(&kw[k >> 2][(2 * (k & 3) + kap) * (BITS / 2)], half);
#pragma unroll
                        for (int p = 0; p < PREC; ++p)
#pragma unroll
                            for (int rb = 0; rb < NB; ++rb) s[rb][k] = mfma_f16(c, qa[rb][kap][half][p], s[rb][k]);
                    }
            if (ONE) load_codes(v_tile(here), vw);
            else load_codes(k_tile(next), kw);
            ka.load(k_tile(next), kAuxAt, l);
            va.load(v_tile(next), kAuxAt, l);

            if (uneven) {
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) {
                    const float low = sm.low[16 * rb + n];
                    if (PREC == 2) beta[rb] *= low;
#pragma unroll
                    for (int k = 0; k < 8; ++k) s[rb][k] *= low;
                }
            }

            // softmax, with p a as operands
            float gamma[NB], part[NB];
            v4u pa[NB][2][2][PREC];  // [rb][sg][half]
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const v4f z = *reinterpret_cast<const v4f*>(&aux[2][64 * (k >> 2) + 16 * (k & 3) + 4 * G]);
                const v4f la = *reinterpret_cast<const v4f*>(&aux[3][64 * (k >> 2) + 16 * (k & 3) + 4 * G]);
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) s[rb][k] = (PREC == 2 ? s[rb][k] + beta[rb] : s[rb][k]) * z + la;
            }
#pragma unroll
            for (int rb = 0; rb < NB; ++rb) {
                float top = s[rb][0][0];
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, s[rb][k][i]);
                raise(across_groups(top, max2), m[rb], sum[rb], o[rb]);
                gamma[rb] = part[rb] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v4f ra, ba;
                if constexpr (PREC == 2) {
                    ra = *reinterpret_cast<const v4f*>(&aux[4][64 * (k >> 2) + 16 * (k & 3) + 4 * G]);
                    ba = *reinterpret_cast<const v4f*>(&aux[5][64 * (k >> 2) + 16 * (k & 3) + 4 * G]);
                }
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) {
                    float p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[i] = exp2_fast(s[rb][k][i] - m[rb]);
                        if constexpr (PREC == 2) {
                            part[rb] += p[i] * ra[i];
                            gamma[rb] += p[i] * ba[i];
                        }
                    }
                    uint32_t w0[PREC], w1[PREC];
                    split_pair<PREC>(p[0], p[2], w0);
                    split_pair<PREC>(p[1], p[3], w1);
#pragma unroll
                    for (int x = 0; x < PREC; ++x) {
                        pa[rb][k >> 2][(k & 3) >> 1][x][2 * (k & 1)] = w0[x];
                        pa[rb][k >> 2][(k & 3) >> 1][x][2 * (k & 1) + 1] = w1[x];
                    }
                }
            }
#pragma unroll
            for (int rb = 0; rb < NB; ++rb) {
                if constexpr (PREC == 1) {  // rows n of A: 1 / a, its rest, b / a, its rest, by n % 4
                    v4f y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int sg = 0; sg < 2; ++sg)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
                            y = mfma_f16(*reinterpret_cast<const v4u*>(&sm.more[wave][2 + (n & 3)][16 * (2 * sg + half) + 4 * G]), pa[rb][sg][half][0], y);
                    sum[rb] += (y[0] + y[1]) * sum_up;
                    gamma[rb] = (y[2] + y[3]) * b_up;
                } else {
                    sum[rb] += across_groups(part[rb], add2);
                    gamma[rb] = across_groups(gamma[rb], add2) * (1.f / kUnitV);
                }
            }
            // sums: channel 16 w + 4 G + i in o[rb][w][i]
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                v4f y[NB];
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) y[rb] = PREC == 2 ? v4f{0.f, 0.f, 0.f, 0.f} : v4f{gamma[rb], gamma[rb], gamma[rb], gamma[rb]};
#pragma unroll
                for (int sg = 0; sg < 2; ++sg)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const v4u c = code_operand<BITS, PREC, KVARN_VALUES>(&vw[sg][w * (BITS / 2)], half);
#pragma unroll
                        for (int p = 0; p < PREC; ++p)
#pragma unroll
                            for (int rb = 0; rb < NB; ++rb) y[rb] = mfma_f16(c, pa[rb][sg][half][p], y[rb]);
                    }
                const v4f z = *reinterpret_cast<const v4f*>(&aux[6][16 * w + 4 * G]);
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) o[rb][w] += (PREC == 2 ? y[rb] + gamma[rb] : y[rb]) * z;
            }
            if (ONE) load_codes(k_tile(next), kw);
            else load_codes(v_tile(next), vw);
        }
        // Tiles of steps far apart: their elements code a + b in 32 bits, and products of pieces of bf16, whose exponents
        // go as far, as for the chunks below, 32 tokens at a time.  Behind the others, so that these have the registers.  A tile takes
        // four to five times as long as there: 32 sequences of 32k, 64 drafts, bf16: 6256 us with all tiles here, 1530 with one in
        // 64, 1353 with none; 4 of 8k, group 16, 4 bits, fp32: 253, 76 and 72.
#pragma unroll 1
        for (int t = left ? t0 : t1; t < t1; ++t) {
            constexpr int NP = PREC + 1, W = BITS / 2;
            constexpr uint32_t kMask = BITS == 2 ? 0x03u : 0x0Fu;
            // (What follows from the lane is formed here: there are no registers to keep it over the loop above.)
            int lane = threadIdx.x & 63;
            asm volatile("" : "+v"(lane));
            const int G = lane >> 4, n = lane & 15;
            const size_t at = tile_at(t);
            const Tile kt = k_tile(at), vt = v_tile(at);
            ka.load(kt, kAuxAt, lane);
            va.load(vt, kAuxAt, lane);
            float2 x, y, z, vx, vy, vz;
            ka.get(x, y, z);
            va.get(vx, vy, vz);
            const float k_up = power_of_keys(x, PREC == 2 ? make_float2(y.x + kMid * x.x, y.y + kMid * x.y) : y);
            const float v_up = power_of_values(vx), k_min = fminf(x.x, x.y), v_min = fminf(vx.x, vx.y);
            bool far = __any(k_min < apart_k * k_up || k_up >= kMost || v_min < kApartV<PREC> * v_up || v_up > kMostV);
            if constexpr (PREC == 2) {
                load_codes(kt, kw);
                load_codes(vt, vw);
                far = far || zero_range(kw, true) || zero_range(vw, false);
            }
            if (!far) continue;
            wave_sync();
            *reinterpret_cast<float2*>(&aux[0][2 * lane]) = x;
            *reinterpret_cast<float2*>(&aux[1][2 * lane]) = y;
            *reinterpret_cast<float2*>(&aux[2][2 * lane]) = make_float2(z.x * a.scale_log2, z.y * a.scale_log2);
            *reinterpret_cast<float2*>(&aux[3][2 * lane]) = vx;
            *reinterpret_cast<float2*>(&aux[4][2 * lane]) = vy;
            *reinterpret_cast<float2*>(&aux[5][2 * lane]) = vz;
            wave_sync();
            auto word = [&](const Tile& tile, int sg, int i) { return tile.load4(16u * lane + 1024u * (sg * BITS + i / 4) + 4u * (i % 4), 0); };
            // Eight elements, codes e at position `first + e / 4` of a unit: pieces of pairs that follow one another.
            auto elements = [&](uint32_t w, int first, const float* sa, const float* sb, v4u(&out)[NP]) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const uint32_t c = w >> (BITS * ((BITS == 2 ? first : 0) + e / 4) + 8 * (e % 4));
                    const float2 fa = *reinterpret_cast<const float2*>(sa + e), fb = *reinterpret_cast<const float2*>(sb + e);
                    uint32_t p[NP];
                    split_bf16<NP>((float)(c & kMask) * fa.x + fb.x, (float)(c >> 8 & kMask) * fa.y + fb.y, p);
#pragma unroll
                    for (int i = 0; i < NP; ++i) out[i][e / 2] = p[i];
                }
            };
            // pieces i and j of the factors, as far as they count
            auto products = [&](const v4u(&x)[NP], const v4u(&y)[NP], v4f& to) {
#pragma unroll
                for (int i = NP - 1; i >= 0; --i)
#pragma unroll
                    for (int j = NP - 1 - i; j >= 0; --j) to = mfma_bf16(x[i], y[j], to);
            };
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                const int sg = c >> 1, half = c & 1, first = 32 * c;
                v4f s[NB][2];
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) s[rb][0] = s[rb][1] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int kh = 0; kh < 4; ++kh) {  // channels 64 (kh / 2) + 16 G + 8 (kh % 2) ..
                    const int from = 64 * (kh >> 1) + 16 * G + 8 * (kh & 1);
                    v4u q[NB][NP], k[NP];
#pragma unroll
                    for (int rb = 0; rb < NB; ++rb)
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            const float2 f = *reinterpret_cast<const float2*>(&sm.q[16 * rb + n][from + e]);
                            uint32_t p[NP];
                            split_bf16<NP>(f.x, f.y, p);
#pragma unroll
                            for (int i = 0; i < NP; ++i) q[rb][i][e / 2] = p[i];
                        }
#pragma unroll
                    for (int tau = 0; tau < 2; ++tau) {
                        const int unit = 2 * (2 * half + tau) + (kh >> 1);
                        elements(word(kt, sg, unit * W + (BITS == 4 ? kh & 1 : 0)), 2 * (kh & 1), &aux[0][from], &aux[1][from], k);
#pragma unroll
                        for (int rb = 0; rb < NB; ++rb) products(k, q[rb], s[rb][tau]);
                    }
                }
                v4u pv[NB][NP];
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) {
                    float top = kNone, part = 0.f;
#pragma unroll
                    for (int tau = 0; tau < 2; ++tau) {
                        s[rb][tau] *= *reinterpret_cast<const v4f*>(&aux[2][first + 16 * tau + 4 * G]);
                        if (uneven) s[rb][tau] *= sm.low[16 * rb + n];
#pragma unroll
                        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[rb][tau][i]);
                    }
                    raise(across_groups(top, max2), m[rb], sum[rb], o[rb]);
#pragma unroll
                    for (int tau = 0; tau < 2; ++tau)
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            const float p0 = exp2_fast(s[rb][tau][i] - m[rb]), p1 = exp2_fast(s[rb][tau][i + 1] - m[rb]);
                            part += p0 + p1;
                            uint32_t p[NP];
                            split_bf16<NP>(p0, p1, p);
#pragma unroll
                            for (int x = 0; x < NP; ++x) pv[rb][x][2 * tau + i / 2] = p[x];
                        }
                    sum[rb] += across_groups(part, add2);
                }
                // tokens first + 16 (e / 4) + 4 G + e % 4 of channels 16 w + n
                float va[8], vb[8];
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    *reinterpret_cast<v4f*>(va + e) = *reinterpret_cast<const v4f*>(&aux[3][first + 4 * e + 4 * G]);
                    *reinterpret_cast<v4f*>(vb + e) = *reinterpret_cast<const v4f*>(&aux[4][first + 4 * e + 4 * G]);
                }
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    v4u v[NP];
                    elements(word(vt, sg, w * W + (BITS == 4 ? half : 0)), 2 * half, va, vb, v);
                    const v4f s2 = *reinterpret_cast<const v4f*>(&aux[5][16 * w + 4 * G]);
#pragma unroll
                    for (int rb = 0; rb < NB; ++rb) {
                        v4f y{0.f, 0.f, 0.f, 0.f};
                        products(v, pv[rb], y);
                        o[rb][w] += y * s2;
                    }
                }
            }
        }
    }

    if (AHEAD && c0 < c1) load_keys(chunk_at(c0));  // asked for before the rotation

    // ---- back from the rotated domain ----------------------------------------------------------------
    // Channel bits 0, 1 (i) and 4, 5, 6 (w) are register bits, 2 and 3 lane bits.  The row swaps exchange a
    // lane bit with register bit 0 of w: afterwards lane group G holds channels 8 G .. 8 G + 7 of each 32.
    // They are put where the chunks' products have them, channel 32 mm + 8 G + 2 i + e in o[rb][2 mm + e][i].
    if (t0 < t1) {
#pragma unroll
        for (int rb = 0; rb < NB; ++rb) {
            if (a.rotate) {
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    v4f x = o[rb][w];
                    x = v4f{x[0] + x[1], x[0] - x[1], x[2] + x[3], x[2] - x[3]};
                    o[rb][w] = v4f{x[0] + x[2], x[1] + x[3], x[0] - x[2], x[1] - x[3]};
                }
#pragma unroll
                for (int d = 1; d < 8; d *= 2)
#pragma unroll
                    for (int w = 0; w < 8; ++w)
                        if (!(w & d)) {
                            const v4f x = o[rb][w], y = o[rb][w + d];
                            o[rb][w] = x + y;
                            o[rb][w + d] = x - y;
                        }
            }
#pragma unroll
            for (int w = 0; w < 8; w += 2) {
                float z[8];  // channels 32 (w / 2) + 8 G + ..
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[rb][w][i]), __float_as_uint(o[rb][w + 1][i]), false, false);
                    const float u = __uint_as_float(x[0]), v = __uint_as_float(x[1]);
                    const float u1 = a.rotate ? u + v : u, v1 = a.rotate ? u - v : v;
                    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(u1), __float_as_uint(v1), false, false);
                    const float u2 = __uint_as_float(y[0]), v2 = __uint_as_float(y[1]);
                    z[i] = a.rotate ? (u2 + v2) * kInvSqrt128 : u2;
                    z[4 + i] = a.rotate ? (u2 - v2) * kInvSqrt128 : v2;
                }
                o[rb][w] = v4f{z[0], z[2], z[4], z[6]};
                o[rb][w + 1] = v4f{z[1], z[3], z[5], z[7]};
            }
        }
    }

    // ---- chunks of 32 bf16 rows ----------------------------------------------------------------------
    if (c0 < c1) {
        constexpr int NP = PREC + 1;  // bf16 pieces of fp32 queries and of probabilities
        const int qp = a.q_bf16 ? 1 : NP;
        uint64_t sees[NB];
#pragma unroll
        for (int rb = 0; rb < NB; ++rb) {
            int draft, head;
            const bool ok = row_of(a, pl, 16 * rb + n, draft, head);
            sees[rb] = !ok ? 0 : a.mask ? a.mask[(int64_t)pl.b * a.n_draft + draft] : draft >= 63 ? ~0ull : (2ull << draft) - 1;
        }
#pragma unroll 1
        for (int c = c0; c < c1; ++c) {
            const Chunk ch = chunk_at(c);
            if (!AHEAD) load_keys(ch);
            const int first = ch.first, last = ch.last;
            const bool drafts = ch.drafts;
            if (ch.f32) {
                const float* f = static_cast<const float*>(ch.k) + ch.base;
#pragma unroll
                for (int tau = 0; tau < 2; ++tau)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float4* r = reinterpret_cast<const float4*>(f + key_at(ch, tau, k));
                        const float4 x = r[0], y = r[1];
                        kr[tau][k] = v4u{bf16_pair(x.x, x.y), bf16_pair(x.z, x.w), bf16_pair(y.x, y.y), bf16_pair(y.z, y.w)};
                    }
            }
            v4f s[NB][2];
#pragma unroll
            for (int rb = 0; rb < NB; ++rb) s[rb][0] = s[rb][1] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < NP; ++p)
                if (p < qp)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int rb = 0; rb < NB; ++rb) {
                            const v4u q = *reinterpret_cast<const v4u*>(&sm.plain[p][16 * rb + n][16 * k + 4 * G]);
#pragma unroll
                            for (int tau = 0; tau < 2; ++tau) s[rb][tau] = mfma_bf16(kr[tau][k], q, s[rb][tau]);
                        }
            // values of tokens 16 tau + 4 G + i, channels 32 mm + 2 n and + 1 (in the keys' registers)
            uint32_t vr[4][8];
            if (ch.f32) {
                const float* f = static_cast<const float*>(ch.v) + ch.base;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t row = min(first + 16 * (k >> 2) + 4 * G + (k & 3), last - 1) * ch.stride + 2u * n;
#pragma unroll
                    for (int mm = 0; mm < 4; ++mm) {
                        const float2 x = *reinterpret_cast<const float2*>(f + (row + 32u * mm));
                        vr[mm][k] = bf16_pair(x.x, x.y);
                    }
                }
            } else {
                const uint16_t* f = static_cast<const uint16_t*>(ch.v) + ch.base;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t row = min(first + 16 * (k >> 2) + 4 * G + (k & 3), last - 1) * ch.stride + 2u * n;
#pragma unroll
                    for (int mm = 0; mm < 4; ++mm) vr[mm][k] = *reinterpret_cast<const uint32_t*>(f + (row + 32u * mm));
                }
            }
            v4u pv[NB][NP];
#pragma unroll
            for (int rb = 0; rb < NB; ++rb) {
                float top = kNone;
#pragma unroll
                for (int tau = 0; tau < 2; ++tau)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = first + 16 * tau + 4 * G + i;
                        const bool seen = t < last && (!drafts || (sees[rb] >> (t & 63) & 1));
                        s[rb][tau][i] = seen ? s[rb][tau][i] * a.scale_log2 : -INFINITY;
                        top = fmaxf(top, s[rb][tau][i]);
                    }
                raise(across_groups(top, max2), m[rb], sum[rb], o[rb]);
                float part = 0.f;
#pragma unroll
                for (int tau = 0; tau < 2; ++tau)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = exp2_fast(s[rb][tau][i] - m[rb]);
                        s[rb][tau][i] = p;
                        part += p;
                    }
                sum[rb] += across_groups(part, add2);
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    uint32_t w[NP];
                    split_bf16<NP>(s[rb][d >> 1][2 * (d & 1)], s[rb][d >> 1][2 * (d & 1) + 1], w);
#pragma unroll
                    for (int p = 0; p < NP; ++p) pv[rb][p][d] = w[p];
                }
            }
            typedef uint16_t v2s __attribute__((ext_vector_type(2)));
            v2s most{0, 0};  // the largest magnitude's bits, in halves
#pragma unroll
            for (int mm = 0; mm < 4; ++mm)
#pragma unroll
                for (int k = 0; k < 8; ++k) most = __builtin_elementwise_max(most, __builtin_bit_cast(v2s, vr[mm][k] & 0x7FFF7FFFu));
            if (__any(most[0] >= 0x7F80 || most[1] >= 0x7F80)) {
                // An infinity or a NaN among the values: a product would spread it to rows that do not see its token and, of
                // the last row, to the places behind it (0 times infinity), and a piece of a probability may be 0 or of
                // the other sign.  One product at a time, leaving out probabilities of 0.
                float* pr = sm.own[wave];
#pragma unroll
                for (int rb = 0; rb < NB; ++rb)
#pragma unroll
                    for (int k = 0; k < 8; ++k) pr[(16 * rb + n) * kRC + 16 * (k >> 2) + 4 * G + (k & 3)] = s[rb][k >> 2][k & 3];
                wave_sync();
                for (int t = 0; t < last - first; ++t)
                    for (int rb = 0; rb < NB; ++rb) {
                        const float p = pr[(16 * rb + n) * kRC + t];
                        if (p == 0.f) continue;
#pragma unroll
                        for (int mm = 0; mm < 4; ++mm) {
                            const int64_t at = ch.base + (int64_t)(first + t) * ch.stride + 32 * mm + 8 * G;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float v = ch.f32 ? bf16_to_f32(f32_to_bf16(static_cast<const float*>(ch.v)[at + i])) : bf16_to_f32(static_cast<const uint16_t*>(ch.v)[at + i]);
                                if (rb == 0) o[0][2 * mm + (i & 1)][i >> 1] += p * v;
                                else o[NB - 1][2 * mm + (i & 1)][i >> 1] += p * v;
                            }
                        }
                    }
                wave_sync();
            } else {
#pragma unroll
                for (int mm = 0; mm < 4; ++mm)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        // A row n is channel 32 mm + 2 n + e, so lane group G's results are channels 32 mm + 8 G + 2 i + e
                        v4u va;
#pragma unroll
                        for (int d = 0; d < 4; ++d)
                            va[d] = __builtin_amdgcn_perm(vr[mm][2 * d + 1], vr[mm][2 * d], e ? 0x07060302u : 0x05040100u);
#pragma unroll
                        for (int p = 0; p < NP; ++p)
#pragma unroll
                            for (int rb = 0; rb < NB; ++rb) o[rb][2 * mm + e] = mfma_bf16(va, pv[rb][p], o[rb][2 * mm + e]);
                    }
            }
            if (AHEAD && c + 1 < c1) load_keys(chunk_at(c + 1));
        }
    }

    // ---- the waves' parts together ---------------------------------------------------------------------
    __syncthreads();  // the queries and the waves' own rows are done with
#pragma unroll
    for (int rb = 0; rb < NB; ++rb) {
        float* row = sm.o[wave][16 * rb + n];
#pragma unroll
        for (int mm = 0; mm < 4; ++mm) {
            const v4f x = o[rb][2 * mm], y = o[rb][2 * mm + 1];
            *reinterpret_cast<v4f*>(row + 32 * mm + 8 * G) = v4f{x[0], y[0], x[1], y[1]};
            *reinterpret_cast<v4f*>(row + 32 * mm + 8 * G + 4) = v4f{x[2], y[2], x[3], y[3]};
        }
        if (G == 0) {
            row[kD] = m[rb];
            row[kD + 1] = sum[rb];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int r = (int)(threadIdx.x >> 4) + 16 * i, c8 = 8 * (threadIdx.x & 15);
        int draft, head;
        if (r >= 16 * NB || !row_of(a, pl, r, draft, head)) continue;
        float top = kNone, total = 0.f, x[8] = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, sm.o[w][r][kD]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float* row = sm.o[w][r];
            // a wave that saw nothing is left out (its reference may be the common one)
            const float f = row[kD + 1] != 0.f ? exp2_fast(row[kD] - top) : 0.f;
            total += f * row[kD + 1];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += f * row[c8 + e];
        }
        if (parts > 1) {
            float* ws = a.ws + (((pl.stream * a.n_chunk + chunk) * a.n_wg + wgi) * (16 * NB) + r) * kRow;
            *reinterpret_cast<float4*>(ws + c8) = make_float4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<float4*>(ws + c8 + 4) = make_float4(x[4], x[5], x[6], x[7]);
            // (By all lanes of the row, with one value: a branch for one of them ends where its row's does, and the compiler
            // then restored a register of the next row for that one lane alone.)
            *reinterpret_cast<float2*>(ws + kD) = make_float2(top, total);
            continue;
        }
        const float inv = total != 0.f ? 1.f / total : 0.f;
        const int64_t at = ((int64_t)pl.b * a.n_draft + draft) * a.out_stride + (int64_t)head * kD + c8;
        if (a.out_bf16) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = bf16_pair(x[2 * e] * inv, x[2 * e + 1] * inv);
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + at) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            float* f = static_cast<float*>(a.out) + at;
            *reinterpret_cast<float4*>(f) = make_float4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
            *reinterpret_cast<float4*>(f + 4) = make_float4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv);
        }
    }
}

// The workgroups' parts of a query row: one wave per row, two channels per lane.  Bound by latency: the parts'
// references and sums in one round of loads, a part per lane, then their rows, eight in flight.
__global__ __launch_bounds__(256) void k_tree_merge(TreeArgs a) {
    const int l = threadIdx.x & 63;
    const uint32_t id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t row = id / (uint32_t)a.n_q;
    const int head = (int)(id - row * (uint32_t)a.n_q), b = (int)(row / (uint32_t)a.n_draft);
    if (b >= a.c.batch) return;
    const int64_t bi = row;
    const int draft = (int)(row - (uint32_t)b * (uint32_t)a.n_draft);
    const Regions rg(a, b);
    const int parts = rg.parts(a);
    if (draft >= rg.live || parts <= 1) return;  // (a single part has written its rows itself)
    const int64_t stream = (int64_t)b * a.c.n_kv + head / a.g;
    const int r = draft * a.g + head % a.g, rows = 16 * a.row_blocks;
    const float* ws = a.ws + ((stream * a.n_chunk + r / rows) * a.n_wg * rows + r % rows) * (int64_t)kRow;
    const int64_t step = (int64_t)rows * kRow;
    const float2 mine = *reinterpret_cast<const float2*>(ws + min(l, parts - 1) * step + kD);
    const bool counts = l < parts && mine.y != 0.f;
    float top = counts ? mine.x : kNone;
    for (int m = 32; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
    const float f = counts ? exp2_fast(mine.x - top) : 0.f;
    float total = f * mine.y, x0 = 0.f, x1 = 0.f;
    if (!counts) total = 0.f;
    for (int m = 32; m; m >>= 1) total += __shfl_xor(total, m);
    for (int w0 = 0; w0 < parts; w0 += 8) {
        float2 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const float2*>(ws + min(w0 + i, parts - 1) * step + 2 * l);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float g = __shfl(f, w0 + i);  // 0 behind the last part
            x0 += g * x[i].x;
            x1 += g * x[i].y;
        }
    }
    const float inv = total != 0.f ? 1.f / total : 0.f;
    const int64_t at = bi * a.out_stride + (int64_t)head * kD + 2 * l;
    if (a.out_bf16)
        *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + at) = bf16_pair(x0 * inv, x1 * inv);
    else
        *reinterpret_cast<float2*>(static_cast<float*>(a.out) + at) = make_float2(x0 * inv, x1 * inv);
}

template <int BITS, int CMP, int PREC, int NB, int WAVES>
hipError_t launch_cfg(const TreeArgs& a, hipStream_t stream) {
    const int64_t grid = ((int64_t)a.c.batch * a.c.n_kv + 7) / 8 * 8 * a.n_wg * a.n_chunk;
    if (grid * 64 * WAVES > 0xFFFFFFFFll) return hipErrorInvalidValue;
    constexpr size_t lds = sizeof(TreeSmem<PREC, NB, WAVES>);
    hipLaunchKernelGGL((k_tree<BITS, CMP, PREC, NB, WAVES>), dim3((unsigned)grid), dim3(64 * WAVES), lds, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_wg == 1) return e;
    const int64_t rows = (int64_t)a.c.batch * a.n_draft * a.n_q;  // (of grids with several parts: below 2^20)
    hipLaunchKernelGGL(k_tree_merge, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <int BITS, int CMP>
hipError_t launch_bits(const TreeArgs& a, hipStream_t stream) {
    if (!a.out_bf16) return a.waves == 8 ? launch_cfg<BITS, CMP, 2, 1, 8>(a, stream) : launch_cfg<BITS, CMP, 2, 1, 4>(a, stream);
    if (a.row_blocks == 2) return launch_cfg<BITS, CMP, 1, 2, 4>(a, stream);
    return a.waves == 8 ? launch_cfg<BITS, CMP, 1, 1, 8>(a, stream) : launch_cfg<BITS, CMP, 1, 1, 4>(a, stream);
}

TreePlan plan_of(const kvarn_cache& c, int n_sink, int n_q, int n_draft, int max_len, bool out_bf16) {
    return plan_tree(c.batch, c.n_kv, n_q, n_draft, max_len, n_sink, c.max_blocks, !out_bf16);
}

}  // namespace

size_t tree_workspace_bytes(const kvarn_cache& c, int n_sink, int n_q, int n_draft, int max_len) {
    size_t most = 0;
    for (bool bf16 : {false, true}) {
        const TreePlan p = plan_of(c, n_sink, n_q, n_draft, max_len, bf16);
        if (p.n_wg > 1) most = std::max(most, (size_t)c.batch * c.n_kv * p.n_chunk * p.n_wg * 16 * p.row_blocks * kRow * sizeof(float));
    }
    return most;
}

hipError_t launch_tree(const TreeArgs& args, hipStream_t stream) {
    TreeArgs a = args;
    const TreePlan p = plan_of(a.c, a.n_sink, a.n_q, a.n_draft, a.max_len, a.out_bf16);
    a.row_blocks = p.row_blocks;
    a.n_chunk = p.n_chunk;
    a.n_wg = p.n_wg;
    a.share = p.share;
    a.order = p.order;
    a.waves = p.waves;
    if (a.compact) return a.bits == 2 ? launch_bits<2, 1>(a, stream) : launch_bits<4, 1>(a, stream);
    return a.bits == 2 ? launch_bits<2, 0>(a, stream) : launch_bits<4, 0>(a, stream);
}

}  // namespace kvarn
