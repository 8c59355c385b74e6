// Verification of drafted tokens (include/kvarn.h, kvarn_verify_drafts).
//
// The rule with draft rows is that of k rounds of rejection, each round drawing one child from q against what the
// rounds before have left of p: w_0 = p, w_{k+1} = max(w_k / sum w_k - q, 0).  All of these are max(p - a q, 0) up to
// a factor, with a_{k+1} = a_k + S_k, S_k = sum max(p - a_k q, 0) and S_0 = 1 (divide by the factor: w_k / sum w_k =
// max(p - a_k q, 0) / S_k, and subtracting q moves a by S_k), so a round needs one number and one pass over two rows.
//
// A row is read in ranges of 1024 entries, a wave per range.  For the next token each range's sum of weights is kept:
// their running sum says in which range it lies, and only that one is read again.  Sums over a range's lanes, over
// ranges and over what a sequence does are formed in 64 bits and always in the same order.
//
// One workgroup per sequence walks its tree (k_verify).  Where that leaves most of the card idle, two launches go
// before it: k_rows forms every row's norm, by parts over the whole card, and k_rest the sums of the ranges at the
// node where the walk first needs them, by several workgroups per sequence that each walk so far.

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "lanes.hpp"

namespace kvarn {
namespace {

constexpr int kRange = 1024, kMaxRanges = KVARN_MAX_VOCAB / kRange;

// ---- 16 entries of a row per lane ----

// In pieces of 16 bytes of the lanes side by side, or (CONSECUTIVE) a lane's 16 entries one after the other.
template <int BF16, bool CONSECUTIVE>
__device__ __forceinline__ int entry(int lane, int e) {
    constexpr int N = BF16 ? 8 : 4;
    return CONSECUTIVE ? 16 * lane + e : e / N * 64 * N + lane * N + e % N;
}
template <int BF16>
struct Range {
    static constexpr int N = BF16 ? 8 : 4;
    typedef uint32_t v4 __attribute__((ext_vector_type(4)));
    typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));  // rows are aligned to an element only
    v4 w[16 / N];

    // Of a range that ends inside the row.
    template <bool CONSECUTIVE>
    __device__ __forceinline__ void load(const char* row, int r, int lane) {
        constexpr int es = BF16 ? 2 : 4;
        const char* at = row + (int64_t)r * (kRange * es);
#pragma unroll
        for (int i = 0; i < 16 / N; ++i) w[i] = *reinterpret_cast<const u4*>(at + entry<BF16, CONSECUTIVE>(lane, i * N) * es);
    }
    // Of any: entries at and behind vocab as `none` (one entry's bits).
    template <bool CONSECUTIVE>
    __device__ __forceinline__ void load_part(const char* row, int r, int vocab, int lane, uint32_t none) {
        constexpr int es = BF16 ? 2 : 4;
        const char* at = row + (int64_t)r * (kRange * es);
        const uint32_t word = BF16 ? none << 16 | none : none;
#pragma unroll
        for (int i = 0; i < 16 / N; ++i) {
            const int e0 = entry<BF16, CONSECUTIVE>(lane, i * N), n = vocab - r * kRange - e0;  // entries of this piece that are there
            w[i] = v4{word, word, word, word};
            if (n >= N) {
                w[i] = *reinterpret_cast<const u4*>(at + e0 * es);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (e >= n) continue;
                    if constexpr (BF16) {
                        const uint32_t x = reinterpret_cast<const uint16_t*>(at)[e0 + e];
                        w[i][e / 2] = e % 2 ? (w[i][e / 2] & 0xFFFFu) | x << 16 : (w[i][e / 2] & 0xFFFF0000u) | x;
                    } else {
                        w[i][e] = reinterpret_cast<const uint32_t*>(at)[e0 + e];
                    }
                }
            }
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (BF16) return __uint_as_float(e % 2 ? w[e / 8][e % 8 / 2] & 0xFFFF0000u : w[e / 8][e % 8 / 2] << 16);
        else return __uint_as_float(w[e / 4][e % 4]);
    }
};
template <int BF16, int LOGITS>
constexpr uint32_t kNone = !LOGITS ? 0u : BF16 ? 0xFF80u : 0xFF800000u;  // 0, or -infinity

// ---- moves and sums over a wave ----

template <int M>
__device__ __forceinline__ double lane_xor(double x, int l) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __float_as_uint(lane_xor<M>(__uint_as_float((uint32_t)b), l));
    const uint32_t hi = __float_as_uint(lane_xor<M>(__uint_as_float((uint32_t)(b >> 32)), l));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <class F, class T>
__device__ __forceinline__ T over_lanes(T x, int l, F f) {
    x = f(x, lane_xor<1>(x, l));
    x = f(x, lane_xor<2>(x, l));
    x = f(x, lane_xor<4>(x, l));
    x = f(x, lane_xor<8>(x, l));
    x = f(x, lane_xor<16>(x, l));
    return f(x, lane_xor<32>(x, l));
}
template <class T>
__device__ __forceinline__ T sum_lanes(T x, int l) {
    return over_lanes(x, l, [](T a, T b) { return a + b; });
}
__device__ __forceinline__ float max_lanes(float x, int l) {
    return over_lanes(x, l, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ int min_lanes(int x, int l) {
    return __float_as_int(over_lanes(__int_as_float(x), l, [](float a, float b) { return __int_as_float(min(__float_as_int(a), __float_as_int(b))); }));
}
// max(x, 0), 0 for NaN, in one instruction.
__device__ __forceinline__ float above_0(float x) { return __builtin_amdgcn_fmed3f(x, 0.f, INFINITY); }
__device__ __forceinline__ double of_lane(double x, int l) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, l), hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), l);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// The sum of 16, by halves.
template <class T>
__device__ __forceinline__ T sum16(T (&w)[16]) {
#pragma unroll
    for (int n = 8; n > 0; n /= 2)
#pragma unroll
        for (int e = 0; e < n; ++e) w[e] += w[e + n];
    return w[0];
}

// ---- weights ----

// 2^y for y from -1100 (0 there, and for NaN) to 1000 in 64 bits: 2^k 2^r with k the nearest whole number, the second by
// the polynomial of degree 8 that meets it at the zeros of the Chebyshev polynomial of degree 9 on [-1/2, 1/2] (off by 1.1e-12
// at most).  64 bits because a running sum has a border at every entry: moved by 3e-8 each, as by weights of 32 bits, the
// borders of 10^5 entries make a next token that differs from exact sums' once in some thousand draws.  (Additions and
// products run at the rate of 32 bits here.)
__device__ __forceinline__ double power(double y) {
    y = __builtin_fmax(y, -1100.0);
    const double k = __builtin_rint(y), r = y - k;
    double p = 1.3255224878668817e-06;
    p = fma(p, r, 1.5310079402249296e-05);
    p = fma(p, r, 1.5403455852453838e-04);
    p = fma(p, r, 1.3333450568000645e-03);
    p = fma(p, r, 9.618129159402558e-03);
    p = fma(p, r, 5.550410941205933e-02);
    p = fma(p, r, 2.402265069581299e-01);
    p = fma(p, r, 6.931471805459335e-01);
    p = fma(p, r, 1.0);
    return __builtin_ldexp(p, (int)k);
}
// A logit x weighs 2^(c (x - top)), c = scale * log2(e), relative to a reference that is noted with every sum.  Any does that
// keeps the sum in range: one of the larger entries.
__device__ __forceinline__ double weight(float x, float top, double c) { return power(c * ((double)x - (double)top)); }
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }
// For any reference: +infinity, which infinite entries share (but at c = NaN, where nothing has weight: power(NaN) is 0 too), and
// -infinity, where nothing has any.
__device__ __forceinline__ double weight_of_any(float x, float top, double c) {
    return finite(top) ? weight(x, top, c) : top == INFINITY && x == INFINITY && c > 0 ? 1.0 : 0.0;
}

// A row of logits, or part of one: the reference and the sum of the weights.
struct Norm {
    float top;
    double sum;
    __device__ __forceinline__ void add(float top2, double sum2, double c) {
        if (!(sum2 > 0)) return;
        if (top2 > top) sum *= weight_of_any(top, top2, c), top = top2;
        sum += top2 == top ? sum2 : sum2 * weight_of_any(top2, top, c);
    }
};
// The lanes' norms as one.
__device__ __forceinline__ Norm joined(Norm n, int lane, double c) {
    const float top = max_lanes(n.sum > 0 ? n.top : -INFINITY, lane);
    return Norm{top, sum_lanes(n.sum > 0 ? (n.top == top ? n.sum : n.sum * weight_of_any(n.top, top, c)) : 0.0, lane)};
}
// A lane's sum of the weights of a range, relative to top, which the wave's lanes share: the one given, or where that is
// -infinity or does not do, one of the range's own.
template <int BF16>
__device__ __forceinline__ double sum_range(const Range<BF16>& x, int lane, double c, float& top) {
    double w[16];
    if (top == -INFINITY) top = max_lanes(x.get(0), lane);
    if (finite(top)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = weight(x.get(e), top, c);
        const double v = sum16(w);
        if (!__any(!(v < 1e290))) return v;  // (longer sums stay in range, too)
    }
    // infinite entries, nothing but -infinity and NaN, or far more than the reference
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, x.get(e));
    top = max_lanes(m, lane);
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = weight_of_any(x.get(e), top, c);
    return sum16(w);
}

// The same with exponentials in 32 bits, off by 2e-5 at most (three roundings of an exponent of at most 100): enough for a
// decision about one child, which has one border, not one per entry, unless it is close to that.  256 chains of 5 over 131072
// bf16 logits 177 us, with all norms in 64 bits 225.  An x - top that overflows is an exponent of -340 or less, but where c is under
// 1e-36: there in 64 bits.
template <int BF16>
__device__ __forceinline__ double sum_range_fast(const Range<BF16>& x, int lane, double c, float& top) {
    if (top == -INFINITY) top = max_lanes(x.get(0), lane);
    if (finite(top) && c >= 1e-36) {
        float w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = __builtin_amdgcn_exp2f((x.get(e) - top) * (float)c);
        const float v = sum16(w);
        if (!__any(!(v < 1e30f))) return (double)v;
    }
    return sum_range(x, lane, c, top);
}

// ---- every row's norm, by parts ----

__device__ __forceinline__ double inverse_temperature(const VerifyArgs& a, int b, bool logits) {
    const float scale = logits && a.scale ? a.scale[b] : 1.f;
    return scale > 0.f ? (double)scale * 1.4426950408889634074 : (double)NAN;
}
// (an inverse temperature near the end of fp32 is as good as an infinite one)
__device__ __forceinline__ bool is_greedy(const VerifyArgs& a, double c) { return !a.uniform || c > 6e36f * 1.4426950408889634074; }

template <int BF16>
__device__ __forceinline__ void largest_of(const Range<BF16>& x, int first, int lane, float& top, int& where) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (x.get(e) > top) top = x.get(e), where = first + entry<BF16, false>(lane, e);
}
template <int BF16>
__device__ __forceinline__ float entry_of(const char* row, int i) {
    return BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(row)[i]) : reinterpret_cast<const float*>(row)[i];
}

// The workspace: each row's ranges' norms and its parts' (target rows, then draft rows), each sequence's sums and
// where its walk came to.
struct Stop {
    int node, count, flags, path[KVARN_MAX_DRAFTS];  // flags: 1 rest, 2 done
    uint64_t children, gone;
    double taken, left, ratio;
    Norm np, nq;
};
struct Layout {
    int64_t rows;
    int ranges, parts;  // of a row
    __host__ __device__ int64_t part_at(int64_t row) const { return rows * ranges + row * parts; }
    __host__ __device__ int64_t norms() const { return rows * (ranges + parts); }
};
constexpr int kRowsWaves = 4, kStep = 4;  // of k_rows: ranges per wave, which its loads bring together
__host__ __device__ inline Layout layout(int batch, int n_draft, int vocab) {
    Layout l;
    l.rows = 2 * (int64_t)batch * n_draft;
    l.ranges = (vocab + kRange - 1) / kRange;
    l.parts = (l.ranges + kStep * kRowsWaves - 1) / (kStep * kRowsWaves);
    return l;
}

// A workgroup per part of a row (grid: parts, rows of one kind, kinds); ranges r, r + 4, ... of the part to wave r.
// All of a row's sums are relative to one reference, taken from its first entries, wherever that does.
// What is written of a range or a part: its norm, or (greedy) its largest entry and the index of that in the place of
// the sum.  Bound by the vector units where norms are formed, some 22 instructions per entry: 1152 rows of 128000 bf16 entries
// 120 us, vector units busy for 77 %, 2.5 TB/s; 72 rows 12 us.  Largest entries are bound by HBM (5.8 TB/s).
template <int BF16>
__global__ __launch_bounds__(64 * kRowsWaves) void k_rows(VerifyArgs a) {
    __shared__ Norm of_wave[kRowsWaves];
    constexpr int es = BF16 ? 2 : 4;
    constexpr uint32_t none = kNone<BF16, 1>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = a.n_draft;
    const Layout l = layout(a.batch, t, a.vocab);
    const int part = blockIdx.x % l.parts, at = blockIdx.x / l.parts, b = at / t, node = at - b * t;
    const bool of_draft = blockIdx.y;
    const int live = a.n_live ? min(max(a.n_live[b], 0), t) : t;
    if (node >= live) return;
    if (of_draft) {  // only where there are children
        const bool child = lane > node && lane < live && (a.parent ? a.parent[(int64_t)b * t + lane] == node : lane == node + 1);
        if (!__any(child)) return;
    }
    const char* row = of_draft ? static_cast<const char*>(a.draft) + at * a.draft_stride * es : static_cast<const char*>(a.target) + at * a.target_stride * es;
    const int r0 = part * kStep * kRowsWaves + wave, whole = a.vocab / kRange;
    Range<BF16> x[kStep];
    if (r0 + (kStep - 1) * kRowsWaves < whole) {
#pragma unroll
        for (int i = 0; i < kStep; ++i) x[i].template load<false>(row, r0 + i * kRowsWaves, lane);
    } else {
#pragma unroll
        for (int i = 0; i < kStep; ++i) x[i].template load_part<false>(row, r0 + i * kRowsWaves, a.vocab, lane, none);
    }
    const float sample = entry_of<BF16>(row, min(lane, a.vocab - 1));
    const double c = inverse_temperature(a, b, a.form == KVARN_LOGITS);
    const bool greedy = is_greedy(a, c);
    const int64_t row_at = (of_draft ? l.rows / 2 : 0) + at;
    Norm* norms = static_cast<Norm*>(a.ws);
    Norm mine{-INFINITY, 0};
    if (greedy) {
        float top = -INFINITY;
        int where = 0x7FFFFFFF;
#pragma unroll
        for (int i = 0; i < kStep; ++i)
            largest_of(x[i], (r0 + i * kRowsWaves) * kRange, lane, top, where);
        const float high = max_lanes(top, lane);
        mine = Norm{high, (double)min_lanes(top == high ? where : 0x7FFFFFFF, lane)};  // (in every lane)
    } else {
        const float first = max_lanes(sample, lane);
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
            const int r = r0 + i * kRowsWaves;
            if (r >= l.ranges) break;
            float ref = first;
            const double v = running(sum_range(x[i], lane, c, ref));
            if (lane == 63) norms[row_at * l.ranges + r] = Norm{ref, v}, mine.add(ref, v, c);
        }
    }
    if (lane == 63) of_wave[wave] = mine;
    __syncthreads();
    if (wave != 0) return;
    if (greedy) {
        mine = of_wave[lane % kRowsWaves];
        const float high = max_lanes(mine.top, lane);
        mine = Norm{high, (double)min_lanes(mine.top == high ? (int)mine.sum : 0x7FFFFFFF, lane)};
    } else {
        mine = joined(lane < kRowsWaves ? of_wave[lane] : Norm{-INFINITY, 0}, lane, c);
    }
    if (lane == 0) norms[l.part_at(row_at) + part] = mine;
}

// ---- the walk ----

template <int WAVES>
struct Lds {
    double part[kMaxRanges];  // each range's sum of weights
    float refs[kMaxRanges];   // logits, where these are relative to a reference for each range: that
    Norm norm[2][WAVES];      // the waves' parts of a row's norm
    float top[WAVES];         // (greedy) of its largest entry
    int at[WAVES];
};

// One sequence's walk, the same in every lane and wave of a workgroup.  STORED: k_rows has formed the rows' norms.
template <int BF16, int LOGITS, int STORED, int WAVES>
struct Walk {
    static constexpr int es = BF16 ? 2 : 4;
    static constexpr uint32_t none = kNone<BF16, LOGITS>;
    const VerifyArgs& a;
    Lds<WAVES>& lds;
    const int b, lane, wave, t, vocab, ranges;
    const int64_t at;
    int live, token, parent;
    double c, u;
    bool able, greedy, drawn;
    float in_p = 0, in_q = 0;
    // STORED: the norms of node `lane`'s rows, or (greedy) its largest entry's index
    Norm node_p{0, 1}, node_q{0, 1};
    int best = -1;
    // the node, its rows, the children that are still to be considered, and what those refused have left
    int node = 0, count, next = -1, path;
    const char *row, *q_row;
    Norm np, nq;
    double pc, qc, taken, left, ratio;
    uint64_t children, gone;
    bool rough;  // np and nq in 32 bits

    __device__ __forceinline__ Walk(const VerifyArgs& args, Lds<WAVES>& l, int seq)
        : a(args), lds(l), b(seq), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), t(args.n_draft),
          vocab(args.vocab), ranges((args.vocab + kRange - 1) / kRange), at((int64_t)seq * args.n_draft) {
        live = a.n_live ? min(max(a.n_live[b], 0), t) : t;
        c = inverse_temperature(a, b, LOGITS);
        greedy = is_greedy(a, c);
        drawn = a.draft != nullptr;
        u = greedy || lane >= t ? 0.0 : (double)a.uniform[at + lane];
        count = live > 0 ? 1 : 0;
        path = lane < count ? 0 : -1;
    }
    // The drafts, lane i holding draft i.
    __device__ __forceinline__ void read_drafts() {
        const bool here = lane > 0 && lane < live;
        parent = !here ? -1 : a.parent ? a.parent[at + lane] : lane - 1;
        token = here ? a.tokens[at + lane] : -1;
        able = here && parent >= 0 && parent < lane && token >= 0 && token < vocab;
        // its token's entries in its parent's rows
        if (able && !greedy) {
            in_p = entry_of<BF16>(target_row(parent), token);
            if (drawn) in_q = entry_of<BF16>(draft_row(parent), token);
        }
        if constexpr (STORED) {
            if (lane < live) {
                const Layout l = layout(a.batch, t, vocab);
                const Norm* p = static_cast<const Norm*>(a.ws) + l.part_at(at + lane);
                if (greedy) {
                    float top = -INFINITY;
                    for (int i = 0; i < l.parts; ++i)
                        if (p[i].top > top) top = p[i].top, best = (int)p[i].sum;
                } else {
                    node_p = sum_parts(p, l.parts);
                }
            }
            uint64_t with = 0;  // nodes with children
            for (uint64_t m = __ballot(able); m; m &= m - 1) with |= 1ull << __builtin_amdgcn_readlane(parent, __builtin_ctzll(m));
            if (drawn && !greedy && (with >> lane & 1)) {
                const Layout l = layout(a.batch, t, vocab);
                node_q = sum_parts(static_cast<const Norm*>(a.ws) + l.part_at((int64_t)a.batch * t + at + lane), l.parts);
            }
            // each child's probabilities
            const int up = max(parent, 0);
            pc = prob(in_p, Norm{__shfl(node_p.top, up), __shfl(node_p.sum, up)});
            qc = drawn ? prob(in_q, Norm{__shfl(node_q.top, up), __shfl(node_q.sum, up)}) : 0;
        }
    }
    // A row's norm from those of its parts, by one lane.
    __device__ __forceinline__ Norm sum_parts(const Norm* p, int parts) const {
        Norm n{-INFINITY, 0};
        for (int i = 0; i < parts; i += 4) {  // (four loads at a time)
            Norm x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = p[min(i + k, parts - 1)];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < parts) n.add(x[k].top, x[k].sum, c);
        }
        return n;
    }
    __device__ __forceinline__ const char* target_row(int i) const { return static_cast<const char*>(a.target) + (at + i) * a.target_stride * es; }
    __device__ __forceinline__ const char* draft_row(int i) const { return static_cast<const char*>(a.draft) + (at + i) * a.draft_stride * es; }
    __device__ __forceinline__ double prob(float x, const Norm& n) const {  // an entry's probability in 64 bits
        if constexpr (!LOGITS) return x == x ? (double)x : 0.0;
        return n.sum > 0 ? weight_of_any(x, n.top, c) / n.sum : 0.0;
    }
    // f(r, p's range, q's range) for r = first, first + step, ...  One group's loads are in flight while another is worked on:
    // with 32-bit exponentials throughout, 256 chains of 5 over 131072 bf16 logits 106 us in place of 113 by groups of twice the
    // size one after the other.  (No branch round the loads: behind one the compiler would wait for all of them.)
    template <bool TWO, class F>
    __device__ __forceinline__ void each_range(int first, int step, uint32_t nothing, F f) const {
        constexpr int G = BF16 ? 2 : 1;
        const int whole = vocab / kRange;
        Range<BF16> p0[G], q0[TWO ? G : 1], p1[G], q1[TWO ? G : 1];
        auto load = [&](Range<BF16>(&p)[G], Range<BF16>(&q)[TWO ? G : 1], int r) {  // (behind the end, the last once more)
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const int k = min(r + i * step, whole - 1);
                p[i].template load<false>(row, k, lane);
                if constexpr (TWO) q[i].template load<false>(q_row, k, lane);
            }
        };
        auto use = [&](const Range<BF16>(&p)[G], const Range<BF16>(&q)[TWO ? G : 1], int r) {
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (r + i * step < whole) f(r + i * step, p[i], q[TWO ? i : 0]);
        };
        if (first < whole) load(p0, q0, first);
        for (int r = first; r < whole; r += 2 * G * step) {
            load(p1, q1, r + G * step);
            use(p0, q0, r);
            load(p0, q0, r + 2 * G * step);
            use(p1, q1, r + G * step);
        }
        if (whole < ranges && whole >= first && (whole - first) % step == 0) {
            Range<BF16> p, q;
            p.template load_part<false>(row, whole, vocab, lane, nothing);
            if constexpr (TWO) q.template load_part<false>(q_row, whole, vocab, lane, nothing);
            f(whole, p, q);
        }
    }
    // Norms of one row or of two, read by the whole workgroup.  KEEP: one row, with each range's sum and reference in LDS.
    // FAST: in 32 bits.
    template <bool KEEP, bool TWO, bool FAST>
    __device__ __forceinline__ void read_norms() {
        Norm x{-INFINITY, 0}, y = x;
        float tp = -INFINITY, tq = -INFINITY;
        __syncthreads();
        // a range into a lane's share, in the reference of the ranges before it
        auto add = [&](Norm& n, float& top, const Range<BF16>& z, int r) {
            double v = FAST ? sum_range_fast(z, lane, c, top) : sum_range(z, lane, c, top);
            if constexpr (KEEP) {
                v = running(v);
                if (lane == 63) lds.part[r] = v, lds.refs[r] = top, n.add(top, v, c);
            } else {
                if (n.top == top) n.sum += v;
                else n.add(top, v, c);
            }
        };
        each_range<TWO>(wave, WAVES, kNone<BF16, 1>, [&](int r, const Range<BF16>& p, const Range<BF16>& q) {
            add(x, tp, p, r);
            if constexpr (TWO) add(y, tq, q, r);
        });
        x = joined(x, lane, c);
        if constexpr (TWO) y = joined(y, lane, c);
        if (lane == 0) lds.norm[0][wave] = x, lds.norm[1][wave] = y;
        __syncthreads();
        np = joined(lane < WAVES ? lds.norm[0][lane] : Norm{-INFINITY, 0}, lane, c);
        if constexpr (TWO) nq = joined(lane < WAVES ? lds.norm[1][lane] : Norm{-INFINITY, 0}, lane, c);
    }

    // The first of the largest entries of the node's row; -1 where there is nothing but NaN and -infinity.
    __device__ __forceinline__ int largest() {
        float top = -INFINITY;
        int where = 0x7FFFFFFF;
        if constexpr (STORED) return __builtin_amdgcn_readlane(best, node);
        each_range<false>(wave, WAVES, kNone<BF16, 1>,
                          [&](int r, const Range<BF16>& x, const Range<BF16>&) { largest_of(x, r * kRange, lane, top, where); });
        const float high = max_lanes(top, lane);
        where = min_lanes(top == high ? where : 0x7FFFFFFF, lane);
        __syncthreads();
        if (lane == 0) lds.top[wave] = high, lds.at[wave] = where;
        __syncthreads();
        top = lds.top[lane % WAVES];
        where = min_lanes(top == max_lanes(top, lane) ? lds.at[lane % WAVES] : 0x7FFFFFFF, lane);
        return where == 0x7FFFFFFF ? -1 : where;
    }

    // To node i: its rows, children and norms.
    bool summed;  // lds.part holds the sums of p's ranges
    __device__ __forceinline__ void enter(int i) {
        node = i;
        row = target_row(i);
        q_row = drawn ? draft_row(i) : nullptr;
        children = __ballot(able && parent == i);
        gone = 0;
        taken = 0;
        left = 1;
        summed = rough = false;
        if (greedy) return;
        np = nq = Norm{0, 1};
        ratio = 0;
        if constexpr (LOGITS) {
            const bool two = drawn && children;
            if constexpr (STORED) {
                np = Norm{__shfl(node_p.top, i), of_lane(node_p.sum, i)};
                if (two) nq = Norm{__shfl(node_q.top, i), of_lane(node_q.sum, i)};
                return;
            }
            rough = children;
            if (two) {
                read_norms<false, true, true>();
            } else if (children) {
                read_norms<false, false, true>();
            } else {
                read_norms<true, false, false>();
                __syncthreads();
                for (int r = threadIdx.x; r < ranges; r += 64 * WAVES) if (lds.refs[r] != np.top) lds.part[r] *= weight_of_any(lds.refs[r], np.top, c);
                __syncthreads();
                summed = true;
            }
        }
        pc = prob(in_p, np);  // (the children's lanes)
        qc = drawn ? prob(in_q, nq) : 0;
    }
    // For one that goes on from where k_rest stopped.
    __device__ __forceinline__ void resume(const Stop& s) {
        node = s.node;
        count = s.count;
        path = s.path[lane];
        rest = s.flags & 1;
        done = s.flags & 2;
        children = s.children;
        gone = s.gone;
        taken = s.taken;
        left = s.left;
        ratio = s.ratio;
        np = s.np;
        nq = s.nq;
        summed = rough = false;
        row = target_row(node);
        q_row = drawn ? draft_row(node) : nullptr;
    }
    __device__ __forceinline__ void note(Stop& s) const {
        s.path[lane] = path;
        if (lane) return;
        s.node = node;
        s.count = count;
        s.flags = (rest ? 1 : 0) | (done ? 2 : 0);
        s.children = children;
        s.gone = gone;
        s.taken = taken;
        s.left = left;
        s.ratio = ratio;
        s.np = np;
        s.nq = nq;
    }

    // On to the next place where ranges have to be summed (true: of what the refused children leave of p, `rest`, or
    // else of p), or to the end.
    bool rest, done;
    __device__ __forceinline__ void advance() {
        while (children) {
            const int i = __builtin_ctzll(children);
            children &= children - 1;
            if (!drawn && (gone & __ballot(token == __builtin_amdgcn_readlane(token, i)))) continue;
            const double ui = of_lane(u, i);
            double pi = of_lane(pc, i), qi = of_lane(qc, i);
            bool hit = drawn ? ui * left * qi < pi - taken * qi : ui * left < pi;
            if constexpr (LOGITS && !STORED) {
                // Norms in 64 bits, from here on, for a decision close to its border, and for what a refused child leaves.
                // (Of candidates, left is off by 2e-5 as a whole.)
                const double border = drawn ? ui * left * qi + taken * qi : ui * left;
                if (rough && ((drawn && !hit) || fabs(pi - border) <= 1e-4 * __builtin_fmax(pi, drawn ? border : ui))) {
                    rough = false;
                    if (drawn) read_norms<false, true, false>();
                    else read_norms<false, false, false>();
                    pc = prob(in_p, np);
                    qc = drawn ? prob(in_q, nq) : 0;
                    left = 1;
                    for (uint64_t g = gone; g; g &= g - 1) left -= of_lane(pc, __builtin_ctzll(g));
                    pi = of_lane(pc, i), qi = of_lane(qc, i);
                    hit = drawn ? ui * qi < pi : ui * left < pi;  // (taken is 0: it grows by refused children)
                }
            }
            if (drawn) {
                if (!hit) {
                    taken += left;
                    // p - taken q, in units of p's sum
                    ratio = LOGITS ? (nq.sum > 0 ? taken * np.sum / nq.sum : 0) : taken;
                    rest = true;
                    return;
                }
            } else {
                if (!hit) {
                    gone |= 1ull << i;
                    left -= pi;
                }
            }
            if (hit) {
                if (lane == count) path = i;
                ++count;
                enter(i);
            }
        }
        done = true;
        rest = drawn ? taken > 0 && left > 0 : gone != 0;
    }

    // The weights of 16 entries, in the row's order if CONSECUTIVE; for logits relative to the row's reference.
    template <bool CONSECUTIVE, bool TWO>
    __device__ __forceinline__ void weights(const Range<BF16>& x, const Range<BF16>& y, int r, double (&w)[16]) const {
        if constexpr (!LOGITS) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                w[e] = (double)above_0(x.get(e));
                if constexpr (TWO) w[e] = __builtin_fmax(fma(-ratio, (double)above_0(y.get(e)), w[e]), 0.0);
            }
        } else if (finite(np.top) && (!TWO || finite(nq.top))) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                w[e] = weight(x.get(e), np.top, c);
                if constexpr (TWO) w[e] = __builtin_fmax(fma(-ratio, weight(y.get(e), nq.top, c), w[e]), 0.0);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                w[e] = weight_of_any(x.get(e), np.top, c);
                if constexpr (TWO) w[e] = __builtin_fmax(fma(-ratio, weight_of_any(y.get(e), nq.top, c), w[e]), 0.0);
            }
        }
        for (uint64_t g = TWO ? 0 : gone; g; g &= g - 1) {
            const int i = __builtin_amdgcn_readlane(token, __builtin_ctzll(g)) - r * kRange;
            if (i < 0 || i >= kRange) continue;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (entry<BF16, CONSECUTIVE>(lane, e) == i) w[e] = 0;
        }
    }
    // The sums of ranges first, first + step, ..., given to `put` in one lane.
    template <bool TWO, class F>
    __device__ __forceinline__ void sum_two(int first, int step, F put) const {
        each_range<TWO>(first, step, none, [&](int r, const Range<BF16>& x, const Range<BF16>& y) {
            double w[16];
            weights<false, TWO>(x, y, r, w);
            const double v = running(sum16(w));
            if (lane == 63) put(r, v);
        });
    }
    template <class F>
    __device__ __forceinline__ void sum_ranges(int first, int step, F put) const {
        if (rest && drawn) sum_two<true>(first, step, put);
        else sum_two<false>(first, step, put);
    }
    // All of them into lds.part.
    __device__ __forceinline__ void pass() {
        __syncthreads();
        sum_ranges(wave, WAVES, [&](int r, double v) { lds.part[r] = v; });
        __syncthreads();
    }
    __device__ __forceinline__ double whole() const {
        double sum = 0;
        for (int r = lane; r < ranges; r += 64) sum += lds.part[r];
        return sum_lanes(sum, lane);
    }

    // The first entry whose running sum of weights exceeds u times the whole.
    __device__ __forceinline__ int draw() const {
        const double mark = of_lane(u, 0) * whole();
        const int per = (ranges + 63) / 64, r0 = lane * per, r1 = min(r0 + per, ranges);
        double mine = 0;
        for (int i = r0; i < r1; ++i) mine += lds.part[i];
        double before = running(mine) - mine, r_before = 0;
        int r = -1, last = -1;  // the range that holds it, and the last range with weight
        for (int i = r0; i < r1; ++i) {
            const double v = lds.part[i];
            if (!(v > 0)) continue;
            last = i;
            if (r < 0 && before + v > mark) r = i, r_before = before;
            before += v;
        }
        const uint64_t found = __ballot(r >= 0), some = __ballot(last >= 0);
        if (!some) return -1;
        if (found) {
            const int l = __builtin_ctzll(found);
            r = __builtin_amdgcn_readlane(r, l);
            r_before = of_lane(r_before, l);
        } else {  // by rounding
            r = __builtin_amdgcn_readlane(last, 63 - __builtin_clzll(some));
            r_before = -INFINITY;
        }
        Range<BF16> x, y;
        double w[16];
        x.template load_part<true>(row, r, vocab, lane, none);
        if (rest && drawn) {
            y.template load_part<true>(q_row, r, vocab, lane, none);
            weights<true, true>(x, y, r, w);
        } else {
            weights<true, false>(x, y, r, w);
        }
        double v = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) v += w[e];
        double run = r_before + (running(v) - v);
        int hit = -1, end = -1;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            run += w[e];
            if (w[e] > 0) end = 16 * lane + e;
            if (w[e] > 0 && hit < 0 && run > mark) hit = 16 * lane + e;
        }
        const uint64_t hits = __ballot(hit >= 0), ends = __ballot(end >= 0);
        if (hits) return r * kRange + __builtin_amdgcn_readlane(hit, __builtin_ctzll(hits));
        return ends ? r * kRange + __builtin_amdgcn_readlane(end, 63 - __builtin_clzll(ends)) : -1;
    }
};

// The sums of a sequence's ranges at the first place that needs them, by gridDim.x workgroups.  Bound by HBM: two rows of
// 128000 fp32 entries for each of 64 sequences 12.3 us, 5.3 TB/s.
constexpr int kRestWaves = 4;
template <int BF16, int LOGITS>
__global__ __launch_bounds__(64 * kRestWaves) void k_rest(VerifyArgs a) {
    __shared__ Lds<kRestWaves> lds;
    Walk<BF16, LOGITS, LOGITS, kRestWaves> w(a, lds, blockIdx.y);
    if (w.live == 0 || w.greedy) return;
    w.read_drafts();
    w.done = false;
    w.enter(0);
    w.advance();
    if (blockIdx.x == 0 && w.wave == 0) w.note(static_cast<Stop*>(a.stops)[w.b]);
    if (LOGITS && !w.rest) return;  // the rows' norms tell them
    double* part = a.sums + (int64_t)w.b * w.ranges;
    w.sum_ranges(blockIdx.x * kRestWaves + w.wave, gridDim.x * kRestWaves, [&](int r, double v) { part[r] = v; });
}

// A workgroup per sequence: the walk, and the next token.  SPREAD: from where k_rest stopped.  Where it walks alone, 256
// chains of 5 drafts over 131072 bf16 logits take 177 us: vector units busy for 54 % of it, and for three quarters of the
// 71 % in which all workgroups run; the rest belongs to the longest paths.  570 MB are read, 3.3 TB/s.  Eight waves: with 16, which
// leave 128 registers each, the next token of 256 sequences from 128000 fp32 probabilities 26.0 us in place of 24.3.
// After k_rest it is bound by latency (its stop and sums, the one range, running sums: 6 us), and on
// trees whose siblings are refused by passes of 7 us each, of two rows of 100003 fp32 entries by one workgroup.
constexpr int kWaves = 8;
template <int BF16, int LOGITS, int STORED, int SPREAD>
__global__ __launch_bounds__(64 * kWaves) void k_verify(VerifyArgs a) {
    __shared__ Lds<kWaves> lds;
    Walk<BF16, LOGITS, STORED, kWaves> w(a, lds, blockIdx.x);
    if (w.live > 0 && w.greedy) {
        w.read_drafts();
        w.enter(0);
        for (;;) {
            w.next = w.largest();
            const uint64_t hit = w.children & __ballot(w.token == w.next);
            if (!hit) break;
            if (w.lane == w.count) w.path = __builtin_ctzll(hit);
            ++w.count;
            w.enter(__builtin_ctzll(hit));
        }
    } else if (w.live > 0) {
        w.done = false;
        auto from_rest = [&] {  // the sums that k_rest has formed
            for (int r = threadIdx.x; r < w.ranges; r += 64 * kWaves) lds.part[r] = a.sums[(int64_t)w.b * w.ranges + r];
            __syncthreads();
        };
        if constexpr (SPREAD) {
            w.resume(static_cast<const Stop*>(a.stops)[w.b]);
            if (!LOGITS || w.rest) from_rest();
            w.summed = w.done && !LOGITS;
            if (w.children || w.gone) {  // otherwise the drafts are not needed any more
                w.read_drafts();
                if constexpr (!STORED) w.pc = w.prob(w.in_p, w.np), w.qc = w.drawn ? w.prob(w.in_q, w.nq) : 0;
            }
            if (!w.done) w.left = LOGITS ? w.whole() / w.np.sum : w.whole();
        } else {
            w.read_drafts();
            w.enter(0);
        }
        while (!w.done) {
            w.advance();
            if (w.done) break;
            w.pass();
            w.left = LOGITS ? w.whole() / w.np.sum : w.whole();
        }
        if (w.drawn && w.taken > 0 && w.left > 0) {
            // (the sums are those of the last refused child)
        } else if constexpr (LOGITS && STORED) {
            __syncthreads();
            const Norm* from = static_cast<const Norm*>(a.ws) + (w.at + w.node) * w.ranges;
            for (int r = threadIdx.x; r < w.ranges; r += 64 * kWaves) lds.part[r] = from[r].top == w.np.top ? from[r].sum : from[r].sum > 0 ? from[r].sum * weight_of_any(from[r].top, w.np.top, w.c) : 0;
            __syncthreads();
            if (w.rest) {  // ranges that candidates have left
                uint64_t todo = w.gone;
                for (int n = 0; todo; todo &= todo - 1, ++n)
                    if (n % kWaves == w.wave) {
                        const int r = __builtin_amdgcn_readlane(w.token, __builtin_ctzll(todo)) / kRange;
                        w.template sum_two<false>(r, 1 << 20, [&](int i, double v) { lds.part[i] = v; });
                    }
                __syncthreads();
            }
        } else if (!w.summed) {
            w.pass();
        }
        w.next = w.draw();
    }
    if (w.wave == 0) {
        if (w.lane < w.t) a.path[w.at + w.lane] = w.path;
        if (w.lane == 0) a.n_path[w.b] = w.count, a.next[w.b] = w.next;
    }
}

// Whether every row's norm is formed before the walk (rows), and by how many workgroups per sequence its first sums are
// (rest).  A workgroup alone takes 0.16 us per range for what a next token needs of a row of bf16 logits, with 4 to 6 us of
// latency at every node; k_rows takes 0.8 ns per range of all rows, needed or not, and its launch.  Measured, the walk alone
// against the launches before it (us, bf16; sequences x drafts, entries):
//   next token    64 x 1, 128000: 29.8 and 19.0;  128 x 1: 29.4, 25.0;  192 x 1: 29.4, 30.1;  64 x 1, 32000: 13.1, 13.2
//   drawn chains  16 x 5, 128000: 156, 38;  64 x 5: 160, 92;  128 x 5: 163, 160;  64 x 5, 32000: 67, 38
//   drawn trees   8 x 24, 128000: 214, 136;  16 x 24: 263, 218;  32 x 24: 362, 369
//   candidates    64 x 8, 128000: 65, 64 to 70;  128 x 8: 68, 116
//   greedy        64 x 1, 128000: 9.2, 8.8;  128 x 1: 9.5, 10.9;  32 x 8: 51, 17;  128 x 8: 65, 49;  48 x 64, 65537: 27, 62
//   probabilities (fp32) 1 x 1, 128000: 10.2, 8.4;  32 x 1: 11.0, 9.5;  64 x 1: 11.1, 12.1;  16 x 1, 64000: 7.9, 8.5;
//                 1 x 8, 128000: 16.8, 9.5;  64 x 8: 24, 19;  128 x 8: 33, 33;  64 x 8, 32000: 12.7, 12.5
struct Plan {
    bool rows;
    int rest;
};
constexpr int kGreedyRows = 1024, kLogitRows = 640, kNextRows = 192;  // at most, for k_rows
constexpr int kRestChains = 96, kRestNext = 48;                       // sequences, for k_rest on probabilities
Plan plan_verify(int batch, int n_draft, int vocab, bool logits, bool draft, bool greedy) {
    const int ranges = (vocab + kRange - 1) / kRange;
    const int64_t rows = (int64_t)batch * n_draft;
    Plan p{false, 0};
    if (n_draft > 1) p.rows = (logits || greedy) && ranges >= 16 && rows <= (greedy ? kGreedyRows : kLogitRows);
    else p.rows = logits && !greedy && ranges >= 64 && rows <= kNextRows;
    const bool rest = logits ? p.rows && draft && n_draft > 1 : n_draft > 1 ? batch <= kRestChains && ranges >= 64 : batch <= kRestNext && ranges >= 96;
    if (rest && !greedy) p.rest = std::min((ranges + 2 * kRestWaves - 1) / (2 * kRestWaves), std::max(1, 2048 / batch));
    return p;
}

template <int BF16, int LOGITS>
void launch_walk(const VerifyArgs& a, const Plan& plan, hipStream_t stream) {
    const dim3 grid(a.batch), block(64 * kWaves);
    if (plan.rest) {
        hipLaunchKernelGGL((k_rest<BF16, LOGITS>), dim3(plan.rest, a.batch), dim3(64 * kRestWaves), 0, stream, a);
        hipLaunchKernelGGL((k_verify<BF16, LOGITS, LOGITS, 1>), grid, block, 0, stream, a);
    } else if (plan.rows) {
        hipLaunchKernelGGL((k_verify<BF16, LOGITS, 1, 0>), grid, block, 0, stream, a);
    } else {
        hipLaunchKernelGGL((k_verify<BF16, LOGITS, 0, 0>), grid, block, 0, stream, a);
    }
}
template <int BF16>
void launch_all(const VerifyArgs& a, const Plan& plan, hipStream_t stream) {
    if (plan.rows) {
        const Layout l = layout(a.batch, a.n_draft, a.vocab);
        const dim3 grid((unsigned)(l.rows / 2 * l.parts), a.draft ? 2 : 1), block(64 * kRowsWaves);
        hipLaunchKernelGGL(k_rows<BF16>, grid, block, 0, stream, a);
    }
    if (a.form == KVARN_LOGITS && a.uniform) launch_walk<BF16, 1>(a, plan, stream);
    else launch_walk<BF16, 0>(a, plan, stream);
}

}  // namespace

size_t verify_workspace_need(int batch, int n_draft, int vocab) {
    const Layout l = layout(batch, n_draft, vocab);
    const Plan logits = plan_verify(batch, n_draft, vocab, true, true, false);
    const bool rows = logits.rows || plan_verify(batch, n_draft, vocab, false, false, true).rows;
    const bool rest = logits.rest > 0 || plan_verify(batch, n_draft, vocab, false, true, false).rest > 0;
    return (rows ? l.norms() * sizeof(Norm) : 0) + (rest ? batch * (sizeof(Stop) + l.ranges * sizeof(double)) : 0);
}

// For a number of drafts the need grows with the batch up to where a launch before the walk is left out; with the entries it always
// grows.
size_t verify_workspace_bytes(int batch, int n_draft, int vocab) {
    size_t most = 0;
    for (int n = 1; n <= n_draft; ++n)
        for (int last : {batch, kGreedyRows / n, kLogitRows / n, kNextRows, kRestChains, kRestNext})
            most = std::max(most, verify_workspace_need(std::min(batch, last), n, vocab));
    return most;
}

hipError_t launch_verify(const VerifyArgs& a0, hipStream_t stream) {
    VerifyArgs a = a0;
    const Plan plan = plan_verify(a.batch, a.n_draft, a.vocab, a.form == KVARN_LOGITS, a.draft, !a.uniform);
    const Layout l = layout(a.batch, a.n_draft, a.vocab);
    if (plan.rest) {
        a.stops = static_cast<Norm*>(a.ws) + (plan.rows ? l.norms() : 0);
        a.sums = reinterpret_cast<double*>(static_cast<Stop*>(a.stops) + a.batch);
    }
    if (a.bf16) launch_all<1>(a, plan, stream);
    else launch_all<0>(a, plan, stream);
    return hipGetLastError();
}

}  // namespace kvarn
