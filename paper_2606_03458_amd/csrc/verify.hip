// Verification of drafted tokens (include/kvarn.h, kvarn_verify_drafts).
//
// The rule with draft rows is that of k rounds of rejection, each round drawing one child from q against what the
// rounds before have left of p: w_0 = p, w_{k+1} = max(w_k / sum w_k - q, 0).  All of these are max(p - a q, 0) up to
// a factor, with a_{k+1} = a_k + S_k, S_k = sum max(p - a_k q, 0) and S_0 = 1 (divide by the factor: w_k / sum w_k =
// max(p - a_k q, 0) / S_k, and subtracting q moves a by S_k), so a round needs one number and one pass over two rows.
//
// One workgroup per sequence walks its tree.  A row is read in ranges of 1024 entries, one wave per range in turn, and
// each range's sum of weights is kept in LDS: their running sum says in which range the next token lies, and only that
// one is read again.  Sums are formed in 64 bits and always in the same order.
#include <type_traits>

#include "common.hpp"

namespace kvarn {
namespace {

constexpr int kRange = 1024, kMaxRanges = KVARN_MAX_VOCAB / kRange, kWaves = 16;

// 16 entries of a row per lane, as pieces of 16 bytes of the lanes side by side (CONSECUTIVE: a lane's 16 entries one
// after the other), entries at and behind vocab as `none`.  Rows are aligned to an element only.
template <int BF16, bool CONSECUTIVE>
__device__ __forceinline__ int entry(int lane, int e) {
    constexpr int N = BF16 ? 8 : 4;
    return CONSECUTIVE ? 16 * lane + e : e / N * 64 * N + lane * N + e % N;
}
template <int BF16, bool CONSECUTIVE>
__device__ __forceinline__ void load_range(const void* row, int first, int vocab, int lane, float none, float (&x)[16]) {
    typedef uint32_t v4 __attribute__((ext_vector_type(4), aligned(2)));
    constexpr int N = BF16 ? 8 : 4, es = BF16 ? 2 : 4;
    const char* at = static_cast<const char*>(row) + (int64_t)first * es;
    if (first + kRange <= vocab) {
        v4 w[16 / N];
#pragma unroll
        for (int i = 0; i < 16 / N; ++i) w[i] = *reinterpret_cast<const v4*>(at + entry<BF16, CONSECUTIVE>(lane, i * N) * es);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            if constexpr (BF16) x[e] = __uint_as_float(e % 2 ? w[e / 8][e % 8 / 2] & 0xFFFF0000u : w[e / 8][e % 8 / 2] << 16);
            else x[e] = __uint_as_float(w[e / 4][e % 4]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int i = entry<BF16, CONSECUTIVE>(lane, e);
            x[e] = none;
            if (first + i < vocab) {
                if constexpr (BF16) x[e] = bf16_to_f32(reinterpret_cast<const uint16_t*>(at)[i]);
                else x[e] = reinterpret_cast<const float*>(at)[i];
            }
        }
    }
}

__device__ __forceinline__ double sum_lanes(double x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m);
    return x;
}
__device__ __forceinline__ float max_lanes(float x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x = fmaxf(x, __shfl_xor(x, m));
    return x;
}

// scale * log2(e) as two floats.
struct Scale {
    float hi, lo;
    double c;
};
// exp(scale * (x - top)) for x <= top, 0 for NaN; the exponent is carried in two floats, so that far entries keep
// their bits (in one, an entry e^-20 below the top is off by 2e-6).
__device__ __forceinline__ float weight(float x, float top, const Scale& s) {
    const float d = x == top ? 0.f : x - top;
    const float hi = d * s.hi, lo = fmaf(d, s.hi, -hi) + d * s.lo;
    const float e = __builtin_amdgcn_exp2f(hi);
    return fmaxf(fmaf(e, lo * 0.69314718f, e), 0.f);
}
__device__ __forceinline__ double weight64(float x, float top, const Scale& s) {
    const double e = exp2((x == top ? 0.0 : (double)x - (double)top) * s.c);
    return e > 0 ? e : 0;
}

// A row of logits: its largest entry and the sum of its weights.
struct Norm {
    float top;
    double sum;
};

template <int BF16, int LOGITS>
__global__ __launch_bounds__(64 * kWaves) void k_verify(VerifyArgs a) {
    __shared__ double part[kMaxRanges];  // each range's sum of weights
    __shared__ double wave_sum[kWaves];
    __shared__ float wave_top[kWaves];
    __shared__ int wave_at[kWaves];
    constexpr int es = BF16 ? 2 : 4;
    const float none = LOGITS ? -INFINITY : 0.f;
    const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = a.n_draft, vocab = a.vocab;
    const int ranges = (vocab + kRange - 1) / kRange;
    const int64_t at = (int64_t)b * t;
    const int live = a.n_live ? min(max(a.n_live[b], 0), t) : t;
    const int parent = lane == 0 || lane >= live ? -1 : a.parent ? a.parent[at + lane] : lane - 1;
    const int token = lane == 0 || lane >= live ? -1 : a.tokens[at + lane];
    const float scale = LOGITS && a.scale ? a.scale[b] : 1.f;
    // (an inverse temperature whose exponents would leave fp32 is as good as an infinite one)
    const bool greedy = !a.uniform || scale > 1e37f;
    const float u = greedy || lane >= t ? 0.f : a.uniform[at + lane];
    Scale s;
    s.c = (scale > 0.f ? (double)scale : (double)NAN) * 1.4426950408889634074;
    s.hi = (float)s.c;
    s.lo = (float)(s.c - (double)s.hi);
    const bool drawn = a.draft != nullptr;

    auto target_row = [&](int node) { return static_cast<const char*>(a.target) + (at + node) * a.target_stride * es; };
    auto draft_row = [&](int node) { return static_cast<const char*>(a.draft) + (at + node) * a.draft_stride * es; };
    auto one = [&](const char* row, int i) { return BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(row)[i]) : reinterpret_cast<const float*>(row)[i]; };

    // The first of the largest entries; -1 where there is nothing but NaN and -infinity.
    auto largest = [&](const char* row) {
        float top = -INFINITY;
        int where = 0x7FFFFFFF;
        for (int r = wave; r < ranges; r += kWaves) {
            float x[16];
            load_range<BF16, false>(row, r * kRange, vocab, lane, -INFINITY, x);
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (x[e] > top) top = x[e], where = r * kRange + entry<BF16, false>(lane, e);
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const float other = __shfl_xor(top, m);
            const int there = __shfl_xor(where, m);
            if (other > top || (other == top && there < where)) top = other, where = there;
        }
        __syncthreads();
        if (lane == 0) wave_top[wave] = top, wave_at[wave] = where;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w)
            if (wave_top[w] > top || (wave_top[w] == top && wave_at[w] < where)) top = wave_top[w], where = wave_at[w];
        return where == 0x7FFFFFFF ? -1 : where;
    };
    // The whole sum of the ranges' parts, every wave for itself.
    auto whole = [&]() {
        double x = 0;
        for (int r = lane; r < ranges; r += 64) x += part[r];
        return sum_lanes(x);
    };
    // A row of logits in one pass.
    auto norm_of = [&](const char* row) {
        float top = -INFINITY;
        double sum = 0;
        __syncthreads();
        for (int r = wave; r < ranges; r += kWaves) {
            float x[16];
            load_range<BF16, false>(row, r * kRange, vocab, lane, -INFINITY, x);
            float m = x[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) m = fmaxf(m, x[e]);
            m = max_lanes(m);
            if (m > -INFINITY) {
                double v = 0;
#pragma unroll
                for (int e = 0; e < 16; ++e) v += (double)weight(x[e], m, s);
                v = sum_lanes(v);
                if (m > top) sum *= weight64(top, m, s), top = m;
                sum += v * weight64(m, top, s);
            }
        }
        if (lane == 0) wave_top[wave] = top, wave_sum[wave] = sum;
        __syncthreads();
        Norm n{-INFINITY, 0};
        for (int w = 0; w < kWaves; ++w) n.top = fmaxf(n.top, wave_top[w]);
        for (int w = 0; w < kWaves; ++w)
            if (wave_top[w] > -INFINITY) n.sum += wave_sum[w] * weight64(wave_top[w], n.top, s);
        if (n.top == -INFINITY) n.top = NAN;  // nothing has weight
        return n;
    };
    auto prob = [&](float x, const Norm& n) {  // an entry's probability in 64 bits
        if constexpr (!LOGITS) return x == x ? (double)x : 0.0;
        const double w = weight64(x, n.top, s) / n.sum;
        return w == w ? w : 0.0;
    };

    int node = 0, count = live > 0 ? 1 : 0, considered = 0, next = -1;
    int path = lane < count ? 0 : -1;
    while (live > 0) {
        const char *row = target_row(node), *q_row = drawn ? draft_row(node) : nullptr;
        uint64_t children = __ballot(lane > considered && parent == node);
        if (greedy) {
            next = largest(row);
            const uint64_t hit = next < 0 ? 0 : children & __ballot(token == next);
            if (!hit) break;
            node = considered = __builtin_ctzll(hit);
        } else {
            Norm np{0, 1}, nq{0, 1};
            double inv_p = 1, inv_q = 1;
            if constexpr (LOGITS) {
                np = norm_of(row);
                inv_p = 1 / np.sum;
                if (drawn && children) {
                    nq = norm_of(q_row);
                    inv_q = 1 / nq.sum;
                }
            }
            uint64_t gone = 0;  // candidates that have left the row
            double taken = 0, left = 1;
            // The weights of 16 entries in the row's order `CONSECUTIVE`: max(p - taken q, 0), or p.
            auto weights = [&](auto consecutive, int r, bool rest, double (&w)[16]) {
                constexpr bool C = decltype(consecutive)::value;
                float x[16], y[16];
                load_range<BF16, C>(row, r * kRange, vocab, lane, none, x);
                if (rest && drawn) load_range<BF16, C>(q_row, r * kRange, vocab, lane, none, y);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    double p = LOGITS ? (double)weight(x[e], np.top, s) * inv_p : (double)x[e];
                    if (rest && drawn) {
                        const double q = LOGITS ? (double)weight(y[e], nq.top, s) * inv_q : (double)y[e];
                        p = fma(-taken, q, p);
                    }
                    w[e] = p > 0 ? p : 0;
                }
                for (uint64_t g = rest && !drawn ? gone : 0; g; g &= g - 1) {
                    const int i = __shfl(token, __builtin_ctzll(g)) - r * kRange;
                    if (i < 0 || i >= kRange) continue;
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (entry<BF16, C>(lane, e) == i) w[e] = 0;
                }
            };
            auto pass = [&](bool rest) {
                __syncthreads();
                for (int r = wave; r < ranges; r += kWaves) {
                    double w[16], v = 0;
                    weights(std::false_type{}, r, rest, w);
#pragma unroll
                    for (int e = 0; e < 16; ++e) v += w[e];
                    v = sum_lanes(v);
                    if (lane == 0) part[r] = v;
                }
                __syncthreads();
                return whole();
            };

            int child = -1;
            for (uint64_t c = children; c && child < 0; c &= c - 1) {
                const int i = __builtin_ctzll(c), tok = __shfl(token, i);
                if (tok < 0 || tok >= vocab) continue;
                const double pc = prob(one(row, tok), np), uc = (double)__shfl(u, i);
                if (drawn) {
                    const double qc = prob(one(q_row, tok), nq);
                    if (uc * left * qc < pc - taken * qc) {
                        child = i;
                    } else {
                        taken += left;
                        left = pass(true);
                    }
                } else if (!__any((gone >> lane & 1) && token == tok)) {
                    if (uc * left < pc) {
                        child = i;
                    } else {
                        gone |= 1ull << i;
                        left -= pc;
                    }
                }
            }
            if (child < 0) {
                // the next token: the first whose running sum exceeds u times the whole
                bool rest = drawn ? taken > 0 : gone != 0;
                double total;
                if (rest && drawn && left > 0) {
                    total = left;
                } else {
                    if (drawn) rest = false;
                    total = pass(rest);
                }
                const double mark = (double)__shfl(u, 0) * total;
                const int per = (ranges + 63) / 64;
                double mine = 0;
                for (int i = 0; i < per; ++i)
                    if (lane * per + i < ranges) mine += part[lane * per + i];
                double upto = mine;
#pragma unroll
                for (int m = 1; m < 64; m *= 2) {
                    const double x = __shfl_up(upto, m);
                    if (lane >= m) upto += x;
                }
                double before = upto - mine;
                int r = -1, last = -1;  // the range that holds it, and the last range with weight
                double r_before = 0;
                for (int i = 0; i < per; ++i) {
                    const int k = lane * per + i;
                    if (k >= ranges || !(part[k] > 0)) continue;
                    last = k;
                    if (r < 0 && before + part[k] > mark) r = k, r_before = before;
                    before += part[k];
                }
                const uint64_t found = __ballot(r >= 0), some = __ballot(last >= 0);
                if (some) {
                    if (found) {
                        const int l = __builtin_ctzll(found);
                        r = __shfl(r, l);
                        r_before = __shfl(r_before, l);
                    } else {  // by rounding
                        r = __shfl(last, 63 - __builtin_clzll(some));
                        r_before = INFINITY;
                    }
                    double w[16];
                    weights(std::true_type{}, r, rest, w);
                    double v = 0;
#pragma unroll
                    for (int e = 0; e < 16; ++e) v += w[e];
                    upto = v;
#pragma unroll
                    for (int m = 1; m < 64; m *= 2) {
                        const double x = __shfl_up(upto, m);
                        if (lane >= m) upto += x;
                    }
                    double run = r_before == INFINITY ? -INFINITY : r_before + (upto - v);
                    int hit = -1, end = -1;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        run += w[e];
                        if (w[e] > 0) end = 16 * lane + e;
                        if (w[e] > 0 && hit < 0 && run > mark) hit = 16 * lane + e;
                    }
                    const uint64_t hits = __ballot(hit >= 0), ends = __ballot(end >= 0);
                    if (hits) next = r * kRange + __shfl(hit, __builtin_ctzll(hits));
                    else if (ends) next = r * kRange + __shfl(end, 63 - __builtin_clzll(ends));
                }
                break;
            }
            node = considered = child;
        }
        if (lane == count) path = node;
        ++count;
    }
    if (wave == 0) {
        if (lane < t) a.path[at + lane] = path;
        if (lane == 0) a.n_path[b] = count, a.next[b] = next;
    }
}

}  // namespace

size_t verify_workspace_bytes(int, int, int) { return 0; }

hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream) {
    const dim3 grid(a.batch), block(64 * kWaves);
    const bool logits = a.form == KVARN_LOGITS && a.uniform;
    if (a.bf16) {
        if (logits) hipLaunchKernelGGL((k_verify<1, 1>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_verify<1, 0>), grid, block, 0, stream, a);
    } else {
        if (logits) hipLaunchKernelGGL((k_verify<0, 1>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_verify<0, 0>), grid, block, 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace kvarn
