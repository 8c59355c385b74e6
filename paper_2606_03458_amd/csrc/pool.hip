// Block tables and the map of a ragged batch's tokens (include/kvarn.h, kvarn_assign_blocks, kvarn_token_map).
#include <algorithm>

#include "common.hpp"
#include "lanes.hpp"

namespace kvarn {
namespace {

// What one sequence does: blocks before and after.
struct Move {
    int have, need;  // have < 0: an invalid count
    bool full;       // needs more than max_blocks
    __device__ int more() const { return max(need - have, 0); }
    __device__ int less() const { return max(have - need, 0); }
};
__device__ __forceinline__ Move move_of(const BlockArgs& a, int b) {
    const int have = a.pool.n_blocks[b], length = (a.lengths ? a.lengths : a.c.seq_len)[b];
    const int64_t body = (int64_t)length + a.extra - a.n_sink, need = body > 0 ? body / kG : 0;
    if (have < 0 || have > a.c.max_blocks) return Move{-1, -1, false};
    if (length < 0) return Move{have, have, false};
    if (need > a.c.max_blocks) return Move{have, have, true};
    return Move{have, (int)need, false};
}

// Every workgroup forms the running sums of what all sequences take and give: thread i those of share i of the
// sequences, as doubles, in which they are exact below 2^53.  A share's first kHeld sequences are kept in LDS.  Then
// each wave moves blocks, 512 of one sequence's row at a time.  The ring's free ids are read from its beginning, and what
// is given back is written behind them, in places that hold no free id, so no order between the workgroups is needed.
// Where more is taken than was free, the k-th block taken is the (k - count)-th given back: whoever takes it reads
// it from the giver's row and clears it there, and the giver leaves it alone.  Counts change after all have read them:
// the workgroup that ends last writes them (ring[2] counts those that have ended, and is 0 again afterwards).
// Bound by latency: counts, sums, ids, the last workgroup's arrival and its stores, one after the other.  64 sequences of which none
// needs a block 5.1 us, 1024 of which a quarter end and a quarter begin (89 000 blocks taken, as many given) 9.5.  Of four waves and 256
// workgroups 10.2, 512 of them 12.5 (each reads all counts and arrives at one word, some 10 ns), of 16 waves and 64 11.5.
constexpr int kPoolWaves = 8, kShares = 64 * kPoolWaves, kHeld = 2, kMoved = 512;
struct PoolLds {
    double took[kShares * kHeld], gave[kShares * kHeld];  // blocks taken and given by the sequences before
    Move move[kShares * kHeld];
    double totals[2][kPoolWaves];
    int last;
};
__global__ __launch_bounds__(kShares) void k_assign_blocks(BlockArgs a, int share, int parts) {
    __shared__ PoolLds lds;
    const int batch = a.c.batch, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int32_t* table = const_cast<int32_t*>(a.c.block_table);
    const int n = a.c.n_phys, first = a.pool.ring[0], count = a.pool.ring[1];
    const int b0 = (int)min((int64_t)tid * share, (int64_t)batch), b1 = min(batch - b0, share) + b0;
    // the share's sequences: those held all at once, then the others
    Move held[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = move_of(a, min(b0 + i, batch - 1));
    double more = 0, less = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        if (b0 + i >= b1) held[i] = Move{0, 0, false};
        more += held[i].more();
        less += held[i].less();
    }
    for (int b = b0 + kHeld; b < b1; ++b) {
        const Move m = move_of(a, b);
        more += m.more();
        less += m.less();
    }
    double x = running(more), y = running(less);
    if (lane == 63) lds.totals[0][wave] = x, lds.totals[1][wave] = y;
    __syncthreads();
    double given = 0;
    x -= more, y -= less;
    for (int w = 0; w < kPoolWaves; ++w) {
        if (w < wave) x += lds.totals[0][w], y += lds.totals[1][w];
        given += lds.totals[1][w];
    }
    const double before = x;
    const bool bad = first < 0 || first >= n || count < 0 || count + given > n;
    const double free = count + given;
    // growth is granted up to the first sequence that the pool does not cover; granted: how much
    double granted = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        lds.took[tid * kHeld + i] = x, lds.gave[tid * kHeld + i] = y, lds.move[tid * kHeld + i] = held[i];
        x += held[i].more(), y += held[i].less();
        if (x <= free) granted = x;
    }
    for (int b = b0 + kHeld; b < b1 && x <= free; ++b) {
        x += move_of(a, b).more();
        if (x <= free) granted = x;
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) granted = fmax(granted, __shfl_xor(granted, m));
    __syncthreads();
    if (lane == 0) lds.totals[0][wave] = granted;
    __syncthreads();
    for (int w = 0; w < kPoolWaves; ++w) granted = fmax(granted, lds.totals[0][w]);
    const int64_t grants = (int64_t)granted;

    uint32_t err = bad && blockIdx.x == 0 ? 8u : 0u;
    const uint32_t items = (uint32_t)batch * (uint32_t)parts, step = gridDim.x * kPoolWaves;
    for (uint32_t id = blockIdx.x * kPoolWaves + wave; id < items; id += step) {
        const int b = (int)(id / (uint32_t)parts), part = (int)(id - (uint32_t)b * parts), of = b / share, i = b - of * share;
        const int at = of * kHeld + min(i, kHeld - 1);
        Move m = lds.move[at];
        int64_t t0 = (int64_t)lds.took[at], g0 = (int64_t)lds.gave[at];
        for (int s = b - i + kHeld; s <= b; ++s) {
            t0 += m.more(), g0 += m.less();
            m = move_of(a, s);
        }
        if (m.have < 0) err |= 8u;
        if (m.full || (m.more() > 0 && t0 + m.more() > grants)) {
            err |= 1u;
            continue;
        }
        if (bad || m.have == m.need) continue;
        int32_t* row = table + (int64_t)b * a.c.max_blocks;
        const int64_t j0 = min(m.have, m.need) + (int64_t)part * kMoved, j1 = min((int64_t)max(m.have, m.need), j0 + kMoved);
        int32_t id_of[kMoved / 64];
        if (m.need > m.have) {
            const int64_t k0 = t0 + (j0 - m.have);
#pragma unroll
            for (int e = 0; e < kMoved / 64; ++e) {
                const int64_t k = k0 + e * 64 + lane, p = first + k;
                if (j0 + e * 64 + lane < j1 && k < count) id_of[e] = a.pool.free_ids[p >= n ? p - n : p];
            }
#pragma unroll
            for (int e = 0; e < kMoved / 64; ++e) {
                const int64_t j = j0 + e * 64 + lane;
                const int64_t k = k0 + e * 64 + lane;
                if (j >= j1) continue;
                if (k >= count) {
                    double r = (double)(k - count);
                    int lo = 0, hi = kShares - 1;  // the last share with gave <= r gives the r-th
                    while (lo < hi) {
                        const int mid = (lo + hi + 1) / 2;
                        if (lds.gave[mid * kHeld] <= r) lo = mid;
                        else hi = mid - 1;
                    }
                    r -= lds.gave[lo * kHeld];
                    int s = lo * share;
                    Move o = move_of(a, s);
                    while (r >= o.less()) r -= o.less(), o = move_of(a, ++s);
                    int32_t* from = table + (int64_t)s * a.c.max_blocks + o.need + (int64_t)r;
                    id_of[e] = *from;
                    *from = -1;
                }
                row[j] = id_of[e];
            }
        } else {
            const int64_t k0 = count + g0 + (j0 - m.need);  // (what is below grants is taken again at once)
#pragma unroll
            for (int e = 0; e < kMoved / 64; ++e)
                if (j0 + e * 64 + lane < j1 && k0 + e * 64 + lane >= grants) id_of[e] = row[j0 + e * 64 + lane];
#pragma unroll
            for (int e = 0; e < kMoved / 64; ++e) {
                const int64_t k = k0 + e * 64 + lane, p = first + k;
                if (j0 + e * 64 + lane >= j1 || k < grants) continue;
                a.pool.free_ids[p >= n ? p - n : p] = id_of[e];
                row[j0 + e * 64 + lane] = -1;
            }
        }
    }
    if (err && lane == 0 && a.c.err_word) __hip_atomic_fetch_or(a.c.err_word, err, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // Nothing that a workgroup has written is read by another here, only the counts must not change before all have read
    // them, and every count that a wave loads it has used before this barrier: no write-back of the L2 is needed (12.6 us
    // in place of 15.4).
    __syncthreads();
    if (tid == 0)
        lds.last = __hip_atomic_fetch_add(a.pool.ring + 2, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    __syncthreads();
    if (!lds.last) return;
    if (!bad) {
        x = before;
        for (int b = b0; b < b1; ++b) {
            Move m;
            if (b - b0 < kHeld) m = lds.move[tid * kHeld + (b - b0)];
            else m = move_of(a, b);
            x += m.more();
            if (m.need < m.have || (m.need > m.have && x <= granted)) a.pool.n_blocks[b] = m.need;
        }
    }
    if (tid == 0) {
        if (!bad) {
            const int64_t p = first + grants;
            a.pool.ring[0] = (int)(p >= n ? p - n : p);
            a.pool.ring[1] = (int)(count + (int64_t)given - grants);
        }
        a.pool.ring[2] = 0;
    }
}

// The last b in 0 .. batch - 1 with cu[b] <= t (0 where there is none), by a whole wave: 64 probes a step.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int batch, int64_t t, int lane) {
    int lo = 0, n = batch;  // the answer is in lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const uint64_t below = __ballot(lane * step < n && cu[min(i, batch - 1)] <= t);
        const int at = below ? 63 - __builtin_clzll(below) : 0;
        n = min(step, n - at * step);
        lo += at * step;
    }
    return lo;
}

// A wave per 256 tokens, 64 side by side.  The first one's sequence is found by 64 probes at a time; where the next 64
// ends of sequences reach behind the wave's last token the lanes hold them, with the sequences' starts, and look a
// token's sequence up among them by halving, otherwise (many short or empty sequences) in memory.  Bound by latency,
// then by the stores: 524309 tokens of
// 193 sequences, paged, 6.6 us (8.4 MB); with four tokens side by side in a lane, each sequence looked up in memory, 8.6.
__global__ __launch_bounds__(256) void k_token_map(MapArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t t0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 256, end = min(a.n_tokens, (int64_t)a.cu[a.c.batch]);
    const int first = sequence_of(a.cu, a.c.batch, t0, lane);
    if (t0 >= end) return;
    const int64_t stop = min(t0 + 256, end);
    // lane i: where sequence first + i begins and ends (behind the last sequence, nowhere), and its start
    const int own = min(first + lane, a.c.batch - 1);
    const int from = a.cu[own], to = first + lane < a.c.batch ? a.cu[own + 1] : INT32_MAX, at = a.start ? a.start[own] : 0;
    const bool here = __shfl(to, 63) >= stop;
    const int64_t batch = a.c.batch, sink = a.n_sink;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t t = t0 + e * 64 + lane;
        int b, c0, c1, s0;
        if (here) {
            int lo = 0;  // ends at or before t
#pragma unroll
            for (int step = 32; step > 0; step /= 2)
                if (__shfl(to, lo + step - 1) <= t) lo += step;
            b = min(first + lo, a.c.batch - 1);
            c0 = __shfl(from, lo), c1 = __shfl(to, lo), s0 = __shfl(at, lo);
        } else {
            int lo = first, hi = a.c.batch - 1;
            while (lo < hi) {
                const int mid = lo + (hi - lo + 1) / 2;
                if (a.cu[mid] <= t) lo = mid;
                else hi = mid - 1;
            }
            b = lo;
            c0 = a.cu[b], c1 = a.cu[b + 1], s0 = a.start ? a.start[b] : 0;
        }
        if (t >= stop) continue;
        const int64_t start = s0, pos = start + (t - c0);
        if (a.seq) a.seq[t] = b;
        if (a.position) a.position[t] = pos >= INT32_MIN && pos <= INT32_MAX ? (int)pos : -1;
        if (!a.row) continue;
        int64_t row = -1;
        if (pos >= 0 && pos < INT32_MAX) {
            if (pos < sink) {
                row = b * sink + pos;
            } else {
                const int64_t body = pos - sink, blk = body / kG, r = body % kG;
                if (blk >= (start + ((int64_t)c1 - c0) - sink) / kG) {
                    row = batch * sink + (int64_t)b * kG + r;
                } else if (blk < a.c.max_blocks) {
                    int64_t tile = (int64_t)b * a.c.max_blocks + blk;
                    if (a.c.block_table) {
                        tile = a.c.block_table[tile];
                        if (tile < 0 || tile >= a.c.n_phys) {
                            tile = -1;
                            if (a.c.err_word) __hip_atomic_fetch_or(a.c.err_word, 2u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        }
                    }
                    if (tile >= 0) row = batch * (sink + kG) + tile * kG + r;
                }
            }
        }
        a.row[t] = row;
    }
}

}  // namespace

hipError_t launch_assign_blocks(const BlockArgs& a, hipStream_t stream) {
    // A wave per 512 entries of a sequence's row, on at most 192 workgroups, each of which reads all counts.
    const int share = (a.c.batch + kShares - 1) / kShares, parts = std::max(1, (int)(((int64_t)a.c.max_blocks + kMoved - 1) / kMoved));
    if ((int64_t)a.c.batch * parts > INT32_MAX) return hipErrorInvalidValue;  // (a table beyond any memory)
    const int64_t groups = std::min<int64_t>(192, ((int64_t)a.c.batch * parts + kPoolWaves - 1) / kPoolWaves);
    hipLaunchKernelGGL(k_assign_blocks, dim3((unsigned)groups), dim3(kShares), 0, stream, a, share, parts);
    return hipGetLastError();
}

hipError_t launch_token_map(const MapArgs& a, hipStream_t stream) {
    const int64_t groups = (a.n_tokens + 1023) / 1024;
    if (groups > 0xFFFFFFFFll / 256) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_token_map, dim3((unsigned)groups), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace kvarn
