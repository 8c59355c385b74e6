// Block tables and the map of a ragged batch's tokens (include/kvarn.h, kvarn_assign_blocks, kvarn_token_map).
#include "common.hpp"

namespace kvarn {
namespace {

// What one sequence does: blocks before and after, and how many it takes or gives.
struct Move {
    int have, need;  // have < 0: an invalid count
    bool full;       // needs more than max_blocks
    __device__ int64_t more() const { return max(need - have, 0); }
    __device__ int64_t less() const { return max(have - need, 0); }
};
__device__ __forceinline__ Move move_of(const BlockArgs& a, int b) {
    const int have = a.pool.n_blocks[b];
    Move m{have, have, false};
    if (have < 0 || have > a.c.max_blocks) return Move{-1, -1, false};
    const int length = a.lengths ? a.lengths[b] : a.c.seq_len[b];
    if (length < 0) return m;
    const int64_t body = (int64_t)length + a.extra - a.n_sink, need = body > 0 ? body / kG : 0;
    if (need > a.c.max_blocks) m.full = true;
    else m.need = (int)need;
    return m;
}

// Every workgroup forms the running sums of what all sequences take and give, thread i those of share i of the
// sequences, and moves the blocks of its own share.  The ring's free ids are read from its beginning, and what is
// given back is written behind them, in places that hold no free id, so no order between the workgroups is needed.
// Where more is taken than was free, the k-th block taken is the (k - count)-th given back: whoever takes it reads it
// from the giver's row and clears it there, and the giver leaves it alone.  Counts change after all have read
// them: the workgroup that ends last writes them (ring[2] counts those that have ended, and is 0 again afterwards).
constexpr int kThreads = 256;
__global__ __launch_bounds__(kThreads) void k_assign_blocks(BlockArgs a, int share) {
    __shared__ int64_t took[kThreads], gave[kThreads];  // blocks taken and given by the shares before
    __shared__ int64_t totals[2][kThreads / 64];
    __shared__ int last;
    const int batch = a.c.batch, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t* table = const_cast<int32_t*>(a.c.block_table);
    const int b0 = (int)min((int64_t)tid * share, (int64_t)batch), b1 = min(batch - b0, share) + b0;
    int64_t more = 0, less = 0;
    for (int b = b0; b < b1; ++b) {
        const Move m = move_of(a, b);
        more += m.more();
        less += m.less();
    }
    int64_t x = more, y = less;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int64_t u = __shfl_up(x, m), v = __shfl_up(y, m);
        if (lane >= m) x += u, y += v;
    }
    if (lane == 63) totals[0][wave] = x, totals[1][wave] = y;
    __syncthreads();
    int64_t given = 0;
    x -= more, y -= less;
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) x += totals[0][w], y += totals[1][w];
        given += totals[1][w];
    }
    took[tid] = x, gave[tid] = y;
    const int n = a.c.n_phys, first = a.pool.ring[0], count = a.pool.ring[1];
    const bool bad = first < 0 || first >= n || count < 0 || count + given > n;
    const int64_t free = count + given;
    // growth is granted up to the first sequence that the pool does not cover; granted: how much
    int64_t granted = 0;
    if (x + more <= free) granted = x + more;
    else
        for (int b = b0; b < b1 && x <= free; ++b) granted = x, x += move_of(a, b).more();
#pragma unroll
    for (int m = 1; m < 64; m *= 2) granted = max(granted, __shfl_xor(granted, m));
    __syncthreads();
    if (lane == 0) totals[0][wave] = granted;
    __syncthreads();
    for (int w = 0; w < kThreads / 64; ++w) granted = max(granted, totals[0][w]);

    uint32_t err = bad && blockIdx.x == 0 ? 8u : 0u;
    const int s0 = blockIdx.x * share, s1 = min(batch - s0, share) + s0;
    int64_t t0 = took[blockIdx.x], g0 = gave[blockIdx.x];
    for (int b = s0; b < s1; ++b) {
        const Move m = move_of(a, b);
        int32_t* row = table + (int64_t)b * a.c.max_blocks;
        if (m.have < 0) err |= 8u;
        if (m.full || (m.more() > 0 && t0 + m.more() > granted)) {
            err |= 1u;
        } else if (!bad) {
            for (int j = m.have + tid; j < m.need; j += kThreads) {
                const int64_t k = t0 + (j - m.have);
                int id;
                if (k < count) {
                    const int64_t at = first + k;
                    id = a.pool.free_ids[at >= n ? at - n : at];
                } else {
                    int64_t r = k - count;
                    int lo = 0, hi = kThreads - 1;  // the last share with gave <= r gives the r-th
                    while (lo < hi) {
                        const int mid = (lo + hi + 1) / 2;
                        if (gave[mid] <= r) lo = mid;
                        else hi = mid - 1;
                    }
                    r -= gave[lo];
                    int s = lo * share;
                    Move o = move_of(a, s);
                    while (r >= o.less()) r -= o.less(), o = move_of(a, ++s);
                    int32_t* from = table + (int64_t)s * a.c.max_blocks + o.need + r;
                    id = *from;
                    *from = -1;
                }
                row[j] = id;
            }
            for (int j = m.need + tid; j < m.have; j += kThreads) {
                const int64_t k = count + g0 + (j - m.need);
                if (k < granted) continue;  // taken again at once
                const int64_t at = first + k;
                a.pool.free_ids[at >= n ? at - n : at] = row[j];
                row[j] = -1;
            }
        }
        t0 += m.more(), g0 += m.less();
    }
    if (err && tid == 0 && a.c.err_word) __hip_atomic_fetch_or(a.c.err_word, err, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (tid == 0)
        last = __hip_atomic_fetch_add(a.pool.ring + 2, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    if (!bad) {
        x = took[tid];
        for (int b = b0; b < b1; ++b) {
            const Move m = move_of(a, b);
            x += m.more();
            if (m.need < m.have || (m.need > m.have && x <= granted)) a.pool.n_blocks[b] = m.need;
        }
    }
    if (tid == 0) {
        if (!bad) {
            const int64_t at = first + granted;
            a.pool.ring[0] = (int)(at >= n ? at - n : at);
            a.pool.ring[1] = (int)(free - granted);
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

// Four tokens per thread.  A workgroup's first and last sequence are found by 64 probes at a time, a thread's own
// between them by halving.
__global__ __launch_bounds__(256) void k_token_map(MapArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t t0 = (int64_t)blockIdx.x * 1024, end = min(a.n_tokens, (int64_t)a.cu[a.c.batch]);
    if (t0 >= end) return;
    int lo = sequence_of(a.cu, a.c.batch, t0, lane);
    int hi = sequence_of(a.cu, a.c.batch, min(t0 + 1024, end) - 1, lane);
    const int64_t t = t0 + threadIdx.x * 4;
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (a.cu[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    int b = lo;
    for (int e = 0; e < 4 && t + e < end; ++e) {
        while (b + 1 < a.c.batch && a.cu[b + 1] <= t + e) ++b;
        const int64_t c0 = a.cu[b], start = a.start ? a.start[b] : 0, pos = start + (t + e - c0);
        if (a.seq) a.seq[t + e] = b;
        if (a.position) a.position[t + e] = pos >= INT32_MIN && pos <= INT32_MAX ? (int)pos : -1;
        if (!a.row) continue;
        const int64_t length = start + ((int64_t)a.cu[b + 1] - c0), batch = a.c.batch, sink = a.n_sink;
        int64_t row = -1;
        if (pos >= 0 && pos < INT32_MAX) {
            if (pos < sink) {
                row = b * sink + pos;
            } else {
                const int64_t body = pos - sink, blk = body / kG, r = body % kG;
                if (blk >= (length - sink) / kG) {
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
        a.row[t + e] = row;
    }
}

}  // namespace

hipError_t launch_assign_blocks(const BlockArgs& a, hipStream_t stream) {
    const int share = (a.c.batch + kThreads - 1) / kThreads, groups = (a.c.batch + share - 1) / share;
    hipLaunchKernelGGL(k_assign_blocks, dim3(groups), dim3(kThreads), 0, stream, a, share);
    return hipGetLastError();
}

hipError_t launch_token_map(const MapArgs& a, hipStream_t stream) {
    const int64_t groups = (a.n_tokens + 1023) / 1024;
    if (groups > 0xFFFFFFFFll / 256) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_token_map, dim3((unsigned)groups), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace kvarn
