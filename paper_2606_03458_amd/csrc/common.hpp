// Shared device/host definitions of libkvarn (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvarn.h"
#include "plan.hpp"

namespace kvarn {

constexpr int kD = 128;  // head_dim (channels per token)
constexpr int64_t kMaxStreams = int64_t(1) << 26;  // (sequence, kv head) pairs a cache may hold

// 1/sqrt(128), rounded to fp32.
constexpr float kInvSqrt128 = 0.08838834764831845f;
constexpr float kLog2e = 1.4426950408889634f;

// aux bytes per tile: three fp32 vectors, or the compact binary16 b + E4M3 a + E4M3 s2
__host__ __device__ inline size_t aux_bytes(int compact) { return compact ? 512 : 3 * 128 * sizeof(float); }
__host__ __device__ inline size_t code_bytes(int bits) { return (size_t)bits * 2048; }
__host__ __device__ inline size_t tile_bytes(int bits, int compact) { return code_bytes(bits) + aux_bytes(compact); }

__device__ __forceinline__ float bf16_to_f32(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }

// fp32 -> bf16, round to nearest even (NaN stays NaN).
__device__ __forceinline__ uint16_t f32_to_bf16(float f) {
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (uint16_t)((u >> 16) | 0x40u);
    u += 0x7FFFu + ((u >> 16) & 1u);
    return (uint16_t)(u >> 16);
}

// Two values to a pair of bf16 in one instruction (round to nearest even, NaN stays NaN).
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, v2bf{(__bf16)lo, (__bf16)hi});
}

// Body tile blk of (sequence b, kv head kh) in the cache's tiles: dense [batch][n_kv][max_blocks],
// or paged (tile kh of pool block block_table[b][blk]).  -1 (and bit 1 of err_word) for a pool
// id outside [0, n_phys).  thread: the caller's, among those that ask together.
__device__ __forceinline__ int64_t body_tile(const kvarn_cache& c, int b, int kh, int blk, int thread = threadIdx.x) {
    if (!c.block_table) return ((int64_t)b * c.n_kv + kh) * c.max_blocks + blk;
    const int id = c.block_table[(size_t)b * c.max_blocks + blk];
    if (id < 0 || id >= c.n_phys) {
        if (thread == 0 && c.err_word)
            __hip_atomic_fetch_or(c.err_word, 2u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return -1;
    }
    return (int64_t)id * c.n_kv + kh;
}

// 16 bytes of a result that this kernel reads again seldom or never, stored past the caches.  For stores that fill
// whole lines, of 128 bytes: parts of lines cost more there (where rows of 256 bytes are 272 apart: 126 us past
// the caches, 94 through them, for rows read back that take 56 and 73 where they fill lines).
__device__ __forceinline__ void store_once(void* p, uint4 v) {
    typedef uint32_t v4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(v4{v.x, v.y, v.z, v.w}, reinterpret_cast<v4*>(p));
}
__device__ __forceinline__ void store_once(void* p, float4 v) {
    typedef float v4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(v4{v.x, v.y, v.z, v.w}, reinterpret_cast<v4*>(p));
}

// Quantizer constants, as passed to kernels.
struct QParams {
    int bits;
    int iters;
    float var_min, var_max, log_lo, log_hi;
    int compact;  // aux format: 0 fp32, 1 compact
    int rotate;   // 1: Hadamard rotation along head_dim before VarN; 0: none (ablations)
};

// Kernel launchers (defined in the .hip files; called by the host API).
hipError_t launch_quantize_tiles(const QParams& qp, int kind, const void* x, bool x_bf16, int64_t n_outer,
                                 int64_t n_inner, int64_t x_outer, int64_t x_inner, int64_t x_token, void* out,
                                 int64_t out_outer, int64_t out_inner, int32_t* best_iter, hipStream_t stream);

// all_due: the caller knows every sequence completes a group with this token (lock-step
// decode): one workgroup per tile.  Otherwise a resident-size grid checks the tiles.
hipError_t launch_flush(const QParams& qp, const kvarn_cache& c, int n_sink, bool all_due, hipStream_t stream);

hipError_t launch_prefill(const QParams& qp, const kvarn_cache& c, int n_sink, const void* k, const void* v,
                          bool x_bf16, const int32_t* cu_seqlens, int max_len, hipStream_t stream);

hipError_t launch_append(const kvarn_cache& c, int n_sink, const void* k_new, const void* v_new, bool bf16,
                         hipStream_t stream);

size_t decode_workspace_bytes(int batch, int n_q, const DecodePlan& plan);

// A lock-step decode step's token, appended by the decode launch itself (bf16 or fp32 rows
// [batch][n_kv][128], 16-byte aligned, fp32 only for dense bodies; len_before >= n_sink and the token
// does not fill the residual).
struct StepAppend {
    int len_before;
    const void* k_new;
    const void* v_new;
    bool f32;
};
hipError_t launch_decode(const kvarn_cache& c, int bits, int compact, int rotate, int n_sink, int n_q, const void* q,
                         bool q_bf16, void* out, bool out_bf16, float sm_scale, const DecodePlan& plan, float* ws,
                         hipStream_t stream, const StepAppend* step = nullptr);

// The same where `lines`, the stores' rows fill whole lines, else through the caches.
template <class V>
__device__ __forceinline__ void store_row(void* p, V v, bool lines) {
    if (lines) store_once(p, v);
    else *reinterpret_cast<V*>(p) = v;
}
// Whether rows at p, `stride` bytes apart, do.
inline bool fills_lines(const void* p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 128 == 0 && stride % 128 == 0; }

// kvarn_rotary's arguments.
struct RotaryArgs {
    kvarn_rope rope;
    const void *q, *k;
    void *q_out, *k_out;
    int64_t q_stride, q_out_stride, k_stride, k_out_stride;
    int n_q, n_kv, bf16, inverse;
    int64_t n_tokens, tokens_per_seq;
    const int32_t *positions, *seq_start;
    bool lines;  // (set by launch_rotary)
    int n_axes;  // kvarn_rotary_axes; 0: one position per token
    int64_t pos_stride, axis_stride;
    uint64_t axis_of[2];  // the axis of pair i: bits 2 (i % 32) of word i / 32
};
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream);

// kvarn_read_tokens' arguments; kinds 1: only kind0.
struct ReadArgs {
    kvarn_cache c;
    int bits, compact, rotate, n_sink;
    const int32_t* first;
    int n_tokens;
    void *k_out, *v_out;
    int bf16;
    int64_t seq_stride, head_stride, token_stride;
    int kinds, kind0;
    int parts;   // (set by launch_read)
    bool lines;  // (the same)
};
hipError_t launch_read(const ReadArgs& a, hipStream_t stream);

// kvarn_append_path's arguments.
struct PathArgs {
    QParams P;
    kvarn_cache c;
    int n_sink;
    int n_draft, max_path, bf16;
    const void *k, *v;
    int64_t kv_stride;
    const int32_t *path, *n_path;
};
hipError_t launch_append_path(const PathArgs& a, hipStream_t stream);

// kvarn_tree_attention's arguments.
struct TreeArgs {
    kvarn_cache c;
    int bits, compact, rotate, n_sink;
    int n_q, g, n_draft;
    const void* q;
    int64_t q_stride;
    int q_bf16;
    const void *k, *v;
    int64_t kv_stride;
    int kv_bf16;
    const uint64_t* mask;
    const int32_t* n_live;
    void* out;
    int64_t out_stride;
    int out_bf16;
    float scale_log2;  // sm_scale * log2(e): logits are kept in log2 units
    int max_len;
    float* ws;         // [stream][n_chunk][n_wg][16 row_blocks][132] partials when n_wg > 1
    int row_blocks, n_chunk, n_wg, share, waves, order;  // the plan's (set by launch_tree)
};
size_t tree_workspace_bytes(const kvarn_cache& c, int n_sink, int n_q, int n_draft, int max_len);
hipError_t launch_tree(const TreeArgs& a, hipStream_t stream);

// kvarn_verify_drafts' arguments.
struct VerifyArgs {
    int batch, n_draft, vocab;
    const int32_t *tokens, *parent, *n_live;
    const void *target, *draft;
    int64_t target_stride, draft_stride;
    int bf16, form;
    const float *scale, *uniform;
    int32_t *path, *n_path, *next;
    void* ws;
    void* stops;  // in the workspace (set by launch_verify)
    double* sums;
};
size_t verify_workspace_need(int batch, int n_draft, int vocab);   // what calls of this size use, in any mode
size_t verify_workspace_bytes(int batch, int n_draft, int vocab);  // the most that calls of up to this size use
hipError_t launch_verify(const VerifyArgs& a, hipStream_t stream);

// kvarn_assign_blocks' arguments.
struct BlockArgs {
    kvarn_cache c;
    int n_sink;
    kvarn_block_pool pool;
    const int32_t* lengths;
    int extra;
};
hipError_t launch_assign_blocks(const BlockArgs& a, hipStream_t stream);

// kvarn_token_map's arguments.
struct MapArgs {
    kvarn_cache c;
    int n_sink;
    const int32_t *cu, *start;
    int64_t n_tokens;
    int32_t *seq, *position;
    int64_t* row;
};
hipError_t launch_token_map(const MapArgs& a, hipStream_t stream);

}  // namespace kvarn
