/*
 * kvarn.h -- C ABI of libkvarn, the KVarN hot path for AMD Instinct MI355X (gfx950).
 *
 * KVarN (arXiv 2606.03458) stores a transformer's K/V cache in three regions (App. D,
 * "Quantization"): the first n_sink tokens of a sequence in 16-bit, a body of quantized
 * 128-token groups, and a residual of the most recent tokens that do not yet fill a group.
 * A group (one 128-token x 128-channel tile of K or of V for one sequence and kv head) is
 * quantized by (Fig. 2, Sec. 3.3):
 *   1. a Hadamard rotation of every token along head_dim (Sec. 2.2, App. A),
 *   2. VarN, alternating log-domain variance normalisation of columns and rows with best-
 *      imbalance tracking (App. H, Algorithm 1; rows = tokens, columns = channels),
 *   3. asymmetric round-to-nearest (Sec. 2.1, Eq. 1): keys per channel, values per token,
 *   4. dual-scale storage with the Sinkhorn scale of the group axis absorbed into the RTN
 *      scale and offset (App. D, "Effective memory overhead").
 * Decode attention reads the packed body, dequantizes with the second scale fused (App. I)
 * and attends over sink + body + residual.
 *
 * Conventions for every entry point:
 *   - All pointers to tensors are DEVICE pointers, owned by the caller, and must stay valid
 *     until the work queued on `stream` has run.  The library allocates no device memory at
 *     run time; its code object holds one static scratch array per device, used only by
 *     kvarn_decode_attention_noalloc.
 *   - Every call only enqueues work on `stream` (asynchronous); none synchronizes.
 *   - Arguments are validated on the host before anything is enqueued.  A failed check
 *     returns a negative kvarn_status and enqueues nothing.  KVARN_EHIP reports a failed
 *     kernel launch.  The library never aborts and throws nothing across this ABI.
 *   - Calls on different caches may run concurrently; calls that touch the same cache must
 *     be ordered by the caller (same stream or events).
 *   - head_dim and the group size are fixed at 128.
 *
 * Packed tile (the library's storage format; the paper fixes only what is stored per group):
 *   bytes [0, bits*2048)          128 x 128 codes of `bits` bits (layout below)
 *   then the aux, in one of two formats (kvarn_params.aux_format):
 *   KVARN_AUX_F32:
 *     512 bytes   a[128]  fp32   keys: RTN scale of channel c times its Sinkhorn channel
 *                                scale; values: of token t
 *     512 bytes   b[128]  fp32   the matching offset (group minimum times the same scale)
 *     512 bytes   s2[128] fp32   second scale: keys per token, values per channel (the other
 *                                Sinkhorn scale)
 *     Tile size 5632 bytes at 2 bits (2.75 bits/element), 9728 at 4 bits.
 *   KVARN_AUX_COMPACT (App. D, "Effective memory overhead": per group of 128 values, both
 *   scales in an 8-bit float format and the zero point in a 16-bit one):
 *     256 bytes   b[128]  IEEE binary16, little-endian
 *     128 bytes   a[128]  OCP E4M3 (4-bit exponent, bias 7, 3-bit mantissa, largest 448)
 *     128 bytes   s2[128] OCP E4M3
 *     s2 is rounded to nearest first and the tile is quantized against the stored s2; a is the
 *     RTN step rounded upward (the stored range covers the group), b the nearest binary16 of
 *     the group minimum, and codes are chosen for the stored a and b.  Scales are kept within
 *     [2^-6, 448] and b within +-65504.  When the largest step of a tile exceeds 448, a
 *     tile-wide power of two 2^e moves from a and b into s2 (the smallest e that fits, as far
 *     as the largest s2 stays within 448; only when no other-axis scale is below 2^-6), which
 *     leaves every dequantized value unchanged.  Tile size 4608 bytes at 2 bits (2.25 bits/element),
 *     8704 at 4 bits.
 *   Dequantized rotated tile, both formats: keys (code[t][c]*a[c] + b[c]) * s2[t]; values
 *   (code[t][c]*a[t] + b[t]) * s2[c]; un-rotate each token with the orthonormal Hadamard
 *   matrix.
 *   Code layout: codes form units of 16; a unit is bits/2 little-endian 32-bit words.  With
 *   u = 512*sigma + 8*L + w (L in 0..63, w in 0..7) and p = 8/bits, unit u starts at word
 *   512*(bits/2)*sigma + 256*(w/p) + 4*L + (bits/2)*(w%p).  Code e = 4*s + q (s, q in 0..3)
 *   of a unit sits in word s/p of the unit, at bit 8*q + bits*(s%p).  For token t, channel c,
 *   sigma = t/64:
 *     keys:   u = (sigma*64 + 16*((c%64)/16) + t%16)*8 + 2*((t%64)/16) + c/64,  e = c % 16
 *     values: u = (sigma*64 + 16*((t%16)/4) + c%16)*8 + c/16,  e = 4*((t%64)/16) + t%4
 *   (Each 64-token half of a tile is the register image of 64 GPU lanes x 8 units: lane L
 *   holds units 8L .. 8L+7 as 2 or 4 pieces of 16 bytes, piece k at byte 1024*k + 16*L of
 *   the half, so that each 16-byte load of a wave reads 1 KB of consecutive bytes.)
 */
#ifndef KVARN_H
#define KVARN_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KVARN_API __attribute__((visibility("default")))

typedef enum {
    KVARN_OK = 0,
    KVARN_EINVAL = -1,       /* null pointer, bad size, stride or dtype                      */
    KVARN_EUNSUPPORTED = -2, /* valid request the library does not implement (e.g. bits=3)  */
    KVARN_ECAPACITY = -3,    /* the cache has no room for the requested tokens              */
    KVARN_EHIP = -4,         /* a HIP launch or query failed                                */
    KVARN_EWORKSPACE = -5    /* workspace missing or smaller than kvarn_decode_workspace_bytes */
} kvarn_status;

typedef enum { KVARN_F32 = 0, KVARN_BF16 = 1 } kvarn_dtype;
typedef enum { KVARN_KEYS = 0, KVARN_VALUES = 1 } kvarn_kind;

/* Quantizer constants (App. H, Algorithm 1).  kvarn_params_init fills the defaults. */
typedef struct {
    int32_t bits;       /* 2 or 4                                                      */
    int32_t varn_iters; /* K of Algorithm 1: 8 (runtime experiment, Sec. 4.2); 0..64      */
    int32_t n_sink;     /* tokens kept in bf16 at the start of a sequence: 0 or up to 1024 */
    float var_min;      /* c_min: variances are clamped to [var_min, var_max]; 1e-8     */
    float var_max;      /* c_max: 1e8 (the paper gives no values for c_min, c_max)      */
    float log_lo;       /* clamp of the cumulative log-scales: -0.3 (Algorithm 1)       */
    float log_hi;       /* 10.0 (Algorithm 1)                                           */
    int32_t aux_format; /* KVARN_AUX_F32 (default) or KVARN_AUX_COMPACT                  */
    int32_t rotate;     /* 1 (default): Hadamard rotation before VarN, as KVarN does.  0: no
                         * rotation -- with varn_iters = 0 the quantizer is KIVI-style RTN,
                         * with varn_iters > 0 VarN alone (the ablations of Fig. 1).  Tiles
                         * then hold the unrotated domain and decode skips both rotations;
                         * every call on one cache must use the same value. */
} kvarn_params;
typedef enum { KVARN_AUX_F32 = 0, KVARN_AUX_COMPACT = 1 } kvarn_aux_format;
/* Accepted ranges (else KVARN_EINVAL): 1e-30 <= var_min <= var_max <= 1e30 and
 * -40 <= log_lo <= log_hi <= 40, which keeps every scale exp(+-L) and every log of a clamped
 * variance inside the normal fp32 range. */

/* The cache of `batch` sequences with n_kv kv heads each (a model's layers may be folded
 * into batch; batch * n_kv at most 2^26, else KVARN_EINVAL).  Device buffers, all
 * caller-allocated (sizes from kvarn_cache_sizes):
 *   k_body, v_body   [batch][n_kv][max_blocks] packed tiles of kvarn_tile_bytes(p)
 *   k_resid, v_resid [batch][n_kv][128][128]    bf16, tokens as given (unrotated)
 *   k_sink, v_sink   [batch][n_kv][n_sink][128] bf16, or NULL when n_sink == 0
 *   seq_len          [batch] int32: tokens held by each sequence (all regions)
 *   err_word         one uint32 or NULL: a kernel that finds no room sets bit 0 and drops
 *                    the write instead of writing out of bounds (a backstop only: the host
 *                    check of kvarn_append_token catches overflow from its length hint); an
 *                    invalid block id (below) sets bit 1; a fused append step over a
 *                    sequence whose length is not the host's (kvarn_append_decode) sets bit 2.
 *   block_table      NULL for the dense body above.  Otherwise the paged layout of serving
 *                    engines: block_table is [batch][max_blocks] int32 on the device and
 *                    k_body, v_body are pools of n_phys blocks, [n_phys][n_kv] tiles each;
 *                    body tile blk of (sequence b, kv head h) is tile h of pool block
 *                    block_table[b][blk].  Only the entries of tiles a call touches are read.
 *                    An id outside [0, n_phys) sets bit 1 of err_word; kvarn_tree_attention then
 *                    leaves out the sequence's body, decode this tile and others of the sequence
 *                    (which ones depends on the launch), and flush / prefill do not write the
 *                    tile.  (Bit 3: an invalid path, kvarn_append_path, or an invalid count of blocks,
 *                    kvarn_assign_blocks.)
 *   n_phys           pool size in blocks, when block_table is set (pool bytes: n_phys * n_kv *
 *                    kvarn_tile_bytes(p) for each of k_body and v_body).
 * A sequence of length L holds min(L, n_sink) sink tokens, (L - n_sink)/128 body tiles and
 * (L - n_sink) % 128 residual tokens (0 body and residual tokens while L <= n_sink). */
typedef struct {
    int32_t batch, n_kv, max_blocks;
    void *k_body, *v_body;
    void *k_resid, *v_resid;
    void *k_sink, *v_sink;
    int32_t *seq_len;
    uint32_t *err_word;
    const int32_t *block_table;
    int32_t n_phys;
} kvarn_cache;

/* Fill `p` with the defaults for `bits` (2 or 4; fp32 aux).  Returns KVARN_EINVAL for a null
 * `p`, KVARN_EUNSUPPORTED for other bit widths. */
KVARN_API int kvarn_params_init(kvarn_params *p, int32_t bits);

/* Bytes of one packed tile for p's bits and aux format (5632 / 9728 with fp32 aux, 4608 / 8704
 * compact); 0 for invalid parameters. */
KVARN_API size_t kvarn_tile_bytes(const kvarn_params *p);

/* Byte sizes of the seven cache buffers, in the order k_body, v_body, k_resid, v_resid,
 * k_sink, v_sink, seq_len.  Returns KVARN_EINVAL for null pointers or non-positive sizes. */
KVARN_API int kvarn_cache_sizes(const kvarn_params *p, int32_t batch, int32_t n_kv, int32_t max_blocks, size_t sizes[7]);

/*
 * Quantize n_outer x n_inner independent tiles (Fig. 2: Hadamard, VarN, RTN, pack).
 *   kind    KVARN_KEYS (RTN per channel) or KVARN_VALUES (RTN per token)
 *   x       tile (i, j) starts at element x + i*x_outer_stride + j*x_inner_stride; token t of
 *           it at + t*x_token_stride; its 128 channels are contiguous.  dtype fp32 or bf16.
 *           The input is unrotated: the library applies the Hadamard rotation.
 *   out     tile (i, j) is written at byte out + (i*out_outer_stride + j*out_inner_stride) *
 *           kvarn_tile_bytes(p) (strides counted in tiles).
 *   best_iter  optional [n_outer*n_inner] int32 (row-major over (i, j)): the VarN iteration
 *           whose scales were kept (0 = the initial unit scales); NULL to skip.
 * Strides must be non-negative, x_token_stride >= 128; x, and every x stride times the
 * element size, must be multiples of 16 bytes (rows are read as 16-byte vectors); out must
 * be 16-byte aligned.  n_outer or n_inner == 0 is a no-op.
 * Prefill: quantize [batch*n_kv][T/128] tiles straight into k_body / v_body and set seq_len.
 */
KVARN_API int kvarn_quantize_block(const kvarn_params *p, int32_t kind, const void *x, int32_t x_dtype, int64_t n_outer,
                         int64_t n_inner, int64_t x_outer_stride, int64_t x_inner_stride, int64_t x_token_stride,
                         void *out, int64_t out_outer_stride, int64_t out_inner_stride, int32_t *best_iter,
                         hipStream_t stream);

/*
 * Prefill whole prompts of different lengths in one call (the bulk write before decode):
 *   k, v        [total_tokens][n_kv][128] in `dtype` (fp32 or bf16), unrotated, 16-byte
 *               aligned; sequence b owns rows cu_seqlens[b] .. cu_seqlens[b+1] - 1
 *   cu_seqlens  [batch + 1] int32 on the device: row offsets, non-decreasing, cu_seqlens[0] = 0
 *   max_len     host bound on the prompt lengths; it sizes the launch
 * Each sequence's contents are replaced by its prompt of length L: seq_len[b] = L, the first
 * min(L, n_sink) tokens go to the sink, every full 128-token group after them is quantized
 * (Fig. 2) into body tiles 0, 1, ... (through block_table when paged), and the remaining
 * (L - n_sink) % 128 tokens go to the residual, as the same tokens appended one by one would
 * leave them.  Sink and residual are stored as bf16.  A sequence with L > max_len or needing
 * more than max_blocks tiles is not written: its seq_len is set to 0 and bit 0 of err_word is
 * set.  Returns KVARN_EINVAL for null or misaligned pointers, a bad dtype or max_len < 0.
 */
KVARN_API int kvarn_prefill(const kvarn_params *p, const kvarn_cache *cache, const void *k, const void *v,
                            int32_t dtype, const int32_t *cu_seqlens, int32_t max_len, hipStream_t stream);

/*
 * Append one token to every (sequence, kv head) (the streaming write of Fig. 4's pseudo-decode):
 *   k_new, v_new  [batch][n_kv][128] in `dtype` (fp32 or bf16; stored as bf16, unrotated).
 * The token goes to the sink while a sequence is shorter than n_sink, otherwise to the
 * residual; a residual that reaches 128 tokens is quantized (keys and values) into the next
 * body tile and emptied, within this call.  seq_len is incremented on the device.
 *   host_len_before  the common length of all sequences before this call (lock-step decode),
 *           used to check capacity on the host and to launch the flush only when one is due;
 *           pass -1 if lengths differ or are unknown: the flush kernel then runs every call
 *           on a grid of resident size (768 workgroups) whose workgroups check the tiles in
 *           turn, each sequence deciding on the device, and overflow is caught by err_word only.
 * Returns KVARN_ECAPACITY (enqueuing nothing) if the hint shows that a flush would need body
 * tile max_blocks.
 */
KVARN_API int kvarn_append_token(const kvarn_params *p, const kvarn_cache *cache, const void *k_new, const void *v_new,
                       int32_t dtype, int32_t host_len_before, hipStream_t stream);

/* Workspace bytes that kvarn_decode_attention asks for with these sizes: room for the partials of
 * (sequence, kv head) pairs that take several workgroups; 0 for 256 pairs (for more than 8 query heads
 * per kv head, each counted ceil(heads / 8) times) and more, for short sequences, and when an argument
 * is invalid.  A call may write fewer partials than there is room for, or none, but a buffer of this
 * size has to be there. */
KVARN_API size_t kvarn_decode_workspace_bytes(const kvarn_params *p, const kvarn_cache *cache, int32_t n_q,
                                    int32_t max_len_hint);

/*
 * Decode attention of one query token per sequence over its whole cache:
 *   out[b][h][:] = softmax(sm_scale * q[b][h] . K^T) V over the sink, body and residual of
 *   sequence b, kv head h / (n_q / n_kv).  The body is dequantized in registers with both
 *   scales fused (App. I); the query is rotated once so body logits are computed in the
 *   rotated domain, and the body's output is rotated back once per query head (App. A).
 *   q    [batch][n_q][128] fp32 or bf16 (post-RoPE, unrotated)
 *   out  [batch][n_q][128] in out_dtype (fp32 or bf16)
 *   max_len_hint  an upper bound of every seq_len (sizes the launch plan)
 *   workspace  device buffer of at least kvarn_decode_workspace_bytes(...) bytes, 16-byte
 *           aligned; may be NULL when that size is 0
 * n_q must be a positive multiple of n_kv with n_q / n_kv <= 16; q 4-byte and out 8-byte
 * aligned.  A sequence of length 0 produces zeros.
 */
KVARN_API int kvarn_decode_attention(const kvarn_params *p, const kvarn_cache *cache, int32_t n_q, const void *q,
                           int32_t q_dtype, void *out, int32_t out_dtype, float sm_scale, int32_t max_len_hint,
                           void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * One decode step of a lock-step batch (Fig. 4: each generated token is appended to the cache,
 * then attended over it, new token included; App. D three-region cache): the results of
 * kvarn_append_token(p, cache, k_new, v_new, kv_dtype, host_len_before) followed by
 * kvarn_decode_attention(p, cache, n_q, q, q_dtype, out, out_dtype, sm_scale,
 * host_len_before + 1, workspace, workspace_bytes), bit for bit, in cache and output.
 *   host_len_before  required: the length of every sequence before the call (seq_len on the
 *           device must hold it).
 *   workspace  as for kvarn_decode_attention with max_len_hint = host_len_before + 1.
 * When the token goes to the residual without filling it, k_new, v_new are 16-byte aligned and the
 * token is bf16 or the body dense, the append runs inside the decode launch: the wave that attends
 * the residual's last chunk reads the new row from k_new / v_new and stores it into the residual,
 * and seq_len is set to host_len_before + 1 without the decode reading it; one launch instead of
 * two.  A sequence whose seq_len is not host_len_before is then left unchanged and bit 2 of err_word
 * is set (its output is not meaningful).  Otherwise (a sink token, a flush, fp32 tokens of a paged
 * cache) the call runs the two entry points' kernels in turn.
 * Errors: those of both entry points, all checked before anything is enqueued; KVARN_EINVAL for
 * host_len_before < 0 or = INT32_MAX.
 */
KVARN_API int kvarn_append_decode(const kvarn_params *p, const kvarn_cache *cache, const void *k_new,
                                  const void *v_new, int32_t kv_dtype, int32_t host_len_before, int32_t n_q,
                                  const void *q, int32_t q_dtype, void *out, int32_t out_dtype, float sm_scale,
                                  void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Decode attention that allocates nothing, for callers that cannot allocate device memory:
 * code under HIP graph capture, tight serving loops, harnesses that forbid allocation.
 * Arguments and results are those of kvarn_decode_attention without the workspace: the workgroups'
 * partials go to a scratch array of KVARN_NOALLOC_SCRATCH_BYTES (32 MiB) that the library
 * holds in static device memory, one array per device, kept until the process ends.  Its
 * device address is looked up once per device (hipGetSymbolAddress, on the first call with
 * that device current, guarded by a mutex); no call allocates or frees anything.
 *   - Plans whose partials need more than KVARN_NOALLOC_SCRATCH_BYTES (as
 *     kvarn_decode_workspace_bytes reports) return KVARN_EWORKSPACE and enqueue nothing.
 *   - Every call on one device shares that device's array: calls that may overlap on one
 *     device (other streams, other host threads) race on it and must be ordered by the
 *     caller.  The array keeps the last call's partials; no call relies on its contents.
 */
#define KVARN_NOALLOC_SCRATCH_BYTES (32u << 20)
KVARN_API int kvarn_decode_attention_noalloc(const kvarn_params *p, const kvarn_cache *cache, int32_t n_q,
                                             const void *q, int32_t q_dtype, void *out, int32_t out_dtype,
                                             float sm_scale, int32_t max_len_hint, hipStream_t stream);

/*
 * Rotary positions.  A head's first rot_dim channels form rot_dim / 2 pairs, and pair i of a token at
 * position m turns by the angle m * freq[i]:
 *   x' = amplitude * (x cos - y sin),  y' = amplitude * (x sin + y cos)
 * Channels from rot_dim on are passed on as they are (amplitude does not touch them).  Keys enter the
 * cache, and queries the attention calls, after this.
 */
typedef enum {
    KVARN_ROPE_HALF = 0,       /* pair i is channels i and i + rot_dim / 2 */
    KVARN_ROPE_INTERLEAVED = 1 /* pair i is channels 2 i and 2 i + 1       */
} kvarn_rope_layout;
typedef struct {
    int32_t rot_dim;    /* even, 2 .. 128                                             */
    int32_t layout;     /* kvarn_rope_layout                                          */
    float amplitude;    /* factor of the rotated channels: 1, or as kvarn_rope_frequencies says; finite */
    const double *freq; /* DEVICE, [rot_dim / 2]: radians per position, finite        */
} kvarn_rope;

/* How the frequencies base^(-2 i / rot_dim) are scaled for contexts `factor` times as long. */
typedef enum {
    KVARN_ROPE_PLAIN = 0,  /* not at all                                                             */
    KVARN_ROPE_LINEAR = 1, /* freq / factor (positions interpolated)                                 */
    KVARN_ROPE_BASE = 2,   /* base * factor^(rot_dim / (rot_dim - 2)): the longest wave is stretched
                            * by factor, the shortest stays                                          */
    KVARN_ROPE_BANDS = 3,  /* by the turns t = original_length * freq / 2 pi over the original length:
                            * t >= high as it is, t <= low freq / factor, between them
                            * (1 - s) freq / factor + s freq with s = (t - low) / (high - low)       */
    KVARN_ROPE_RAMP = 4    /* the same two ends by the pair's index: a pair of t turns has index
                            * d(t) = rot_dim ln(original_length / 2 pi t) / (2 ln base); s falls from
                            * 1 to 0 between floor(d(high)) and ceil(d(low)), both clamped to
                            * [0, rot_dim - 1]; amplitude 0.1 ln(factor) + 1 for factor > 1           */
} kvarn_rope_scaling_kind;
typedef struct {
    int32_t kind;           /* kvarn_rope_scaling_kind                                 */
    double factor;          /* > 0 (not for KVARN_ROPE_PLAIN)                          */
    double original_length; /* > 0: tokens of the contexts trained on (BANDS, RAMP)    */
    double low, high;       /* turns, 0 < low < high (BANDS, RAMP)                     */
} kvarn_rope_scaling;

/* Fills freq[rot_dim / 2] and *amplitude, both in HOST memory, for base > 1; scaling may be NULL (plain).
 * Returns KVARN_EINVAL for null pointers and values outside the ranges above (KVARN_ROPE_BASE needs
 * rot_dim > 2), and where the scaled base or a frequency would leave the range of a double. */
KVARN_API int kvarn_rope_frequencies(int32_t rot_dim, double base, const kvarn_rope_scaling *scaling, double *freq,
                                     double *amplitude);

/*
 * Rotate the heads of n_tokens tokens, queries and keys in one call:
 *   q, k          token t's heads at element t * q_stride (t * k_stride): n_q (n_kv) heads of 128
 *                 channels one after the other, in `dtype` (fp32 or bf16).  n_q or n_kv may be 0 (its
 *                 pointers are then not looked at).
 *   q_out, k_out  the same with strides q_out_stride, k_out_stride.  They may be q and k themselves
 *                 (same pointer and stride: in place); otherwise they must not overlap any input.
 *   positions     DEVICE, [n_tokens] int32, or NULL: the token's index in its sequence
 *   seq_start     DEVICE, [n_tokens / tokens_per_seq] int32 added to the positions of each sequence's
 *                 tokens_per_seq tokens, or NULL.  With a cache's seq_len and positions NULL these are
 *                 the positions of the tokens that come next; with a draft tree's depths as positions,
 *                 those of its drafts.  The sum is taken in 64 bits.
 *   inverse       1: by -m * freq, with the same amplitude (the transposed map: the gradient with
 *                 respect to q and k; with amplitude 1, positions taken off again).  0: as above.
 * tokens_per_seq >= 1 must divide n_tokens.  Strides are in elements, at least the heads' width (for
 * more than one token); pointers are aligned to an element.  Angles are formed in 64 bits, so that far
 * positions keep their precision, and products and sums in 32.  Rows whose pointers and strides are
 * multiples of 16 bytes, with rot_dim a multiple of 16, go 16 bytes at a time; others by pairs.
 * n_tokens == 0 is a no-op.
 */
KVARN_API int kvarn_rotary(const kvarn_rope *rope, const void *q, int32_t n_q, int64_t q_stride, void *q_out,
                           int64_t q_out_stride, const void *k, int32_t n_kv, int64_t k_stride, void *k_out,
                           int64_t k_out_stride, int32_t dtype, int64_t n_tokens, const int32_t *positions,
                           const int32_t *seq_start, int64_t tokens_per_seq, int32_t inverse, hipStream_t stream);

/*
 * Rotary positions with several axes: a token of an image or a video has a time, a height and a width, and
 * each pair of channels turns by one of them,
 *   pair i of a token turns by the angle (positions of the pair's axis) * freq[i],
 * otherwise as kvarn_rotary.  A text token has the same position on every axis.
 */
#define KVARN_MAX_AXES 4
typedef struct {
    int32_t n_axes;   /* 1 .. KVARN_MAX_AXES                              */
    uint8_t axis[64]; /* the axis of pair i < rot_dim / 2, below n_axes   */
} kvarn_rope_axes;
typedef enum {
    KVARN_AXES_SECTIONS = 0, /* the first sections[0] pairs are axis 0's, the next sections[1] axis 1's, ...   */
    KVARN_AXES_IN_TURN = 1   /* pairs go to the axes in turn, passing over one that has its sections[a] already */
} kvarn_axes_order;

/* Fills *axes (HOST memory).  The sections are not negative and add up to rot_dim / 2, else KVARN_EINVAL, as for
 * null pointers and a bad rot_dim, n_axes or order. */
KVARN_API int kvarn_rope_axes_init(kvarn_rope_axes *axes, int32_t rot_dim, int32_t n_axes, const int32_t *sections,
                                   int32_t order);

/*
 * Rotate the heads of n_tokens tokens, queries and keys in one call, as kvarn_rotary with its arguments but for
 *   positions     DEVICE: axis a of token t at element t * pos_stride + a * axis_stride, int32; not NULL.
 *                 [n_axes][n_tokens] has the strides 1 and n_tokens, [n_tokens][n_axes] n_axes and 1.
 *   seq_start     added to every axis of its sequence's tokens, or NULL
 * pos_stride and axis_stride are not negative.  inverse = 1 is the gradient with respect to q and k (positions
 * and frequencies have none).
 */
KVARN_API int kvarn_rotary_axes(const kvarn_rope *rope, const kvarn_rope_axes *axes, const void *q, int32_t n_q,
                                int64_t q_stride, void *q_out, int64_t q_out_stride, const void *k, int32_t n_kv,
                                int64_t k_stride, void *k_out, int64_t k_out_stride, int32_t dtype, int64_t n_tokens,
                                const int32_t *positions, int64_t pos_stride, int64_t axis_stride,
                                const int32_t *seq_start, int64_t tokens_per_seq, int32_t inverse, hipStream_t stream);

/*
 * Read cached tokens back as rows (the cache is not changed):
 *   first     DEVICE, [batch] int32: the first token read of each sequence, or NULL for 0
 *   n_tokens  tokens read of each sequence, first[b] .. first[b] + n_tokens - 1
 *   k_out, v_out  token first[b] + i of (sequence b, kv head h) at element b * seq_stride +
 *             h * head_stride + i * token_stride, 128 channels in out_dtype (fp32 or bf16); either may
 *             be NULL (not read), not both.  16-byte aligned, strides non-negative, a multiple of 16
 *             bytes, and such that rows do not overlap.
 * Sink and residual rows come as stored; body rows are dequantized and their rotation is undone in 32
 * bits, rounded once (for a bf16 out of a rotated cache as a matrix product with exact codes, whose steps a, of
 * values s2, are carried in 22 bits).  Rows of tokens that a sequence does not hold (before 0 or at and behind its
 * length) are left as they were, and so are those of a tile whose block id is not valid (bit 1 of
 * err_word).  n_tokens == 0 is a no-op.
 */
KVARN_API int kvarn_read_tokens(const kvarn_params *p, const kvarn_cache *cache, const int32_t *first,
                                int32_t n_tokens, void *k_out, void *v_out, int32_t out_dtype, int64_t seq_stride,
                                int64_t head_stride, int64_t token_stride, hipStream_t stream);

/* Drafts per sequence of kvarn_tree_attention and kvarn_append_path at most. */
#define KVARN_MAX_DRAFTS 64

/* Workspace bytes that kvarn_tree_attention asks for with these sizes (0 where it needs none, and when an
 * argument is invalid). */
KVARN_API size_t kvarn_tree_workspace_bytes(const kvarn_params *p, const kvarn_cache *cache, int32_t n_q,
                                            int32_t n_draft, int32_t max_len_hint);

/*
 * Attention of drafted tokens (speculative decoding's check of a token tree): draft i of sequence b
 * attends over the sequence's whole cache and over the drafts that its mask names, without any of them
 * entering the cache:
 *   out[b][i][h] = softmax(sm_scale * q[b][i][h] . K^T) V
 *   n_draft   drafts per sequence that the buffers hold, 1 .. KVARN_MAX_DRAFTS
 *   q, out    draft i of sequence b at element (b * n_draft + i) * q_stride (out_stride): n_q heads of 128
 *             channels in q_dtype (out_dtype), fp32 or bf16; q after its rotary position
 *   k_draft, v_draft  the same with kv_stride and n_kv heads in kv_dtype; fp32 is rounded to bf16
 *             first, as appending would
 *   mask      DEVICE, [batch][n_draft] 64-bit words: bit j of draft i's word lets it see draft j.  A
 *             draft sees itself only by its own bit; bits of drafts that are not there count for
 *             nothing.  NULL: a chain (draft i sees drafts 0 .. i).
 *   n_live    DEVICE, [batch] int32: sequence b has drafts 0 .. n_live[b] - 1 (clamped to 0 .. n_draft);
 *             the others' rows of out are left as they were.  NULL: all n_draft.
 *   max_len_hint  an upper bound of every seq_len (sizes the launch plan)
 *   workspace  device buffer of at least kvarn_tree_workspace_bytes(...) bytes, 16-byte aligned; may be
 *             NULL when that size is 0.  Calls that may overlap (other streams, graphs) need one each; no
 *             call relies on its contents.
 * n_q must be a positive multiple of n_kv with n_q / n_kv <= 16.  Pointers are 16-byte aligned (mask 8,
 * n_live 4), strides multiples of 16 bytes, at least the heads' width and at most 2^23 elements.  A draft that sees nothing (an
 * empty cache and an empty mask) gets zeros; what a masked draft holds, infinities and NaN too, does not
 * reach the others.  out must not overlap the inputs.
 * Keys and values of the body enter as their exact codes, queries times the keys' steps and probabilities times
 * the values' in 11 bits for a bf16 out and in 22 bits for an fp32 out, offsets and second scales in 22 bits
 * or more, sums and the softmax's maximum and sum in 32; groups of 128 tokens whose steps lie far apart by their
 * elements, and sink, residual and drafts, with queries (as given where they are bf16) and probabilities in 16 and 24 bits.
 * Probabilities times steps (these relative to the largest of their group) keep their bits down to 2^-28 of the
 * row's largest (fp32 out: 2^-17) and are rounded to 2^-39 of it below.
 * Values whose products come within 2^24 of the end of the fp32 range are not meaningful.
 */
KVARN_API int kvarn_tree_attention(const kvarn_params *p, const kvarn_cache *cache, int32_t n_q, int32_t n_draft,
                                   const void *q, int64_t q_stride, int32_t q_dtype, const void *k_draft,
                                   const void *v_draft, int64_t kv_stride, int32_t kv_dtype, const uint64_t *mask,
                                   const int32_t *n_live, void *out, int64_t out_stride, int32_t out_dtype,
                                   float sm_scale, int32_t max_len_hint, void *workspace, size_t workspace_bytes,
                                   hipStream_t stream);

/*
 * Append the accepted drafts of every sequence: drafts path[b][0], path[b][1], ... path[b][n_path[b] - 1]
 * enter sequence b's cache in this order, as so many kvarn_append_token calls would put them (sink, then
 * residual; a residual that fills is quantized and goes on empty; the same bytes).
 *   k_draft, v_draft, kv_stride, dtype, n_draft  as for kvarn_tree_attention
 *   path      DEVICE, [batch][max_path] int32, or NULL for 0, 1, 2, ...; an index may occur again
 *   max_path  1 .. KVARN_MAX_DRAFTS (at most n_draft without a path)
 *   n_path    DEVICE, [batch] int32, 0 .. max_path; 0 leaves the sequence as it is
 * A sequence is left unchanged, and the others are not, where its count is outside 0 .. max_path or one of
 * its first n_path indices outside 0 .. n_draft - 1 (bit 3 of err_word), or where the group that would fill
 * needs body tile max_blocks (bit 0).  A filled group whose block id is not valid is not written (bit 1),
 * as by kvarn_append_token.
 */
KVARN_API int kvarn_append_path(const kvarn_params *p, const kvarn_cache *cache, int32_t n_draft, const void *k_draft,
                                const void *v_draft, int64_t kv_stride, int32_t dtype, const int32_t *path,
                                int32_t max_path, const int32_t *n_path, hipStream_t stream);

/*
 * Verification of drafted tokens against the model's probabilities: which drafts of each sequence's tree are
 * accepted, and the token that follows them, distributed as if the model had been asked token by token.
 *
 * Draft 0 of a sequence is certain (the token that the step before ended with); the others hang on drafts before
 * them.  From draft 0 on, the children of the node reached are considered in the order of their index: the
 * first that is accepted is the next node; where none is, the walk ends and the next token is drawn.  With p the
 * target row of the node, q its draft row, c a child's token and u its random number:
 *   with draft rows (the children were drawn independently from q):  a = 0 and S = 1 at first;
 *       accepted if u S q(c) < p(c) - a q(c); else a becomes a + S and S the sum of max(p - a q, 0);
 *       the next token's weights are max(p - a q, 0), or p where they are all 0
 *   without (candidates of any origin):  S = 1 at first; accepted if u S < p(c); else p(c) leaves S and the row
 *       (a token that has left is passed over);
 *       the next token's weights are what is left of p
 *   greedy:  accepted if c is the row's largest entry, the lowest index of several; the next token is that entry
 * The next token is the first whose running sum of weights exceeds u times the whole sum.  Children with a token
 * outside 0 .. vocab - 1 are passed over.
 *
 *   n_draft   drafts per sequence that the buffers hold, draft 0 included: 1 .. KVARN_MAX_DRAFTS.  With 1 the
 *             call draws the next token.
 *   vocab     entries of a row, 1 .. KVARN_MAX_VOCAB
 *   tokens    DEVICE, [batch][n_draft] int32 (those of draft 0 are not looked at); NULL for n_draft = 1
 *   parent    DEVICE, [batch][n_draft] int32: the draft that each hangs on.  A draft whose parent is not before it is
 *             never reached; draft 0's is not looked at.  NULL: a chain (draft i hangs on i - 1).
 *   n_live    DEVICE, [batch] int32: sequence b has drafts 0 .. n_live[b] - 1 (clamped to 0 .. n_draft).  One
 *             with none gets n_path 0 and next -1.  NULL: all n_draft.
 *   target    the model's row behind draft i of sequence b at element (b * n_draft + i) * target_stride
 *   draft     the row that the children of draft i were drawn from at (b * n_draft + i) * draft_stride (rows of
 *             drafts without children are not looked at), or NULL: candidates
 *   dtype     of both, fp32 or bf16; aligned to an element, strides in elements, at least vocab
 *   form      KVARN_PROBABILITIES: rows that sum to 1, as a sampler leaves them; or KVARN_LOGITS: p and q are the
 *             softmax of scale[b] * row
 *   scale     DEVICE, [batch] fp32, inverse temperatures (logits only), or NULL for 1; an infinite one (or
 *             beyond 6e36) makes its sequence greedy, one that is not positive leaves its rows without weight
 *   uniform   DEVICE, [batch][n_draft] fp32 in [0, 1): draft i's random number, and at 0 the next token's.
 *             NULL: all sequences are greedy (draft, scale and form are then not looked at)
 *   path      DEVICE, [batch][n_draft] int32: the accepted drafts, 0 first, as kvarn_append_path takes them; -1
 *             behind them
 *   n_path    DEVICE, [batch] int32: their number
 *   next      DEVICE, [batch] int32: the next token; -1 for a row without weight
 *   workspace device buffer of at least kvarn_verify_workspace_bytes(...) bytes of this size or a larger one, 16-byte aligned; may
 *             be NULL when that size is 0.  Calls that may overlap (other streams, graphs) need one each; no call relies on its
 *             contents.
 * NaN entries have no weight, and neither has a logit of -infinity; logits of +infinity share the whole weight.
 * Decisions, weights and sums are those of 64 bits, the weights of logits good to 2^-39: where refused children leave less than
 * that part of a row, rounding decides which of the row's entries follow.  The results are the same for the same
 * arguments.  Negative or infinite probabilities are not meaningful.  batch == 0 is a no-op; more than 2^22 sequences are refused.
 */
#define KVARN_MAX_VOCAB (1 << 20)
typedef enum { KVARN_PROBABILITIES = 0, KVARN_LOGITS = 1 } kvarn_row_form;
/* Workspace bytes for kvarn_verify_drafts, enough for every call of at most so many sequences, drafts and entries: a buffer for
 * the largest serves the smaller ones, of which some need more than the largest itself.  0 where none needs any, and
 * when an argument is invalid. */
KVARN_API size_t kvarn_verify_workspace_bytes(int32_t batch, int32_t n_draft, int32_t vocab);
KVARN_API int kvarn_verify_drafts(int32_t batch, int32_t n_draft, int32_t vocab, const int32_t *tokens,
                                  const int32_t *parent, const int32_t *n_live, const void *target,
                                  int64_t target_stride, const void *draft, int64_t draft_stride, int32_t dtype,
                                  int32_t form, const float *scale, const float *uniform, int32_t *path, int32_t *n_path,
                                  int32_t *next, void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * The pool of a paged cache: which blocks are free, and how many each sequence holds.  Device buffers, allocated and
 * initialised by the caller:
 *   free_ids  [n_phys] int32: a ring of the free blocks' ids.  At first all ids, in any order.
 *   ring      [4] int32: where the ring begins, how many ids it holds (at first 0 and n_phys), and two words of the
 *             library's, 0 between calls
 *   n_blocks  [batch] int32: blocks that each sequence holds, the first entries of its row of the block table (at
 *             first 0)
 */
typedef struct {
    int32_t *free_ids;
    int32_t *ring;
    int32_t *n_blocks;
} kvarn_block_pool;

/*
 * Fit every sequence's blocks to its length: sequence b comes to hold max(lengths[b] + extra - n_sink, 0) / 128
 * blocks, rounded down, what a cache of that many tokens needs (the rest stays in the residual).  Call it before
 * the tokens are appended.
 *   cache     paged; block_table is WRITTEN by this call: entries gained hold the new ids, entries given back -1
 *   lengths   DEVICE, [batch] int32, or NULL for the cache's seq_len.  A sequence of a negative one is left as it
 *             is; 0 (and extra 0) gives back all that it holds.  (Blocks are given back whatever they hold: a
 *             length below the cache's own gives up tokens.)
 *   extra     tokens on top of every length that is not negative, >= 0
 * Blocks are given back first, in the order of the sequences and of their rows, to the end of the ring; then they are
 * taken from its beginning in the same order, so one given back is taken again as late as may be.  Results do not
 * depend on the launch.  A sequence that needs more than max_blocks is left as it is; so are, from the first
 * sequence on whose growth the pool does not cover, all that would grow (bit 0 of err_word).  A count outside
 * 0 .. max_blocks leaves its sequence, and a ring that does not fit the pool all of them, unchanged (bit 3).
 * KVARN_EINVAL for a cache without block table.  Calls on one pool are ordered by the caller.
 */
KVARN_API int kvarn_assign_blocks(const kvarn_params *p, const kvarn_cache *cache, const kvarn_block_pool *pool,
                                  const int32_t *lengths, int32_t extra, hipStream_t stream);

/*
 * Where the tokens of a ragged batch belong:  rows cu_seqlens[b] .. cu_seqlens[b+1] - 1 are sequence b's tokens
 * start[b], start[b] + 1, ...
 *   cu_seqlens  DEVICE, [batch + 1] int32, non-decreasing, cu_seqlens[0] = 0
 *   start       DEVICE, [batch] int32, or NULL for 0.  With a cache's seq_len these are the tokens that come next.
 *   n_tokens    rows that the outputs hold; those at and behind cu_seqlens[batch] are left as they were
 *   seq         DEVICE, [n_tokens] int32, or NULL: the sequence
 *   position    DEVICE, [n_tokens] int32, or NULL: the position, as kvarn_rotary takes it
 *   row         DEVICE, [n_tokens] int64, or NULL: the row of a kv head's tokens that it has once all of them are in
 *               the cache, counted over the regions one after the other:
 *                 b * n_sink + position                       in the sink (position < n_sink)
 *                 batch * n_sink + b * 128 + r                in the residual (its row r)
 *                 batch * (n_sink + 128) + tile * 128 + r     in the body: row r of pool block tile, or of a
 *                                                             dense cache's tile b * max_blocks + block
 *               -1 where there is none: a position outside 0 .. 2^31 - 2, a block at or behind max_blocks, an id outside
 *               the pool (bit 1 of err_word).
 * Not all three are NULL.  Positions outside 32 bits are given as -1.  n_tokens == 0 is a no-op.
 */
KVARN_API int kvarn_token_map(const kvarn_params *p, const kvarn_cache *cache, const int32_t *cu_seqlens,
                              const int32_t *start, int64_t n_tokens, int32_t *seq, int32_t *position, int64_t *row,
                              hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* KVARN_H */
