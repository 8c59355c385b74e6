// Host side of the libkvarn C ABI: argument validation (before anything is enqueued), launch
// planning and kernel launches.  No device memory is allocated here.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <mutex>

#include "common.hpp"

using namespace kvarn;

// Split partials of kvarn_decode_attention_noalloc: one array per device, held until the
// process ends.  In host code `scratch` only names the symbol; its device address on the
// current device comes from hipGetSymbolAddress (scratch_ptr below) and is the only form
// passed to kernels.
static __device__ __align__(256) uint8_t scratch[KVARN_NOALLOC_SCRATCH_BYTES];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch[kMaxDevices] = {};

// Device address of the current device's scratch array, looked up once per device.
hipError_t scratch_ptr(void** out) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch[dev]) {
        void* ptr = nullptr;
        e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return e;
        g_scratch[dev] = ptr;
    }
    *out = g_scratch[dev];
    return hipSuccess;
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_params(const kvarn_params* p) {
    if (!p) return KVARN_EINVAL;
    if (p->bits != 2 && p->bits != 4) return KVARN_EUNSUPPORTED;
    if (p->aux_format != KVARN_AUX_F32 && p->aux_format != KVARN_AUX_COMPACT) return KVARN_EUNSUPPORTED;
    if (p->rotate != 0 && p->rotate != 1) return KVARN_EINVAL;
    if (p->varn_iters < 0 || p->varn_iters > 64) return KVARN_EINVAL;
    if (p->n_sink < 0 || p->n_sink > 1024) return KVARN_EINVAL;
    // ranges that keep exp(+-L) and log(v) of the quantizer inside the normal fp32 range
    if (!(p->var_min >= 1e-30f) || !(p->var_max <= 1e30f) || p->var_min > p->var_max) return KVARN_EINVAL;
    if (!(p->log_lo >= -40.f) || !(p->log_hi <= 40.f) || p->log_lo > p->log_hi) return KVARN_EINVAL;
    return KVARN_OK;
}

// Arguments of an append; *flush: whether the call has to launch the flush (always without the
// length hint, else when the token fills the residual).
int append_check(const kvarn_params* p, const kvarn_cache* cache, const void* k_new, const void* v_new, int32_t dtype,
                 int32_t host_len_before, bool* flush);

QParams qparams(const kvarn_params* p) {
    return QParams{p->bits, p->varn_iters, p->var_min, p->var_max, p->log_lo, p->log_hi,
                   p->aux_format == KVARN_AUX_COMPACT ? 1 : 0, p->rotate};
}

int check_cache(const kvarn_params* p, const kvarn_cache* c) {
    if (!c) return KVARN_EINVAL;
    if (c->batch <= 0 || c->n_kv <= 0 || c->max_blocks < 0) return KVARN_EINVAL;
    // kernels index (sequence, kv head, K|V) in 32 bits
    if ((int64_t)c->batch * c->n_kv > kMaxStreams) return KVARN_EINVAL;
    if (!c->k_body || !c->v_body || !c->k_resid || !c->v_resid || !c->seq_len) return KVARN_EINVAL;
    if (p->n_sink > 0 && (!c->k_sink || !c->v_sink)) return KVARN_EINVAL;
    if (!aligned(c->k_body, 16) || !aligned(c->v_body, 16) || !aligned(c->k_resid, 16) || !aligned(c->v_resid, 16))
        return KVARN_EINVAL;
    if (p->n_sink > 0 && (!aligned(c->k_sink, 16) || !aligned(c->v_sink, 16))) return KVARN_EINVAL;
    if (!aligned(c->seq_len, 4)) return KVARN_EINVAL;
    if (c->block_table && (c->n_phys <= 0 || !aligned(c->block_table, 4))) return KVARN_EINVAL;
    return KVARN_OK;
}

int check_dtype(int32_t d) { return (d == KVARN_F32 || d == KVARN_BF16) ? KVARN_OK : KVARN_EINVAL; }

int append_check(const kvarn_params* p, const kvarn_cache* cache, const void* k_new, const void* v_new, int32_t dtype,
                 int32_t host_len_before, bool* flush) {
    int st = check_params(p);
    if (st) return st;
    st = check_cache(p, cache);
    if (st) return st;
    if (check_dtype(dtype)) return KVARN_EINVAL;
    if (!k_new || !v_new) return KVARN_EINVAL;
    const size_t va = dtype == KVARN_BF16 ? 8 : 16;
    if (!aligned(k_new, va) || !aligned(v_new, va)) return KVARN_EINVAL;
    if (host_len_before < -1) return KVARN_EINVAL;
    *flush = true;
    if (host_len_before >= 0) {
        const int len = host_len_before;
        *flush = false;
        if (len >= p->n_sink) {
            const int r = (len - p->n_sink) % kG, nb = (len - p->n_sink) / kG;
            if (r == kG - 1) {
                if (nb >= cache->max_blocks) return KVARN_ECAPACITY;
                *flush = true;
            }
        }
    }
    return KVARN_OK;
}

}  // namespace

extern "C" {

int kvarn_params_init(kvarn_params* p, int32_t bits) {
    if (!p) return KVARN_EINVAL;
    if (bits != 2 && bits != 4) return KVARN_EUNSUPPORTED;
    p->bits = bits;
    p->varn_iters = 8;
    p->n_sink = 0;
    p->var_min = 1e-8f;
    p->var_max = 1e8f;
    p->log_lo = -0.3f;
    p->log_hi = 10.0f;
    p->aux_format = KVARN_AUX_F32;
    p->rotate = 1;
    return KVARN_OK;
}

size_t kvarn_tile_bytes(const kvarn_params* p) {
    return check_params(p) ? 0 : tile_bytes(p->bits, p->aux_format == KVARN_AUX_COMPACT);
}

int kvarn_cache_sizes(const kvarn_params* p, int32_t batch, int32_t n_kv, int32_t max_blocks, size_t sizes[7]) {
    int st = check_params(p);
    if (st) return st;
    if (!sizes || batch <= 0 || n_kv <= 0 || max_blocks < 0) return KVARN_EINVAL;
    if ((int64_t)batch * n_kv > kMaxStreams) return KVARN_EINVAL;
    const size_t streams = (size_t)batch * n_kv;
    sizes[0] = sizes[1] = streams * max_blocks * tile_bytes(p->bits, p->aux_format == KVARN_AUX_COMPACT);
    sizes[2] = sizes[3] = streams * kG * kD * sizeof(uint16_t);
    sizes[4] = sizes[5] = streams * (size_t)p->n_sink * kD * sizeof(uint16_t);
    sizes[6] = (size_t)batch * sizeof(int32_t);
    return KVARN_OK;
}

int kvarn_quantize_block(const kvarn_params* p, int32_t kind, const void* x, int32_t x_dtype, int64_t n_outer,
                         int64_t n_inner, int64_t x_outer_stride, int64_t x_inner_stride, int64_t x_token_stride,
                         void* out, int64_t out_outer_stride, int64_t out_inner_stride, int32_t* best_iter,
                         hipStream_t stream) {
    int st = check_params(p);
    if (st) return st;
    if (kind != KVARN_KEYS && kind != KVARN_VALUES) return KVARN_EINVAL;
    if (check_dtype(x_dtype)) return KVARN_EINVAL;
    if (n_outer < 0 || n_inner < 0 || x_outer_stride < 0 || x_inner_stride < 0 || x_token_stride < 0 ||
        out_outer_stride < 0 || out_inner_stride < 0)
        return KVARN_EINVAL;
    if (n_outer == 0 || n_inner == 0) return KVARN_OK;
    if (!x || !out) return KVARN_EINVAL;
    const int64_t esz = x_dtype == KVARN_BF16 ? 2 : 4;
    // rows are read as 16-byte vectors
    if (!aligned(x, 16) || (x_token_stride * esz) % 16 || (x_outer_stride * esz) % 16 || (x_inner_stride * esz) % 16)
        return KVARN_EINVAL;
    if (x_token_stride < kD) return KVARN_EINVAL;  // tokens must not overlap
    if (!aligned(out, 16)) return KVARN_EINVAL;
    if (best_iter && !aligned(best_iter, 4)) return KVARN_EINVAL;
    hipError_t e = launch_quantize_tiles(qparams(p), kind, x, x_dtype == KVARN_BF16, n_outer, n_inner, x_outer_stride,
                                         x_inner_stride, x_token_stride, out, out_outer_stride, out_inner_stride,
                                         best_iter, stream);
    return e == hipSuccess ? KVARN_OK : KVARN_EHIP;
}

int kvarn_append_token(const kvarn_params* p, const kvarn_cache* cache, const void* k_new, const void* v_new,
                       int32_t dtype, int32_t host_len_before, hipStream_t stream) {
    bool flush = true;
    const int st = append_check(p, cache, k_new, v_new, dtype, host_len_before, &flush);
    if (st) return st;
    hipError_t e = launch_append(*cache, p->n_sink, k_new, v_new, dtype == KVARN_BF16, stream);
    if (e != hipSuccess) return KVARN_EHIP;
    if (flush) {
        e = launch_flush(qparams(p), *cache, p->n_sink, host_len_before >= 0, stream);
        if (e != hipSuccess) return KVARN_EHIP;
    }
    return KVARN_OK;
}

int kvarn_prefill(const kvarn_params* p, const kvarn_cache* cache, const void* k, const void* v, int32_t dtype,
                  const int32_t* cu_seqlens, int32_t max_len, hipStream_t stream) {
    int st = check_params(p);
    if (st) return st;
    st = check_cache(p, cache);
    if (st) return st;
    if (check_dtype(dtype)) return KVARN_EINVAL;
    if (!k || !v || !cu_seqlens || max_len < 0) return KVARN_EINVAL;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(cu_seqlens, 4)) return KVARN_EINVAL;
    const hipError_t e = launch_prefill(qparams(p), *cache, p->n_sink, k, v, dtype == KVARN_BF16, cu_seqlens, max_len,
                                        stream);
    return e == hipSuccess ? KVARN_OK : KVARN_EHIP;
}

size_t kvarn_decode_workspace_bytes(const kvarn_params* p, const kvarn_cache* cache, int32_t n_q,
                                    int32_t max_len_hint) {
    if (check_params(p) || !cache || cache->batch <= 0 || cache->n_kv <= 0 || n_q <= 0 || max_len_hint < 0) return 0;
    const DecodePlan plan = plan_decode(cache->batch, cache->n_kv, n_q, p->bits, max_len_hint, p->n_sink, cache->max_blocks, false);
    return decode_workspace_bytes(cache->batch, n_q, plan);
}

}  // extern "C"

namespace {

// Validation and planning shared by the decode entry points; nothing is enqueued.  ws == nullptr
// with use_scratch: the partials go to the library's per-device scratch array (*workspace is set
// to it).  equal: as for plan_decode.
int decode_check(const kvarn_params* p, const kvarn_cache* cache, int32_t n_q, const void* q, int32_t q_dtype,
                 const void* out, int32_t out_dtype, float sm_scale, int32_t max_len_hint, bool equal, void** workspace,
                 size_t workspace_bytes, bool use_scratch, DecodePlan* plan) {
    int st = check_params(p);
    if (st) return st;
    st = check_cache(p, cache);
    if (st) return st;
    if (n_q <= 0 || n_q % cache->n_kv != 0 || n_q / cache->n_kv > 16) return KVARN_EINVAL;
    if (check_dtype(q_dtype) || check_dtype(out_dtype)) return KVARN_EINVAL;
    if (!q || !out || !std::isfinite(sm_scale) || max_len_hint < 0) return KVARN_EINVAL;
    if (!aligned(q, 4) || !aligned(out, 8)) return KVARN_EINVAL;
    *plan = plan_decode(cache->batch, cache->n_kv, n_q, p->bits, max_len_hint, p->n_sink, cache->max_blocks, equal);
    const size_t need = decode_workspace_bytes(cache->batch, n_q, *plan);
    if (use_scratch) {
        if (need > KVARN_NOALLOC_SCRATCH_BYTES) return KVARN_EWORKSPACE;
        *workspace = nullptr;
        if (need > 0 && scratch_ptr(workspace) != hipSuccess) return KVARN_EHIP;
    } else if (need > 0 && (!*workspace || workspace_bytes < need || !aligned(*workspace, 16))) {
        return KVARN_EWORKSPACE;
    }
    return KVARN_OK;
}

int decode_launch(const kvarn_params* p, const kvarn_cache* cache, int32_t n_q, const void* q, int32_t q_dtype,
                  void* out, int32_t out_dtype, float sm_scale, const DecodePlan& plan, void* workspace,
                  hipStream_t stream, const StepAppend* step = nullptr) {
    const hipError_t e = launch_decode(*cache, p->bits, p->aux_format == KVARN_AUX_COMPACT, p->rotate, p->n_sink, n_q,
                                       q, q_dtype == KVARN_BF16, out, out_dtype == KVARN_BF16, sm_scale, plan,
                                       static_cast<float*>(workspace), stream, step);
    return e == hipSuccess ? KVARN_OK : KVARN_EHIP;
}

int decode_impl(const kvarn_params* p, const kvarn_cache* cache, int32_t n_q, const void* q, int32_t q_dtype,
                void* out, int32_t out_dtype, float sm_scale, int32_t max_len_hint, void* workspace,
                size_t workspace_bytes, bool use_scratch, hipStream_t stream) {
    DecodePlan plan;
    const int st = decode_check(p, cache, n_q, q, q_dtype, out, out_dtype, sm_scale, max_len_hint, false, &workspace,
                                workspace_bytes, use_scratch, &plan);
    if (st) return st;
    return decode_launch(p, cache, n_q, q, q_dtype, out, out_dtype, sm_scale, plan, workspace, stream);
}

}  // namespace

extern "C" {

int kvarn_decode_attention(const kvarn_params* p, const kvarn_cache* cache, int32_t n_q, const void* q,
                           int32_t q_dtype, void* out, int32_t out_dtype, float sm_scale, int32_t max_len_hint,
                           void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return decode_impl(p, cache, n_q, q, q_dtype, out, out_dtype, sm_scale, max_len_hint, workspace, workspace_bytes,
                       false, stream);
}

int kvarn_decode_attention_noalloc(const kvarn_params* p, const kvarn_cache* cache, int32_t n_q, const void* q,
                                   int32_t q_dtype, void* out, int32_t out_dtype, float sm_scale,
                                   int32_t max_len_hint, hipStream_t stream) {
    return decode_impl(p, cache, n_q, q, q_dtype, out, out_dtype, sm_scale, max_len_hint, nullptr, 0, true, stream);
}

int kvarn_append_decode(const kvarn_params* p, const kvarn_cache* cache, const void* k_new, const void* v_new,
                        int32_t kv_dtype, int32_t host_len_before, int32_t n_q, const void* q, int32_t q_dtype,
                        void* out, int32_t out_dtype, float sm_scale, void* workspace, size_t workspace_bytes,
                        hipStream_t stream) {
    if (host_len_before < 0 || host_len_before == INT32_MAX) return KVARN_EINVAL;
    bool flush = true;
    int st = append_check(p, cache, k_new, v_new, kv_dtype, host_len_before, &flush);
    if (st) return st;
    DecodePlan plan;
    st = decode_check(p, cache, n_q, q, q_dtype, out, out_dtype, sm_scale, host_len_before + 1, true, &workspace,
                      workspace_bytes, false, &plan);
    if (st) return st;
    if (host_len_before >= p->n_sink && !flush && aligned(k_new, 16) && aligned(v_new, 16) &&
        (kv_dtype == KVARN_BF16 || !cache->block_table)) {
        const StepAppend step{host_len_before, k_new, v_new, kv_dtype == KVARN_F32};
        return decode_launch(p, cache, n_q, q, q_dtype, out, out_dtype, sm_scale, plan, workspace, stream, &step);
    }
    hipError_t e = launch_append(*cache, p->n_sink, k_new, v_new, kv_dtype == KVARN_BF16, stream);
    if (e == hipSuccess && flush) e = launch_flush(qparams(p), *cache, p->n_sink, true, stream);
    if (e != hipSuccess) return KVARN_EHIP;
    return decode_launch(p, cache, n_q, q, q_dtype, out, out_dtype, sm_scale, plan, workspace, stream);
}

}  // extern "C"

// ---- rotary positions, drafted tokens, reading back ---------------------------------------------

namespace {

// Rows of `heads` heads at `stride` elements, read or written 16 bytes at a time.
bool rows_ok(const void* p, int64_t stride, int64_t heads, size_t esize) {
    return p && aligned(p, 16) && stride >= heads * kD && stride <= (1 << 23) && (stride * (int64_t)esize) % 16 == 0;
}
size_t esize_of(int32_t dtype) { return dtype == KVARN_BF16 ? 2 : 4; }

bool scaling_ok(const kvarn_rope_scaling* s, int32_t rot_dim) {
    if (!s || s->kind == KVARN_ROPE_PLAIN) return true;
    if (s->kind < KVARN_ROPE_PLAIN || s->kind > KVARN_ROPE_RAMP) return false;
    if (!(s->factor > 0) || !std::isfinite(s->factor)) return false;
    if (s->kind == KVARN_ROPE_BASE) return rot_dim > 2;
    if (s->kind == KVARN_ROPE_LINEAR) return true;
    return s->original_length > 0 && std::isfinite(s->original_length) && s->low > 0 && s->high > s->low &&
           std::isfinite(s->high);
}

int rope_check(const kvarn_rope* r) {
    if (!r || r->rot_dim < 2 || r->rot_dim > kD || r->rot_dim % 2) return KVARN_EINVAL;
    if (r->layout != KVARN_ROPE_HALF && r->layout != KVARN_ROPE_INTERLEAVED) return KVARN_EINVAL;
    if (!std::isfinite(r->amplitude) || !r->freq || !aligned(r->freq, 8)) return KVARN_EINVAL;
    return KVARN_OK;
}

int tree_check(const kvarn_params* p, const kvarn_cache* cache, int32_t n_q, int32_t n_draft) {
    int st = check_params(p);
    if (st) return st;
    st = check_cache(p, cache);
    if (st) return st;
    if (n_q <= 0 || n_q % cache->n_kv != 0 || n_q / cache->n_kv > 16) return KVARN_EINVAL;
    return n_draft < 1 || n_draft > KVARN_MAX_DRAFTS ? KVARN_EINVAL : KVARN_OK;
}

}  // namespace

extern "C" {

int kvarn_rope_frequencies(int32_t rot_dim, double base, const kvarn_rope_scaling* s, double* freq, double* amplitude) {
    if (!freq || !amplitude || rot_dim < 2 || rot_dim > kD || rot_dim % 2) return KVARN_EINVAL;
    if (!(base > 1) || !std::isfinite(base) || !scaling_ok(s, rot_dim)) return KVARN_EINVAL;
    const int kind = s ? s->kind : KVARN_ROPE_PLAIN;
    const double two_pi = 6.283185307179586476925286766559;
    if (kind == KVARN_ROPE_BASE) base *= std::pow(s->factor, (double)rot_dim / (rot_dim - 2));
    if (!std::isfinite(base) || base <= 0) return KVARN_EINVAL;
    // (the fastest pair: the first, or the last where the scaled base is below 1)
    const double fastest = std::max(1.0, std::pow(base, -2.0 * (rot_dim / 2 - 1) / rot_dim));
    if (!std::isfinite(fastest) || (kind != KVARN_ROPE_PLAIN && kind != KVARN_ROPE_BASE && !std::isfinite(fastest / s->factor)))
        return KVARN_EINVAL;
    *amplitude = kind == KVARN_ROPE_RAMP && s->factor > 1 ? 0.1 * std::log(s->factor) + 1.0 : 1.0;
    double lo = 0, hi = 0;
    if (kind == KVARN_ROPE_RAMP) {
        auto index = [&](double turns) { return rot_dim * std::log(s->original_length / (two_pi * turns)) / (2 * std::log(base)); };
        lo = std::min(std::max(std::floor(index(s->high)), 0.0), rot_dim - 1.0);
        hi = std::min(std::max(std::ceil(index(s->low)), 0.0), rot_dim - 1.0);
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot_dim), keep = 1.0;
        if (kind == KVARN_ROPE_LINEAR) keep = 0.0;
        if (kind == KVARN_ROPE_BANDS) keep = (s->original_length * f / two_pi - s->low) / (s->high - s->low);
        if (kind == KVARN_ROPE_RAMP) keep = hi > lo ? 1.0 - (i - lo) / (hi - lo) : (i <= lo ? 1.0 : 0.0);
        keep = std::min(std::max(keep, 0.0), 1.0);
        freq[i] = keep == 1.0 ? f : (1.0 - keep) * f / s->factor + keep * f;
    }
    return KVARN_OK;
}

int kvarn_rotary(const kvarn_rope* rope, const void* q, int32_t n_q, int64_t q_stride, void* q_out, int64_t q_out_stride,
                 const void* k, int32_t n_kv, int64_t k_stride, void* k_out, int64_t k_out_stride, int32_t dtype,
                 int64_t n_tokens, const int32_t* positions, const int32_t* seq_start, int64_t tokens_per_seq,
                 int32_t inverse, hipStream_t stream) {
    if (rope_check(rope) || check_dtype(dtype)) return KVARN_EINVAL;
    if (n_q < 0 || n_kv < 0 || (n_q == 0 && n_kv == 0) || n_q > (1 << 20) || n_kv > (1 << 20)) return KVARN_EINVAL;
    if (n_tokens < 0 || tokens_per_seq < 1 || n_tokens % tokens_per_seq || inverse < 0 || inverse > 1) return KVARN_EINVAL;
    if ((positions && !aligned(positions, 4)) || (seq_start && !aligned(seq_start, 4))) return KVARN_EINVAL;
    if (n_tokens == 0) return KVARN_OK;
    const size_t es = esize_of(dtype);
    auto side = [&](const void* x, const void* y, int64_t heads, int64_t sx, int64_t sy) {
        if (heads == 0) return true;
        if (!x || !y || !aligned(x, es) || !aligned(y, es) || sx < 0 || sy < 0) return false;
        if (n_tokens > 1 && (sx < heads * kD || sy < heads * kD)) return false;
        if (x == y && n_tokens > 1 && sx != sy) return false;  // in place: the same rows
        return sx <= INT64_MAX / 32 / n_tokens && sy <= INT64_MAX / 32 / n_tokens;
    };
    if (!side(q, q_out, n_q, q_stride, q_out_stride) || !side(k, k_out, n_kv, k_stride, k_out_stride)) return KVARN_EINVAL;
    const RotaryArgs a{*rope, q, k, q_out, k_out, q_stride, q_out_stride, k_stride, k_out_stride, n_q, n_kv,
                       dtype == KVARN_BF16, inverse, n_tokens, tokens_per_seq, positions, seq_start, false};
    return launch_rotary(a, stream) == hipSuccess ? KVARN_OK : KVARN_EHIP;
}

int kvarn_read_tokens(const kvarn_params* p, const kvarn_cache* cache, const int32_t* first, int32_t n_tokens,
                      void* k_out, void* v_out, int32_t out_dtype, int64_t seq_stride, int64_t head_stride,
                      int64_t token_stride, hipStream_t stream) {
    int st = check_params(p);
    if (st) return st;
    st = check_cache(p, cache);
    if (st) return st;
    if (check_dtype(out_dtype) || n_tokens < 0 || (!k_out && !v_out) || (first && !aligned(first, 4))) return KVARN_EINVAL;
    if (!aligned(k_out, 16) || !aligned(v_out, 16)) return KVARN_EINVAL;
    const int64_t es = (int64_t)esize_of(out_dtype);
    const int64_t most = INT64_MAX / 32;  // every byte offset stays in 64 bits
    for (int64_t s : {seq_stride, head_stride, token_stride})
        if (s < 0 || s > most || (s * es) % 16) return KVARN_EINVAL;
    if (seq_stride > most / cache->batch || head_stride > most / cache->n_kv || token_stride > most / std::max(n_tokens, 1))
        return KVARN_EINVAL;
    // rows that lie on one another
    if ((n_tokens > 1 && token_stride < kD) || (cache->n_kv > 1 && head_stride < kD) || (cache->batch > 1 && seq_stride < kD))
        return KVARN_EINVAL;
    if (n_tokens == 0) return KVARN_OK;
    const ReadArgs a{*cache, p->bits, p->aux_format == KVARN_AUX_COMPACT, p->rotate, p->n_sink, first, n_tokens, k_out, v_out,
                     out_dtype == KVARN_BF16, seq_stride, head_stride, token_stride, k_out && v_out ? 2 : 1,
                     k_out ? KVARN_KEYS : KVARN_VALUES, 0, false};
    return launch_read(a, stream) == hipSuccess ? KVARN_OK : KVARN_EHIP;
}

size_t kvarn_tree_workspace_bytes(const kvarn_params* p, const kvarn_cache* cache, int32_t n_q, int32_t n_draft,
                                  int32_t max_len_hint) {
    if (check_params(p) || !cache || cache->batch <= 0 || cache->n_kv <= 0 || max_len_hint < 0) return 0;
    if (n_q <= 0 || n_q % cache->n_kv != 0 || n_q / cache->n_kv > 16 || n_draft < 1 || n_draft > KVARN_MAX_DRAFTS) return 0;
    return tree_workspace_bytes(*cache, p->n_sink, n_q, n_draft, max_len_hint);
}

int kvarn_tree_attention(const kvarn_params* p, const kvarn_cache* cache, int32_t n_q, int32_t n_draft, const void* q,
                         int64_t q_stride, int32_t q_dtype, const void* k_draft, const void* v_draft, int64_t kv_stride,
                         int32_t kv_dtype, const uint64_t* mask, const int32_t* n_live, void* out, int64_t out_stride,
                         int32_t out_dtype, float sm_scale, int32_t max_len_hint, void* workspace,
                         size_t workspace_bytes, hipStream_t stream) {
    const int st = tree_check(p, cache, n_q, n_draft);
    if (st) return st;
    if (check_dtype(q_dtype) || check_dtype(kv_dtype) || check_dtype(out_dtype)) return KVARN_EINVAL;
    if (!rows_ok(q, q_stride, n_q, esize_of(q_dtype)) || !rows_ok(out, out_stride, n_q, esize_of(out_dtype)) ||
        !rows_ok(k_draft, kv_stride, cache->n_kv, esize_of(kv_dtype)) || !rows_ok(v_draft, kv_stride, cache->n_kv, esize_of(kv_dtype)))
        return KVARN_EINVAL;
    if ((mask && !aligned(mask, 8)) || (n_live && !aligned(n_live, 4))) return KVARN_EINVAL;
    if (!std::isfinite(sm_scale) || max_len_hint < 0) return KVARN_EINVAL;
    const size_t need = tree_workspace_bytes(*cache, p->n_sink, n_q, n_draft, max_len_hint);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return KVARN_EWORKSPACE;
    const TreeArgs a{*cache, p->bits, p->aux_format == KVARN_AUX_COMPACT, p->rotate, p->n_sink, n_q, n_q / cache->n_kv, n_draft,
                     q, q_stride, q_dtype == KVARN_BF16, k_draft, v_draft, kv_stride, kv_dtype == KVARN_BF16, mask, n_live,
                     out, out_stride, out_dtype == KVARN_BF16, sm_scale * kLog2e, max_len_hint, static_cast<float*>(workspace), 0, 0, 0, 0, 0, 0};
    return launch_tree(a, stream) == hipSuccess ? KVARN_OK : KVARN_EHIP;
}

int kvarn_append_path(const kvarn_params* p, const kvarn_cache* cache, int32_t n_draft, const void* k_draft,
                      const void* v_draft, int64_t kv_stride, int32_t dtype, const int32_t* path, int32_t max_path,
                      const int32_t* n_path, hipStream_t stream) {
    int st = check_params(p);
    if (st) return st;
    st = check_cache(p, cache);
    if (st) return st;
    if (n_draft < 1 || n_draft > KVARN_MAX_DRAFTS || check_dtype(dtype)) return KVARN_EINVAL;
    if (max_path < 1 || max_path > KVARN_MAX_DRAFTS || (!path && max_path > n_draft)) return KVARN_EINVAL;
    if (!rows_ok(k_draft, kv_stride, cache->n_kv, esize_of(dtype)) || !rows_ok(v_draft, kv_stride, cache->n_kv, esize_of(dtype)))
        return KVARN_EINVAL;
    if (!n_path || !aligned(n_path, 4) || (path && !aligned(path, 4))) return KVARN_EINVAL;
    const PathArgs a{qparams(p), *cache, p->n_sink, n_draft, max_path, dtype == KVARN_BF16, k_draft, v_draft, kv_stride, path, n_path};
    return launch_append_path(a, stream) == hipSuccess ? KVARN_OK : KVARN_EHIP;
}

}  // extern "C"
