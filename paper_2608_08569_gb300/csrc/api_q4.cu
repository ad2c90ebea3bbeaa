// C ABI of the cache held in 4 bits (declared in include/voxzip.h): argument validation and dispatch.
#include <math.h>

#include <nvtx3/nvToolsExt.h>

#include "q4.cuh"

voxzip_status voxzip_status_word_address(int32_t **addr);  // api.cu

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A descriptor and a cache whose rows the kernels can address: dense scales of D / 32 per row stay 16-byte
// aligned per unit when the capacity is a multiple of 4.
bool cache_ok(const voxzip_cache_desc *d, const voxzip_q4_cache *c) {
    if (d == nullptr || c == nullptr) return false;
    if (d->batch < 1 || d->layers < 1 || d->q_heads < 1 || d->kv_heads < 1 || d->capacity < 1) return false;
    if (d->q_heads % d->kv_heads != 0 || (d->head_dim != 64 && d->head_dim != 128)) return false;
    if (d->dtype != VOXZIP_F32 && d->dtype != VOXZIP_BF16) return false;
    if (d->capacity % VOXZIP_Q4_CAPACITY_MULTIPLE != 0) return false;
    if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->k_exp) return false;
    return aligned16(c->k_codes) && aligned16(c->v_codes) && aligned16(c->k_scale) && aligned16(c->v_scale) &&
           aligned16(c->k_exp);
}

bool layers_ok(const voxzip_cache_desc &d, int32_t begin, int32_t count) {
    return begin >= 0 && count >= 1 && begin + (int64_t)count <= d.layers;
}

// Units of a call fit a grid's x extent.
bool units_ok(const voxzip_cache_desc &d, int32_t layer_count) {
    return (int64_t)layer_count * d.batch * d.kv_heads <= INT32_MAX &&
           (int64_t)layer_count * d.batch <= INT32_MAX;
}

voxzip_status from_cuda(cudaError_t e) { return e == cudaSuccess ? VOXZIP_OK : VOXZIP_ECUDA; }

struct Range {
    explicit Range(const char *name) { nvtxRangePushA(name); }
    ~Range() { nvtxRangePop(); }
};

}  // namespace

extern "C" {

voxzip_status voxzip_q4_pack(const voxzip_cache_desc *desc, const voxzip_q4_cache *q4, int32_t layer_begin,
                             int32_t layer_count, const void *k_cache, const void *v_cache, const int32_t *len,
                             voxzip_stream_t stream) {
    Range range("voxzip_q4_pack");
    if (!cache_ok(desc, q4) || !layers_ok(*desc, layer_begin, layer_count)) return VOXZIP_EINVAL;
    if (!k_cache || !v_cache || !len || !aligned16(k_cache) || !aligned16(v_cache)) return VOXZIP_EINVAL;
    if (!units_ok(*desc, layer_count)) return VOXZIP_EUNSUPPORTED;
    int32_t *status = nullptr;
    const voxzip_status st = voxzip_status_word_address(&status);
    if (st != VOXZIP_OK) return st;
    return from_cuda(voxzip::launch_q4_pack(*desc, voxzip::q4_view(*q4), layer_begin, layer_count, k_cache, v_cache, len,
                                            status, reinterpret_cast<cudaStream_t>(stream)));
}

voxzip_status voxzip_q4_unpack(const voxzip_cache_desc *desc, const voxzip_q4_cache *q4, int32_t layer_begin,
                               int32_t layer_count, const int32_t *len, int32_t first, int32_t rows, void *k_out,
                               void *v_out, voxzip_stream_t stream) {
    Range range("voxzip_q4_unpack");
    if (!cache_ok(desc, q4) || !layers_ok(*desc, layer_begin, layer_count)) return VOXZIP_EINVAL;
    if (!len || !k_out || !v_out || !aligned16(k_out) || !aligned16(v_out) || rows < 1) return VOXZIP_EINVAL;
    if (!units_ok(*desc, layer_count)) return VOXZIP_EUNSUPPORTED;
    int32_t *status = nullptr;
    const voxzip_status st = voxzip_status_word_address(&status);
    if (st != VOXZIP_OK) return st;
    return from_cuda(voxzip::launch_q4_unpack(*desc, voxzip::q4_view(*q4), layer_begin, layer_count, len, first, rows,
                                              k_out, v_out, status, reinterpret_cast<cudaStream_t>(stream)));
}

voxzip_status voxzip_decode_step_q4(const voxzip_cache_desc *desc, const voxzip_q4_cache *q4, int32_t layer_begin,
                                    int32_t layer_count, const void *q, const void *k_new, const void *v_new,
                                    const int32_t *new_pos, float *score, int32_t *pos, int32_t *len, float gamma,
                                    float sm_scale, int32_t max_len, void *out, voxzip_stream_t stream) {
    Range range("voxzip_decode_step_q4");
    if (!cache_ok(desc, q4) || !layers_ok(*desc, layer_begin, layer_count)) return VOXZIP_EINVAL;
    if (!q || !k_new || !v_new || !new_pos || !score || !pos || !len || !out) return VOXZIP_EINVAL;
    if (!(gamma > 0.f && gamma <= 1.f) || isnan(sm_scale) || isinf(sm_scale)) return VOXZIP_EINVAL;
    if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(out) || !aligned16(score))
        return VOXZIP_EINVAL;
    if (desc->q_heads / desc->kv_heads > voxzip::kMaxGroup) return VOXZIP_EUNSUPPORTED;
    if (!units_ok(*desc, layer_count)) return VOXZIP_EUNSUPPORTED;
    int32_t *status = nullptr;
    const voxzip_status st = voxzip_status_word_address(&status);
    if (st != VOXZIP_OK) return st;
    return from_cuda(voxzip::launch_decode_q4(*desc, voxzip::q4_view(*q4), layer_begin, layer_count, q, k_new, v_new,
                                              new_pos, score, pos, len, gamma, sm_scale, max_len, out, status,
                                              reinterpret_cast<cudaStream_t>(stream)));
}

voxzip_status voxzip_evict_q4(const voxzip_cache_desc *desc, const voxzip_q4_cache *q4, int32_t layer_begin,
                              int32_t layer_count, float *score, int32_t *pos, int32_t *len, const int32_t *budget,
                              const voxzip_evict_policy *policy, voxzip_stream_t stream) {
    Range range("voxzip_evict_q4");
    if (!cache_ok(desc, q4) || policy == nullptr || !layers_ok(*desc, layer_begin, layer_count)) return VOXZIP_EINVAL;
    if (!score || !pos || !len || !budget) return VOXZIP_EINVAL;
    const voxzip_evict_policy &p = *policy;
    if (p.sink < 0 || !(p.recent_frac >= 0.f && p.recent_frac <= 1.f)) return VOXZIP_EINVAL;
    if ((p.history != 0 && p.history != 1) || p.budget_stride_b < 0 || p.budget_stride_l < 0) return VOXZIP_EINVAL;
    if (p.compaction != VOXZIP_COMPACT_ORDERED && p.compaction != VOXZIP_COMPACT_FILL) return VOXZIP_EINVAL;
    if (!units_ok(*desc, layer_count)) return VOXZIP_EUNSUPPORTED;
    int32_t *status = nullptr;
    const voxzip_status st = voxzip_status_word_address(&status);
    if (st != VOXZIP_OK) return st;
    return from_cuda(voxzip::launch_evict_q4(*desc, voxzip::q4_view(*q4), layer_begin, layer_count, score, pos, len,
                                             budget, p, status, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
