// C ABI of a turn's prompt (declared in include/voxzip.h): argument validation and dispatch.
#include <math.h>

#include <nvtx3/nvToolsExt.h>

#include "prompt.cuh"

voxzip_status voxzip_status_word_address(int32_t **addr);  // api.cu

namespace {

using voxzip::CacheRows;
using voxzip::RotaryTable;
using voxzip::RowsView;

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool desc_ok(const voxzip_cache_desc *d) {
    if (d == nullptr) return false;
    if (d->batch < 1 || d->layers < 1 || d->q_heads < 1 || d->kv_heads < 1 || d->capacity < 1) return false;
    if (d->q_heads % d->kv_heads != 0 || (d->head_dim != 64 && d->head_dim != 128)) return false;
    if (d->dtype != VOXZIP_F32 && d->dtype != VOXZIP_BF16) return false;
    return (int64_t)d->batch * d->layers * d->kv_heads <= INT32_MAX;
}

bool layers_ok(const voxzip_cache_desc &d, int32_t begin, int32_t count) {
    return begin >= 0 && count >= 1 && begin + (int64_t)count <= d.layers;
}

// Rows whose 16-byte vectors the kernels can load: heads D apart, tokens and layers any multiple of 16 bytes. (A
// stride of one token or one layer is not used.)
bool rows_ok(const voxzip_cache_desc &d, const voxzip_rows *r, int32_t heads, int32_t tokens, int32_t layers) {
    if (r->data == nullptr || !aligned(r->data, 16)) return false;
    const int64_t vec = d.dtype == VOXZIP_BF16 ? 8 : 4;
    if (tokens > 1 && (r->token_stride < (int64_t)heads * d.head_dim || r->token_stride % vec != 0)) return false;
    return layers <= 1 || (r->layer_stride >= 1 && r->layer_stride % vec == 0);
}

RowsView view(const voxzip_rows *r) { return r ? RowsView{r->data, r->token_stride, r->layer_stride} : RowsView{}; }

// f / (2 pi) modulo 1 in 64 bits after the point, rounded: f's mantissa times 1 / (2 pi) with 128 bits, in integers (a
// long double is emulated on Arm: 64 of them took 10 us of a call).
uint64_t turns_of(double f) {
    constexpr uint64_t kHi = 0x28be60db9391054aull, kLo = 0x7f09d5f47d4d3770ull;  // 2^128 / (2 pi)
    int e = 0;
    const uint64_t m = (uint64_t)ldexp(frexp(fabs(f), &e), 53);  // |f| = m 2^(e - 53)
    const unsigned __int128 low = (unsigned __int128)m * kLo, high = (unsigned __int128)m * kHi + (uint64_t)(low >> 64);
    const uint64_t limbs[5] = {(uint64_t)low, (uint64_t)high, (uint64_t)(high >> 64), 0, 0};
    const int shift = 117 - e;  // m C 2^128 times 2^(e - 53 + 64 - 128); at least 97 for f up to 1e6
    if (shift > 192) return 0;
    const int at = shift / 64, by = shift % 64;
    uint64_t t = limbs[at] >> by | (by ? limbs[at + 1] << (64 - by) : 0);
    t += limbs[(shift - 1) / 64] >> (shift - 1) % 64 & 1;
    return f < 0 ? 0 - t : t;
}

bool table_of(const voxzip_rotary_desc *r, const voxzip_cache_desc &d, RotaryTable *t) {
    if (r->rotary_dim < 16 || r->rotary_dim > d.head_dim || r->rotary_dim % 16 != 0) return false;
    if (r->axes < 1 || r->axes > 255 || r->freq == nullptr) return false;
    if (r->pairing != VOXZIP_PAIR_HALVES && r->pairing != VOXZIP_PAIR_ADJACENT) return false;
    *t = RotaryTable{};
    t->half = r->rotary_dim / 2;
    t->adjacent = r->pairing == VOXZIP_PAIR_ADJACENT;
    for (int i = 0; i < t->half; ++i) {
        const int axis = r->axis ? r->axis[i] : 0;
        const double f = r->freq[i];
        if (axis >= r->axes || !(fabs(f) <= 1e6)) return false;
        t->axis[i] = (uint8_t)axis;
        t->turns[i] = turns_of(f);
    }
    return true;
}

bool pages_ok(const voxzip_cache_desc &d, const voxzip_paged_cache *pc) {
    if (pc == nullptr || !pc->k_pool || !pc->v_pool || !pc->page_table || !pc->free_pages || !pc->free_count) return false;
    if (!aligned(pc->k_pool, 16) || !aligned(pc->v_pool, 16)) return false;
    if (pc->max_pages < 1 || (int64_t)pc->max_pages * VOXZIP_PAGE_TOKENS != d.capacity) return false;
    return pc->pages >= (int64_t)d.batch * d.layers * d.kv_heads && (int64_t)pc->pages * VOXZIP_PAGE_TOKENS <= INT32_MAX;
}

CacheRows dense_rows(const voxzip_cache_desc &d, const void *k, const void *v) {
    CacheRows c = {};
    c.k = const_cast<void *>(k);
    c.v = const_cast<void *>(v);
    c.pool_rows = (int64_t)d.batch * d.layers * d.kv_heads * d.capacity;
    return c;
}

CacheRows paged_rows(const voxzip_paged_cache &pc) {
    CacheRows c = {};
    c.k = pc.k_pool;
    c.v = pc.v_pool;
    c.pv = voxzip::PageView{pc.page_table, pc.free_pages, pc.free_count, pc.max_pages};
    c.pool_rows = (int64_t)pc.pages * VOXZIP_PAGE_TOKENS;
    return c;
}

// Launches whose grid extents would not fit.
bool counts_fit(const voxzip_cache_desc &d, int32_t layer_count, int32_t tokens) {
    return (int64_t)layer_count * d.batch * d.kv_heads <= INT32_MAX / 8 && (int64_t)layer_count * tokens <= INT32_MAX &&
           (int64_t)tokens + d.batch <= INT32_MAX;
}

voxzip_status from_cuda(cudaError_t e) { return e == cudaSuccess ? VOXZIP_OK : VOXZIP_ECUDA; }

struct Range {
    explicit Range(const char *name) { nvtxRangePushA(name); }
    ~Range() { nvtxRangePop(); }
};

voxzip_status append(const voxzip_cache_desc &d, const CacheRows &cache, const voxzip_rotary_desc *rotary,
                     int32_t layer_begin, int32_t layer_count, int32_t tokens, const voxzip_rows *q,
                     const voxzip_rows *k, const voxzip_rows *v, const int32_t *positions, const int32_t *new_pos,
                     const int32_t *seq_off, int32_t max_rows, float *score, int32_t *pos, int32_t *len, void *q_out,
                     void *workspace, size_t workspace_bytes, voxzip_stream_t stream) {
    if (!layers_ok(d, layer_begin, layer_count) || tokens < 0 || !seq_off || !len) return VOXZIP_EINVAL;
    if (tokens == 0) return VOXZIP_OK;
    if (!k || !v || (q && !q_out) || (pos && !new_pos)) return VOXZIP_EINVAL;
    if (!rows_ok(d, k, d.kv_heads, tokens, layer_count) || !rows_ok(d, v, d.kv_heads, tokens, layer_count))
        return VOXZIP_EINVAL;
    if (q && (!rows_ok(d, q, d.q_heads, tokens, layer_count) || !aligned(q_out, 16))) return VOXZIP_EINVAL;
    const size_t need = voxzip::append_workspace_bytes(d, layer_count, tokens, max_rows);
    if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return VOXZIP_EINVAL;
    RotaryTable table = {};
    if (rotary && (!positions || !table_of(rotary, d, &table))) return VOXZIP_EINVAL;
    if (!counts_fit(d, layer_count, tokens)) return VOXZIP_EUNSUPPORTED;
    int32_t *status = nullptr;
    voxzip_status st = voxzip_status_word_address(&status);
    if (st != VOXZIP_OK) return st;
    return from_cuda(voxzip::launch_append(d, rotary ? &table : nullptr, layer_begin, layer_count, view(q), view(k),
                                           view(v), positions, new_pos, seq_off, tokens, max_rows, cache, score, pos,
                                           len, q_out, workspace, status, reinterpret_cast<cudaStream_t>(stream)));
}

voxzip_status attention(const voxzip_cache_desc &d, const CacheRows &cache, int32_t layer_begin, int32_t layer_count,
                        int32_t tokens, const voxzip_rows *q, const int32_t *seq_off, const int32_t *len,
                        float sm_scale, int32_t max_rows, int32_t max_len, void *out, void *workspace,
                        size_t workspace_bytes, voxzip_stream_t stream) {
    if (!layers_ok(d, layer_begin, layer_count) || tokens < 0 || !seq_off || !len) return VOXZIP_EINVAL;
    if (isnan(sm_scale) || isinf(sm_scale)) return VOXZIP_EINVAL;
    if (tokens == 0) return VOXZIP_OK;
    if (!q || !rows_ok(d, q, d.q_heads, tokens, layer_count) || !out || !aligned(out, 16)) return VOXZIP_EINVAL;
    if (d.q_heads / d.kv_heads > voxzip::kMaxGroup) return VOXZIP_EUNSUPPORTED;
    if (!counts_fit(d, layer_count, tokens)) return VOXZIP_EUNSUPPORTED;
    // a copy of a bf16 tile names its row by 32 bits
    if (d.dtype == VOXZIP_BF16 && cache.pool_rows > INT32_MAX) return VOXZIP_EUNSUPPORTED;
    const voxzip::PromptPlan plan = voxzip::prompt_plan(d, layer_count, tokens, max_rows, max_len);
    if (plan.ctas > INT32_MAX) return VOXZIP_EUNSUPPORTED;
    const size_t need = plan.workspace;
    if (need > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return VOXZIP_EINVAL;
    int32_t *status = nullptr;
    voxzip_status st = voxzip_status_word_address(&status);
    if (st != VOXZIP_OK) return st;
    return from_cuda(voxzip::launch_prompt_attention(d, layer_begin, layer_count, view(q), seq_off, tokens, cache, len,
                                                     sm_scale, max_rows, max_len, out, workspace, status,
                                                     reinterpret_cast<cudaStream_t>(stream)));
}

}  // namespace

extern "C" {

voxzip_status voxzip_rotary(const voxzip_cache_desc *desc, const voxzip_rotary_desc *rotary, int32_t layer_count,
                            int32_t tokens, const voxzip_rows *q, const voxzip_rows *k, const int32_t *positions,
                            void *q_out, void *k_out, voxzip_stream_t stream) {
    Range range("voxzip_rotary");
    if (!desc_ok(desc) || !rotary || layer_count < 1 || tokens < 0 || (!q && !k)) return VOXZIP_EINVAL;
    RotaryTable table;
    if (!table_of(rotary, *desc, &table)) return VOXZIP_EINVAL;
    if (tokens == 0) return VOXZIP_OK;
    if (!positions) return VOXZIP_EINVAL;
    if (q && (!rows_ok(*desc, q, desc->q_heads, tokens, layer_count) || !q_out || !aligned(q_out, 16)))
        return VOXZIP_EINVAL;
    if (k && (!rows_ok(*desc, k, desc->kv_heads, tokens, layer_count) || !k_out || !aligned(k_out, 16)))
        return VOXZIP_EINVAL;
    if ((int64_t)layer_count * tokens > INT32_MAX) return VOXZIP_EUNSUPPORTED;
    return from_cuda(voxzip::launch_rotary(*desc, table, layer_count, tokens, view(q), view(k), positions, q_out, k_out,
                                           reinterpret_cast<cudaStream_t>(stream)));
}

size_t voxzip_append_workspace_size(const voxzip_cache_desc *desc, int32_t layer_count, int32_t tokens,
                                    int32_t max_rows) {
    Range range("voxzip_append_workspace_size");
    if (!desc_ok(desc) || layer_count < 1 || layer_count > desc->layers || tokens < 1) return 0;
    return voxzip::append_workspace_bytes(*desc, layer_count, tokens, max_rows);
}

voxzip_status voxzip_append(const voxzip_cache_desc *desc, const voxzip_rotary_desc *rotary, int32_t layer_begin,
                            int32_t layer_count, int32_t tokens, const voxzip_rows *q, const voxzip_rows *k,
                            const voxzip_rows *v, const int32_t *positions, const int32_t *new_pos,
                            const int32_t *seq_off, int32_t max_rows, void *k_cache, void *v_cache, float *score,
                            int32_t *pos, int32_t *len, void *q_out, void *workspace, size_t workspace_bytes,
                            voxzip_stream_t stream) {
    Range range("voxzip_append");
    if (!desc_ok(desc) || !k_cache || !v_cache || !aligned(k_cache, 16) || !aligned(v_cache, 16)) return VOXZIP_EINVAL;
    return append(*desc, dense_rows(*desc, k_cache, v_cache), rotary, layer_begin, layer_count, tokens, q, k, v, positions,
                  new_pos, seq_off, max_rows, score, pos, len, q_out, workspace, workspace_bytes, stream);
}

voxzip_status voxzip_append_paged(const voxzip_cache_desc *desc, const voxzip_paged_cache *paged,
                                  const voxzip_rotary_desc *rotary, int32_t layer_begin, int32_t layer_count,
                                  int32_t tokens, const voxzip_rows *q, const voxzip_rows *k, const voxzip_rows *v,
                                  const int32_t *positions, const int32_t *new_pos, const int32_t *seq_off,
                                  int32_t max_rows, float *score, int32_t *pos, int32_t *len, void *q_out,
                                  void *workspace, size_t workspace_bytes, voxzip_stream_t stream) {
    Range range("voxzip_append_paged");
    if (!desc_ok(desc) || !pages_ok(*desc, paged)) return VOXZIP_EINVAL;
    return append(*desc, paged_rows(*paged), rotary, layer_begin, layer_count, tokens, q, k, v, positions, new_pos,
                  seq_off, max_rows, score, pos, len, q_out, workspace, workspace_bytes, stream);
}

size_t voxzip_prompt_attention_workspace_size(const voxzip_cache_desc *desc, int32_t layer_count, int32_t tokens,
                                              int32_t max_rows, int32_t max_len) {
    Range range("voxzip_prompt_attention_workspace_size");
    if (!desc_ok(desc) || layer_count < 1 || layer_count > desc->layers || tokens < 1) return 0;
    if (desc->q_heads / desc->kv_heads > voxzip::kMaxGroup) return 0;
    return voxzip::prompt_plan(*desc, layer_count, tokens, max_rows, max_len).workspace;
}

voxzip_status voxzip_prompt_attention(const voxzip_cache_desc *desc, int32_t layer_begin, int32_t layer_count,
                                      int32_t tokens, const voxzip_rows *q, const int32_t *seq_off,
                                      const void *k_cache, const void *v_cache, const int32_t *len, float sm_scale,
                                      int32_t max_rows, int32_t max_len, void *out, void *workspace,
                                      size_t workspace_bytes, voxzip_stream_t stream) {
    Range range("voxzip_prompt_attention");
    if (!desc_ok(desc) || !k_cache || !v_cache || !aligned(k_cache, 16) || !aligned(v_cache, 16)) return VOXZIP_EINVAL;
    return attention(*desc, dense_rows(*desc, k_cache, v_cache), layer_begin, layer_count, tokens, q, seq_off, len,
                     sm_scale, max_rows, max_len, out, workspace, workspace_bytes, stream);
}

voxzip_status voxzip_prompt_attention_paged(const voxzip_cache_desc *desc, const voxzip_paged_cache *paged,
                                            int32_t layer_begin, int32_t layer_count, int32_t tokens,
                                            const voxzip_rows *q, const int32_t *seq_off, const int32_t *len,
                                            float sm_scale, int32_t max_rows, int32_t max_len, void *out,
                                            void *workspace, size_t workspace_bytes, voxzip_stream_t stream) {
    Range range("voxzip_prompt_attention_paged");
    if (!desc_ok(desc) || !pages_ok(*desc, paged)) return VOXZIP_EINVAL;
    return attention(*desc, paged_rows(*paged), layer_begin, layer_count, tokens, q, seq_off, len, sm_scale, max_rows,
                     max_len, out, workspace, workspace_bytes, stream);
}

}  // extern "C"
