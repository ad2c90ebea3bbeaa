// A turn's prompt: packed rows of several sequences, rotated, appended to a cache and attending over it. Shared by
// rotary.cu, prompt_attn.cu, prompt_attn_mma.cu and the C ABI (api_prompt.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.cuh"
#include "paged.cuh"
#include "voxzip.h"

namespace voxzip {

constexpr int kMaxPairs = 64;  // rotated pairs of a head (D <= 128)

// A rotation as the kernels take it, by value. A frequency is a fraction of a turn per position in 64-bit fixed
// point, so position * frequency modulo a turn is within |position| 2^-65 of one, 2^-34 for any 32-bit position.
struct RotaryTable {
    uint64_t turns[kMaxPairs];
    uint8_t axis[kMaxPairs];
    int32_t half;      // pairs
    int32_t adjacent;  // pairs are channels (2 i, 2 i + 1), not (i, i + half)
};

// Rows [layer][token][head][D] of a packed tensor; strides in elements.
struct RowsView {
    const void *data;
    int64_t token_stride, layer_stride;
};

struct CacheRows {  // where a unit's rows lie: dense slabs (pv.table null) or page pools
    void *k, *v;
    PageView pv;
    int64_t pool_rows;  // rows of k and v: every row index is below it
};

cudaError_t launch_rotary(const voxzip_cache_desc &d, const RotaryTable &table, int32_t layer_count, int32_t tokens,
                          RowsView q, RowsView k, const int32_t *positions, void *q_out, void *k_out,
                          cudaStream_t stream);

size_t append_workspace_bytes(const voxzip_cache_desc &d, int32_t layer_count, int32_t tokens, int32_t max_rows);
cudaError_t launch_append(const voxzip_cache_desc &d, const RotaryTable *table, int32_t layer_begin,
                          int32_t layer_count, RowsView q, RowsView k, RowsView v, const int32_t *positions,
                          const int32_t *new_pos, const int32_t *seq_off, int32_t tokens, int32_t max_rows,
                          const CacheRows &cache, float *score, int32_t *pos, int32_t *len, void *q_out,
                          void *workspace, int32_t *status, cudaStream_t stream);

// The attention of packed rows over their units. Rows of a tile are (token, head of the group) pairs, head fastest:
// the G query heads of a kv-head share its K and V tiles, whatever G is.
struct PromptAttn {
    RowsView q;
    const int32_t *seq_off;
    const int32_t *len;
    CacheRows cache;
    void *out;
    float *part_o;   // [splits][part_tiles][layer_count][Hkv][part_tokens * G][D], of splits > 1
    float2 *part_ml; // the same rows: running maximum (in units of log2) and sum
    int32_t *status;
    float scale_log2;  // logit scale times log2(e)
    int32_t B, L, Hq, Hkv, G, C, T;
    int32_t layer_begin, layer_count;
    int32_t tile_tokens;  // tokens per CTA
    int32_t tiles;        // bound on the tiles of all sequences
    int32_t splits;       // pieces of the keys of the first part_tiles tiles, if they have up to part_tokens tokens
    int32_t part_tiles, part_tokens;
    int64_t kv_rows;  // rows of the K and V tensors (checked builds)
};

// The i-th piece of a launch's work: its tile, split, kv-head and layer. Of one sequence the tiles that see the most keys
// come first, of all heads, so that the last ones to start are short; sequences come in their order.
struct CtaAt {
    int32_t x, split, h, l;
};
__device__ __forceinline__ CtaAt cta_at(const PromptAttn &p, int64_t piece) {
    const uint32_t units = p.Hkv * p.layer_count, i = (uint32_t)piece;
    const uint32_t u = i % units, rest = i / units, split = p.part_tiles * p.splits;
    const bool whole = rest >= split;  // a tile behind those that the workspace has parts for
    return CtaAt{(int32_t)(whole ? rest - split + p.part_tiles : rest / p.splits), (int32_t)(whole ? 0 : rest % p.splits),
                 (int32_t)(u % p.Hkv), (int32_t)(u / p.Hkv)};
}

// A CTA's place: tile `x` of those of all sequences, in packed order, the last tile of a sequence first (it sees the
// most keys, and CTAs start in order).
struct TileAt {
    int32_t b, t0, rows, before;  // sequence, first packed token, tokens of this tile, its first token's index in the sequence
    int32_t m, n;                 // the sequence's tokens, the unit's length
};

// One warp, all lanes. False where x lies behind the last tile or the offsets are malformed up to it. The lengths of the
// units that it may turn out to be are loaded beside the offsets, not after them.
__device__ __forceinline__ bool find_tile(const PromptAttn &p, const CtaAt &cta, TileAt &at) {
    const int lane = threadIdx.x & 31;
    const int32_t B = p.B, T = p.T, per = p.tile_tokens, x = cta.x;
    int32_t first = 0;
    for (int32_t base = 0; base < B; base += 32) {
        const int32_t b = base + lane;
        const int32_t o0 = b < B ? p.seq_off[b] : 0, o1 = b < B ? p.seq_off[b + 1] : 0;
        const int32_t len = b < B ? p.len[((int64_t)b * p.L + p.layer_begin + cta.l) * p.Hkv + cta.h] : 0;
        const bool bad = b < B && (o0 < 0 || o1 < o0 || o1 > T);
        if (__ballot_sync(0xffffffffu, bad)) {
            if (lane == 0) raise_status(p.status, VOXZIP_DEV_BAD_SPANS);
            return false;
        }
        const int32_t n = (o1 - o0) / per + ((o1 - o0) % per != 0);
        int32_t sum = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += up;
        }
        const unsigned past = __ballot_sync(0xffffffffu, x < first + sum);
        if (past) {
            const int src = __ffs(past) - 1;
            const int32_t idx = __shfl_sync(0xffffffffu, n - 1 - (x - (first + sum - n)), src);
            const int32_t s0 = __shfl_sync(0xffffffffu, o0, src), s1 = __shfl_sync(0xffffffffu, o1, src);
            at.b = base + src;
            at.n = __shfl_sync(0xffffffffu, len, src);
            at.m = s1 - s0;
            at.before = idx * per;
            at.t0 = s0 + at.before;
            at.rows = min(per, at.m - at.before);
            return true;
        }
        first += __shfl_sync(0xffffffffu, sum, 31);
    }
    return false;
}

// Whether a tile's keys are shared out among CTAs. The workspace has parts for the tiles of a right hint of the rows; what a
// wrong one did not foresee is done whole.
__device__ __forceinline__ bool in_parts(const PromptAttn &p, int32_t x, const TileAt &at) {
    return p.splits > 1 && x < p.part_tiles && at.rows <= p.part_tokens;
}
// Which of the [splits][part_tiles][layer_count][Hkv] a piece's part is; its rows are (token, head) pairs.
__device__ __forceinline__ int32_t part_of(const PromptAttn &p, const CtaAt &cta) {
    return ((cta.split * p.part_tiles + cta.x) * p.layer_count + cta.l) * p.Hkv + cta.h;
}

// Tiles of a launch at most: every sequence has ceil(m / per) of them.
inline int64_t tile_bound(int64_t tokens, int64_t B, int per) {
    return (tokens + (B < tokens ? B : tokens) * (per - 1)) / per;
}

// Pieces of a launch, one to a CTA.
inline int32_t pieces(const PromptAttn &p) {
    return (p.tiles + p.part_tiles * (p.splits - 1)) * p.Hkv * p.layer_count;
}

cudaError_t launch_prompt_mma(const PromptAttn &p, int D, cudaStream_t stream);

struct PromptPlan {
    int32_t splits, tile_tokens, part_tiles, part_tokens;
    int64_t tiles, ctas;
    size_t workspace;
};
PromptPlan prompt_plan(const voxzip_cache_desc &d, int32_t layer_count, int32_t tokens, int32_t max_rows,
                       int32_t max_len);
cudaError_t launch_prompt_attention(const voxzip_cache_desc &d, int32_t layer_begin, int32_t layer_count, RowsView q,
                                    const int32_t *seq_off, int32_t tokens, const CacheRows &cache,
                                    const int32_t *len, float sm_scale, int32_t max_rows, int32_t max_len, void *out,
                                    void *workspace, int32_t *status, cudaStream_t stream);

}  // namespace voxzip
