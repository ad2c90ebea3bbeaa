// Causal attention of a prompt's packed rows over their units' caches: launch planning, the kernel of fp32 rows and the
// join of split launches. bf16 rows go to the tensor cores (prompt_attn_mma.cu).
//
//   row i of m in a unit of n rows:  o = sum_j w_j v_j / sum_j w_j,  w_j = 2^(c q.k_j - max),  j <= n - m + i
//
// One pass over K and V with the running maximum and sum in registers. A tile's 128 rows are (token, head of the group)
// pairs, so the G heads of a kv-head read its K and V once, and few tokens still fill a tile.
#include <algorithm>

#include "evict_policy.cuh"  // sm_count, once_per_device
#include "prompt.cuh"
#include "ptx.cuh"

namespace voxzip {
namespace {

constexpr int kRows = 128, kKeys = 64;

template <int D> struct Smem {
    static constexpr int kQ = D + 4, kK = D + 4, kP = kRows + 4;  // row lengths: 4 words on, the next row's banks
    float q[kRows * kQ];
    float k[kKeys * kK];
    float v[kKeys * D];
    float p[kKeys * kP];
    TileAt at;
    int ok;
};

// Cache row of slot s, or -1 where its page is not in the pool.
__device__ __forceinline__ int64_t cache_row(const PromptAttn &p, int64_t cu, int32_t s) {
    if (!p.cache.pv.table) return cu * p.C + s;
    const int64_t r = paged_row(p.cache.pv, cu, s);
    return r >= 0 && r < p.cache.pool_rows ? r : -1;
}

// 16 bytes to shared memory in the background; zeros where `from` is null.
__device__ __forceinline__ void copy16(float *to, const float *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(to)), "l"(from), "r"(from ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending> __device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
}

// A pair of products and sums: d += a b.
struct Pair {
    float x, y;
};
__device__ __forceinline__ void fma_pair(Pair &d, float a0, float a1, float b0, float b1) {
    asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%0, %1};\n\t"
        "fma.rn.f32x2 c, a, b, c;\n\tmov.b64 {%0, %1}, c;\n\t}"
        : "+f"(d.x), "+f"(d.y)
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

// Tile rows of K or V: keys [key0, key0 + 64), zeros from `most` on.
template <int D>
__device__ __forceinline__ void copy_keys(const PromptAttn &p, const void *data, int64_t cu, int32_t key0, int32_t most,
                                          float *to, int stride) {
    for (int i = threadIdx.x; i < kKeys * (D / 4); i += 256) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        const float *from = nullptr;
        if (key0 + r < most) {
            const int64_t row = cache_row(p, cu, key0 + r);
            if (row < 0) {
                if (d == 0) raise_status(p.status, VOXZIP_DEV_CAPACITY);
            } else if (VOXZIP_IN_RANGE(p.status, row < p.kv_rows)) {
                from = static_cast<const float *>(data) + row * D + d;
            }
        }
        copy16(to + r * stride + d, from);
    }
    copies_end();
}

// fp32 rows. 256 threads as 16 x 16: thread (ty, tx) has the logits of rows ty + 16 i and keys tx + 16 j, and of the
// output the same rows' channels 4 tx (and 64 + 4 tx). Fused multiply-adds bound it, two to an instruction: per four
// channels 64 of these meet twelve 16-byte reads of shared memory. K's and V's next tiles come while the other's is used.
template <int D>
__global__ void __launch_bounds__(256) prompt_rows_kernel(const PromptAttn p) {
    extern __shared__ __align__(16) uint8_t raw[];
    Smem<D> &sm = *reinterpret_cast<Smem<D> *>(raw);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const CtaAt cta = cta_at(p, blockIdx.x);
    const int h = cta.h, l = cta.l, s = cta.split;
    ptx::grid_dependency_wait();
    ptx::launch_dependents();  // the join may take its place on the SMs
    if (tid < 32) {
        TileAt at;
        const bool ok = find_tile(p, cta, at);
        if (tid == 0) {
            sm.ok = ok;
            if (ok) sm.at = at;
        }
    }
    __syncthreads();
    if (!sm.ok) return;
    const TileAt at = sm.at;
    const int64_t cu = ((int64_t)at.b * p.L + p.layer_begin + l) * p.Hkv + h;
    const int32_t n = at.n;
    if (n < 0 || n > p.C) {
        if (tid == 0) raise_status(p.status, VOXZIP_DEV_CAPACITY);
        return;
    }
    const bool split = in_parts(p, cta.x, at);
    if (!split && s > 0) return;
    const int splits = split ? p.splits : 1;
    const int rows = at.rows * p.G;
    const int32_t first = n - at.m + at.before + 1;  // keys that the tile's first token sees (none if < 1)
    const int32_t most = max(0, first + at.rows - 1);
    // this split's keys
    const int32_t tiles = (most + kKeys - 1) / kKeys, per = (tiles + splits - 1) / splits;
    const int32_t j0 = min(tiles, s * per), j1 = min(tiles, j0 + per);

    if (j0 < j1) {
        for (int i = tid; i < kRows * (D / 4); i += 256) {
            const int r = i / (D / 4), d = i % (D / 4) * 4;
            copy16(&sm.q[r * Smem<D>::kQ + d],
                   r < rows ? static_cast<const float *>(p.q.data) + l * p.q.layer_stride +
                                  (int64_t)(at.t0 + r / p.G) * p.q.token_stride + (int64_t)(h * p.G + r % p.G) * D + d
                            : nullptr);
        }
        copy_keys<D>(p, p.cache.k, cu, j0 * kKeys, most, sm.k, Smem<D>::kK);
        copy_keys<D>(p, p.cache.v, cu, j0 * kKeys, most, sm.v, D);
    }
    int32_t lim[8];  // keys that each of this thread's rows sees
    float mx[8], sum[8];
    Pair o[8][D / 32];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lim[i] = first + (ty + 16 * i) / p.G;
        mx[i] = -INFINITY;
        sum[i] = 0.f;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) o[i][d] = Pair{0.f, 0.f};
    }
    for (int32_t j = j0; j < j1; ++j) {
        const int32_t key0 = j * kKeys;
        copies_wait<1>();  // K (and Q); V may be on its way
        __syncthreads();
        Pair acc[8][4] = {};
#pragma unroll 2
        for (int d = 0; d < D; d += 4) {
            float4 q[8], k[4];
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = *reinterpret_cast<const float4 *>(&sm.q[(ty + 16 * i) * Smem<D>::kQ + d]);
#pragma unroll
            for (int c = 0; c < 4; ++c) k[c] = *reinterpret_cast<const float4 *>(&sm.k[(tx + 16 * c) * Smem<D>::kK + d]);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    fma_pair(acc[i][c], q[i].x, q[i].y, k[c].x, k[c].y);
                    fma_pair(acc[i][c], q[i].z, q[i].w, k[c].z, k[c].w);
                }
        }
        const bool masked = key0 + kKeys > first;  // some row does not see all of this tile
        float x[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                x[i][c] = (acc[i][c].x + acc[i][c].y) * p.scale_log2;
                if (masked && key0 + tx + 16 * c >= lim[i]) x[i][c] = -INFINITY;
                top = fmaxf(top, x[i][c]);
            }
#pragma unroll
            for (int w = 1; w < 16; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            const float was = mx[i], now = fmaxf(was, top);
            const float ref = now == -INFINITY ? 0.f : now;  // a row that has seen no key yet
            const float keep = exp2f(was - ref);
            mx[i] = now;
            sum[i] *= keep;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                x[i][c] = exp2f(x[i][c] - ref);
                sum[i] += x[i][c];
            }
#pragma unroll
            for (int d = 0; d < D / 32; ++d) o[i][d].x *= keep, o[i][d].y *= keep;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float4 *to = reinterpret_cast<float4 *>(&sm.p[(tx + 16 * c) * Smem<D>::kP + ty * 8]);
            to[0] = make_float4(x[0][c], x[1][c], x[2][c], x[3][c]);
            to[1] = make_float4(x[4][c], x[5][c], x[6][c], x[7][c]);
        }
        copies_wait<0>();  // V
        __syncthreads();
        if (j + 1 < j1) copy_keys<D>(p, p.cache.k, cu, key0 + kKeys, most, sm.k, Smem<D>::kK);
        auto accumulate = [&](auto guard) {
#pragma unroll 4
            for (int key = 0; key < kKeys; ++key) {
                const float4 *pr = reinterpret_cast<const float4 *>(&sm.p[key * Smem<D>::kP + ty * 8]);
                const float4 pa = pr[0], pb = pr[1];
                const float w[8] = {pa.x, pa.y, pa.z, pa.w, pb.x, pb.y, pb.z, pb.w};
                float4 v[D / 64];
#pragma unroll
                for (int c = 0; c < D / 64; ++c) v[c] = *reinterpret_cast<const float4 *>(&sm.v[key * D + 64 * c + 4 * tx]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool unseen = decltype(guard)::value && key0 + key >= lim[i];
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) {  // 0 times an infinity behind the mask is not 0
                        const float4 u = unseen ? make_float4(0.f, 0.f, 0.f, 0.f) : v[c];
                        fma_pair(o[i][2 * c], w[i], w[i], u.x, u.y);
                        fma_pair(o[i][2 * c + 1], w[i], w[i], u.z, u.w);
                    }
                }
            }
        };
        if (masked)
            accumulate(std::true_type{});
        else
            accumulate(std::false_type{});
        __syncthreads();
        if (j + 1 < j1) copy_keys<D>(p, p.cache.v, cu, key0 + kKeys, most, sm.v, D);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int w = 1; w < 16; w <<= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], w);
        const int r = ty + 16 * i;
        if (r >= rows) continue;
        const int64_t row = ((int64_t)l * p.T + at.t0 + r / p.G) * p.Hq + h * p.G + r % p.G;
        const int32_t part = split ? part_of(p, cta) * (p.part_tokens * p.G) + r : 0;
        const float scale = split ? 1.f : lim[i] <= 0 ? 0.f : 1.f / sum[i];  // a row that sees nothing is 0
        if (split && tx == 0) p.part_ml[part] = make_float2(mx[i], sum[i]);
        if (split && j0 == j1) continue;  // the join does not read it
        float *to = split ? p.part_o + (int64_t)part * D : static_cast<float *>(p.out) + row * D;
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
            *reinterpret_cast<float4 *>(&to[64 * c + 4 * tx]) =
                make_float4(o[i][2 * c].x * scale, o[i][2 * c].y * scale, o[i][2 * c + 1].x * scale, o[i][2 * c + 1].y * scale);
    }
}

// Joins the splits: out = sum_s o_s 2^(m_s - m) / sum_s l_s 2^(m_s - m), m the greatest m_s. A warp per row of the parts.
template <typename T, int D>
__global__ void __launch_bounds__(256) prompt_join_kernel(const PromptAttn p) {
    const int lane = threadIdx.x & 31;
    const int32_t per = p.part_tokens * p.G, units = p.layer_count * p.Hkv, rows = p.part_tiles * units * per;
    const int32_t at_row = blockIdx.x * 8 + (threadIdx.x >> 5), r = at_row % per, u = at_row / per % units;
    const CtaAt cta{at_row / per / units, 0, u % p.Hkv, u / p.Hkv};
    // (What this reads is older than the launch before, which let this one start only after it had waited itself.)
    TileAt at;
    const bool found = at_row < rows && find_tile(p, cta, at);
    ptx::grid_dependency_wait();  // by every warp: this launch ends after the one before it
    // rows of no tile, of a whole one, and of a unit that was skipped
    if (!found || !in_parts(p, cta.x, at) || r >= at.rows * p.G || at.n < 0 || at.n > p.C) return;
    const int32_t seen = at.n - at.m + at.before + r / p.G + 1;  // keys
    const int64_t row = ((int64_t)cta.l * p.T + at.t0 + r / p.G) * p.Hq + cta.h * p.G + r % p.G;
    // a lane's split's statistics; of all of them the greatest maximum
    float m = -INFINITY;
    for (int s = lane; s < p.splits; s += 32) m = fmaxf(m, p.part_ml[s * rows + at_row].x);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
    if (m == -INFINITY) m = 0.f;
    float sum = 0.f, o[D / 32] = {};
    for (int s0 = 0; s0 < p.splits; s0 += 4) {
        float2 ml[4];
        float part[4][D / 32];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            ml[u] = s0 + u < p.splits ? p.part_ml[(s0 + u) * rows + at_row] : make_float2(-INFINITY, 0.f);
            const bool has = !(ml[u].x == -INFINITY && ml[u].y == 0.f);  // a key of this row
            const float *from = p.part_o + (int64_t)((s0 + u) * rows + at_row) * D + lane * (D / 32);
#pragma unroll
            for (int d = 0; d < D / 32; ++d) part[u][d] = has ? from[d] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float w = exp2f(ml[u].x - m);
            sum = fmaf(ml[u].y, w, sum);
#pragma unroll
            for (int d = 0; d < D / 32; ++d) o[d] = fmaf(part[u][d], w, o[d]);
        }
    }
    const float inv = 1.f / sum;
    T *to = static_cast<T *>(p.out) + row * D + lane * (D / 32);
#pragma unroll
    for (int d = 0; d < D / 32; ++d) to[d] = Elem<T>::from_f(seen <= 0 ? 0.f : o[d] * inv);
}

cudaLaunchConfig_t config(dim3 grid, int threads, size_t smem, cudaStream_t stream, cudaLaunchAttribute *attr) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

template <typename T, int D> cudaError_t launch_join(const PromptAttn &p, cudaStream_t stream) {
    const int rows = p.part_tiles * p.layer_count * p.Hkv * p.part_tokens * p.G;
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = config(dim3((rows + 7) / 8), 256, 0, stream, attr);
    return cudaLaunchKernelEx(&cfg, prompt_join_kernel<T, D>, p);
}

template <int D> cudaError_t launch_rows(const PromptAttn &p, cudaStream_t stream) {
    static std::atomic<uint64_t> done{0};
    cudaError_t e = once_per_device(done, [] {
        return cudaFuncSetAttribute(prompt_rows_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<D>));
    });
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = config(dim3(pieces(p)), 256, sizeof(Smem<D>), stream, attr);
    e = cudaLaunchKernelEx(&cfg, prompt_rows_kernel<D>, p);
    return e != cudaSuccess || p.splits == 1 ? e : launch_join<float, D>(p, stream);
}

}  // namespace

PromptPlan prompt_plan(const voxzip_cache_desc &d, int32_t layer_count, int32_t tokens, int32_t max_rows,
                       int32_t max_len) {
    // Rows and keys of a CTA's tiles. Keys are shared out where there are fewer CTAs than the GPU takes at once. fp32
    // (a key tile is 13.6 us of a CTA's work at the 47 TFLOP/s of a long prompt): up to three for each SM, as the last rows
    // of a prompt see twice the keys of the average one (631 tokens, 32/4 heads: 118 us, 164 unsplit); bf16 (1.5 us): one,
    // with two key tiles or more.
    const int G = d.q_heads / d.kv_heads;
    const bool mma = d.dtype == VOXZIP_BF16;
    const int keys = mma ? 128 : kKeys, least = mma ? 2 : 1, per_sm = mma ? 1 : 3;
    PromptPlan plan;
    plan.tile_tokens = mma ? 2 * (128 / G) : kRows / G;
    if (max_len <= 0 || max_len > d.capacity) max_len = d.capacity;
    const int64_t units = (int64_t)d.kv_heads * layer_count;
    const int64_t most = max_rows > 0 && max_rows < tokens ? max_rows : tokens;  // tokens of a sequence, by the hint
    const int64_t hinted = d.batch * ((most + plan.tile_tokens - 1) / plan.tile_tokens);
    const int64_t key_tiles = ((int64_t)max_len + keys - 1) / keys;
    plan.tiles = tile_bound(tokens, d.batch, plan.tile_tokens);
    const int64_t likely = std::min(plan.tiles, hinted);
    plan.splits = (int32_t)std::max<int64_t>(
        1, std::min<int64_t>((int64_t)per_sm * sm_count() / std::max<int64_t>(1, likely * units), key_tiles / least));
    // Parts are kept for the tiles that the hint allows, which are few where keys are shared out: they take up to
    // per_sm * SMs * 256 rows (bf16 20 MB, fp32 30 MB), whatever the packed tensor holds besides and however wrong the hint.
    plan.part_tiles = plan.splits == 1 ? 0 : (int32_t)likely;
    plan.part_tokens = plan.splits == 1 ? 0 : (int32_t)std::min<int64_t>(plan.tile_tokens, most);
    plan.ctas = (plan.tiles + (int64_t)plan.part_tiles * (plan.splits - 1)) * units;
    const size_t rows = (size_t)plan.splits * plan.part_tiles * units * plan.part_tokens * G;
    plan.workspace = (rows * (d.head_dim * sizeof(float) + sizeof(float2)) + 255) / 256 * 256;
    return plan;
}

cudaError_t launch_prompt_attention(const voxzip_cache_desc &d, int32_t layer_begin, int32_t layer_count, RowsView q,
                                    const int32_t *seq_off, int32_t tokens, const CacheRows &cache,
                                    const int32_t *len, float sm_scale, int32_t max_rows, int32_t max_len, void *out,
                                    void *workspace, int32_t *status, cudaStream_t stream) {
    const PromptPlan plan = prompt_plan(d, layer_count, tokens, max_rows, max_len);
    PromptAttn p = {};
    p.q = q;
    p.seq_off = seq_off;
    p.len = len;
    p.cache = cache;
    p.out = out;
    p.status = status;
    p.scale_log2 = (sm_scale > 0.f ? sm_scale : 1.f / sqrtf((float)d.head_dim)) * 1.4426950408889634f;
    p.B = d.batch;
    p.L = d.layers;
    p.Hq = d.q_heads;
    p.Hkv = d.kv_heads;
    p.G = d.q_heads / d.kv_heads;
    p.C = d.capacity;
    p.T = tokens;
    p.layer_begin = layer_begin;
    p.layer_count = layer_count;
    p.splits = plan.splits;
    p.part_tiles = plan.part_tiles;
    p.part_tokens = plan.part_tokens;
    p.kv_rows = cache.pool_rows;
    if (plan.splits > 1) {
        const size_t rows = (size_t)plan.splits * plan.part_tiles * layer_count * d.kv_heads * plan.part_tokens * p.G;
        p.part_o = static_cast<float *>(workspace);
        p.part_ml = reinterpret_cast<float2 *>(p.part_o + rows * d.head_dim);
    }
    p.tile_tokens = plan.tile_tokens;
    p.tiles = (int32_t)plan.tiles;
    if (d.dtype == VOXZIP_BF16) {
        const cudaError_t e = launch_prompt_mma(p, d.head_dim, stream);
        return e != cudaSuccess || p.splits == 1 ? e
               : d.head_dim == 128               ? launch_join<__nv_bfloat16, 128>(p, stream)
                                                 : launch_join<__nv_bfloat16, 64>(p, stream);
    }
    return d.head_dim == 128 ? launch_rows<128>(p, stream) : launch_rows<64>(p, stream);
}

}  // namespace voxzip
