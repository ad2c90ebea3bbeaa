// Decode step on a cache held in 4 bits, for lengths whose logits no cluster of CTAs can hold in shared memory
// (see decode_q4_mma.cu): append, GQA attention and the decayed-score update (format: q4.cuh).
#include "q4.cuh"

namespace voxzip {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

struct DecodeQ4Params {
    Q4View q4;
    const void *q, *k_new, *v_new;
    const int32_t *new_pos;
    float *score;
    int32_t *pos, *len;
    void *out;
    int32_t *status;
    int32_t B, L, Hq, Hkv, G, C, layer_begin, max_rows;
    float gamma, scale_log2;
};

// One CTA per unit, a row per thread, two passes over K: the softmax's maximum and sum, then its weights. A form
// without a limit on the length, in fp32 throughout, for lengths that the tensor-core kernel does not take: those whose
// logits 16 CTAs of 227 KB do not hold (decode_q4_plan.cuh; voxzip.h lists them). Bound by its own arithmetic: 192
// units of 120 000 rows, G = 8, D = 128 take 48.6 ms in bf16 or fp32 (by bytes 0.5; the tensor-core kernel needs 1.9
// for 100 000), 8 units with G = 16 40.9 ms.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) decode_q4_rows_kernel(const DecodeQ4Params p) {
    constexpr int J = D / kQ4Group;
    __shared__ float qs[kMaxGroup][D];  // times 2^e
    __shared__ float pt[kThreads][kMaxGroup + 1];
    __shared__ float red[kThreads / 32][kMaxGroup][2];
    __shared__ float mz[kMaxGroup][2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const UnitIdx ui = unit_of(blockIdx.x, p.B, p.L, p.Hkv, p.layer_begin);
    ptx::grid_dependency_wait();
    const int32_t n_old = p.len[ui.cache_unit];
    if (n_old < 0 || n_old >= p.C) {
        if (tid == 0) raise_status(p.status, VOXZIP_DEV_CAPACITY);
        return;
    }
    const int32_t n = n_old + 1;
    if (n > p.max_rows) {
        if (tid == 0) raise_status(p.status, VOXZIP_DEV_LEN_HINT);
        return;
    }
    const int64_t act = (int64_t)ui.l_local * p.B + ui.b, row_base = ui.cache_unit * p.C;
    const T *qg = static_cast<const T *>(p.q) + (act * p.Hq + (int64_t)ui.h * p.G) * D;
    const int8_t *ke = p.q4.k_exp + ui.cache_unit * D;
    for (int i = tid; i < p.G * D; i += kThreads) qs[i / D][i % D] = Elem<T>::to_f(qg[i]) * exp2_int(ke[i % D]);
    auto in_cache = [&](int r) { return VOXZIP_IN_RANGE(p.status, r >= 0 && r < p.C); };  // of a row of the unit
    if (warp < 2 && in_cache(n_old)) {  // the appended row
        const T *src = static_cast<const T *>(warp == 0 ? p.k_new : p.v_new) + (act * p.Hkv + ui.h) * D;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (lane < D / 4) {
            x = load4(src + lane * 4);
            if (warp == 0) {
                x.x *= exp2_int(-ke[lane * 4]), x.y *= exp2_int(-ke[lane * 4 + 1]);
                x.z *= exp2_int(-ke[lane * 4 + 2]), x.w *= exp2_int(-ke[lane * 4 + 3]);
            }
        }
        if (warp == 0)
            Q4Row<D, true>(x).store(p.q4.k_codes + (row_base + n_old) * (D / 2), p.q4.k_scale + (row_base + n_old) * J);
        else
            Q4Row<D, false>(x).store(p.q4.v_codes + (row_base + n_old) * (D / 2), p.q4.v_scale + (row_base + n_old) * J);
    }
    if (tid == 0 && in_cache(n_old)) p.pos[row_base + n_old] = p.new_pos[ui.b];
    __syncthreads();

    auto logits = [&](int r, float (&l)[kMaxGroup]) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(p.q4.k_codes + (row_base + r) * (D / 2));
        for (int h = 0; h < kMaxGroup; ++h) l[h] = 0.f;
        for (int j = 0; j < J; ++j) {
            const float s = __bfloat162float(p.q4.k_scale[(row_base + r) * J + j]);
            float acc[kMaxGroup];
#pragma unroll
            for (int h = 0; h < kMaxGroup; ++h) acc[h] = 0.f;
            for (int qd = 0; qd < 4; ++qd) {
                const uint32_t word = w[qd * J + j];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float c = (float)((int)(word >> (4 * (e >> 1) + 16 * (e & 1)) & 15u) - 8);
#pragma unroll
                    for (int h = 0; h < kMaxGroup; ++h)
                        if (h < p.G) acc[h] += c * qs[h][32 * j + 8 * qd + e];
                }
            }
#pragma unroll
            for (int h = 0; h < kMaxGroup; ++h) l[h] += s * acc[h];
        }
#pragma unroll
        for (int h = 0; h < kMaxGroup; ++h) l[h] *= p.scale_log2;
    };

    float m[kMaxGroup], z[kMaxGroup];
#pragma unroll
    for (int h = 0; h < kMaxGroup; ++h) m[h] = -INFINITY, z[h] = 0.f;
    for (int r = tid; r < n && in_cache(r); r += kThreads) {
        float l[kMaxGroup];
        logits(r, l);
#pragma unroll
        for (int h = 0; h < kMaxGroup; ++h) {
            const float mm = fmaxf(m[h], l[h]);
            z[h] = (mm == -INFINITY ? 0.f : z[h] * exp2f(m[h] - mm)) + exp2f(l[h] - mm);
            m[h] = mm;
        }
    }
#pragma unroll
    for (int h = 0; h < kMaxGroup; ++h) {
        for (int o = 16; o > 0; o >>= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m[h], o), z2 = __shfl_xor_sync(0xffffffffu, z[h], o);
            const float mm = fmaxf(m[h], m2);
            z[h] = (m[h] == -INFINITY ? 0.f : z[h] * exp2f(m[h] - mm)) + (m2 == -INFINITY ? 0.f : z2 * exp2f(m2 - mm));
            m[h] = mm;
        }
        if (lane == 0) red[warp][h][0] = m[h], red[warp][h][1] = z[h];
    }
    __syncthreads();
    if (tid < kMaxGroup) {
        float mm = -INFINITY, zz = 0.f;
        for (int w = 0; w < kThreads / 32; ++w) mm = fmaxf(mm, red[w][tid][0]);
        for (int w = 0; w < kThreads / 32; ++w)
            zz += red[w][tid][0] == -INFINITY ? 0.f : red[w][tid][1] * exp2f(red[w][tid][0] - mm);
        mz[tid][0] = mm;
        mz[tid][1] = 1.f / zz;
    }
    __syncthreads();

    // Second pass, kThreads rows at a time: the weights, the scores, and o += p v with a channel per thread.
    constexpr int kParts = kThreads / D;
    const int d = tid % D, part = tid / D, j = d / kQ4Group, at = d % kQ4Group;
    float o[kMaxGroup];
#pragma unroll
    for (int h = 0; h < kMaxGroup; ++h) o[h] = 0.f;
    for (int r0 = 0; r0 < n; r0 += kThreads) {
        const int r = r0 + tid;
        if (r < n && in_cache(r)) {
            float l[kMaxGroup], add = 0.f;
            logits(r, l);
#pragma unroll
            for (int h = 0; h < kMaxGroup; ++h)
                if (h < p.G) {
                    pt[tid][h] = exp2f(l[h] - mz[h][0]) * mz[h][1];
                    add += pt[tid][h];
                }
            float *sc = p.score + row_base + r;
            *sc = r == n_old ? add : p.gamma * *sc + add;
        }
        __syncthreads();
        for (int i = part; i < min(kThreads, n - r0) && in_cache(r0 + i); i += kParts) {
            const int64_t row = row_base + r0 + i;
            const uint32_t w = reinterpret_cast<const uint16_t *>(p.q4.v_codes + row * (D / 2))[(at >> 2) * J + j];
            const float v = (float)((int)(w >> (4 * (at & 3)) & 15u) - 8) * __bfloat162float(p.q4.v_scale[row * J + j]);
#pragma unroll
            for (int h = 0; h < kMaxGroup; ++h)
                if (h < p.G) o[h] += pt[i][h] * v;
        }
        __syncthreads();
    }
    float *os = &pt[0][0];
    T *og = static_cast<T *>(p.out) + (act * p.Hq + (int64_t)ui.h * p.G) * D;
    for (int h = 0; h < p.G; ++h) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < kMaxGroup; ++i)
            if (i == h) x = o[i];
        os[tid] = x;
        __syncthreads();
        if (part == 0) {
            for (int k = 1; k < kParts; ++k) x += os[k * D + d];
            og[h * D + d] = Elem<T>::from_f(x);
        }
        __syncthreads();
    }
    if (tid == 0) p.len[ui.cache_unit] = n;
}

}  // namespace

cudaError_t launch_decode_q4_rows(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                             const void *q, const void *k_new, const void *v_new, const int32_t *new_pos, float *score,
                             int32_t *pos, int32_t *len, float gamma, float sm_scale, int32_t max_len, void *out,
                             int32_t *status, cudaStream_t stream) {
    const float scale = sm_scale > 0.f ? sm_scale : 1.0f / sqrtf((float)d.head_dim);
    const int nmax = (max_len > 0 && max_len < d.capacity) ? max_len : d.capacity;
    const DecodeQ4Params prm{q4, q, k_new, v_new, new_pos, score, pos, len, out, status, d.batch, d.layers, d.q_heads,
                             d.kv_heads, d.q_heads / d.kv_heads, d.capacity, layer_begin, nmax, gamma, scale * kLog2e};
    const unsigned units = (unsigned)(layer_count * d.batch * d.kv_heads);
    const bool bf16 = d.dtype == VOXZIP_BF16;
    if (d.head_dim == 128) {
        if (bf16) decode_q4_rows_kernel<__nv_bfloat16, 128><<<units, kThreads, 0, stream>>>(prm);
        else decode_q4_rows_kernel<float, 128><<<units, kThreads, 0, stream>>>(prm);
    } else {
        if (bf16) decode_q4_rows_kernel<__nv_bfloat16, 64><<<units, kThreads, 0, stream>>>(prm);
        else decode_q4_rows_kernel<float, 64><<<units, kThreads, 0, stream>>>(prm);
    }
    return cudaGetLastError();
}

}  // namespace voxzip
