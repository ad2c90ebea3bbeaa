// Packing a cache into 4 bits and reading it back (format: q4.cuh).
#include "q4.cuh"

namespace voxzip {
namespace {

constexpr int kThreads = 256;

struct PackParams {
    Q4View q4;
    const void *k_cache, *v_cache;
    const int32_t *len;
    int32_t *status;
    int32_t B, L, Hkv, C, layer_begin;
};

// Exponent of one channel: the power of two nearest to the ratio of its largest magnitude to the unit's median
// one, so that channels of ordinary size (within a factor sqrt 2 of the median) stay as they are.
__device__ __forceinline__ int channel_exponent(uint32_t amax, uint32_t mid) {
    const uint32_t inf = 0x7f800000u;
    if (amax == 0u || amax >= inf || mid == 0u || mid >= inf) return 0;
    const float r = __fmul_rn(__fdiv_rn(__uint_as_float(amax), __uint_as_float(mid)), 1.41421354f);
    return min(max((int)(__float_as_uint(r) >> 23) - 127, -kQ4MaxExp), kQ4MaxExp);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) q4_pack_kernel(const PackParams p) {
    __shared__ uint32_t amax[D];
    __shared__ float inv_pow[D];
    __shared__ uint32_t mid;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const UnitIdx ui = unit_of(blockIdx.x, p.B, p.L, p.Hkv, p.layer_begin);
    ptx::grid_dependency_wait();
    int32_t n = p.len[ui.cache_unit];
    if (n < 0 || n > p.C) {
        if (tid == 0) raise_status(p.status, VOXZIP_DEV_CAPACITY);
        return;
    }
    const T *k = static_cast<const T *>(p.k_cache) + ui.cache_unit * p.C * D;
    const T *v = static_cast<const T *>(p.v_cache) + ui.cache_unit * p.C * D;
    for (int d = tid; d < D; d += kThreads) amax[d] = 0u;
    if (tid == 0) mid = 0u;
    __syncthreads();
    const bool on = lane < D / 4;
    uint32_t a[4] = {0u, 0u, 0u, 0u};
    if (on)
        for (int r = warp; r < n; r += kThreads / 32) {
            const float4 x = load4(k + (int64_t)r * D + lane * 4);
            a[0] = max(a[0], __float_as_uint(fabsf(x.x)));
            a[1] = max(a[1], __float_as_uint(fabsf(x.y)));
            a[2] = max(a[2], __float_as_uint(fabsf(x.z)));
            a[3] = max(a[3], __float_as_uint(fabsf(x.w)));
        }
    if (on)
        for (int i = 0; i < 4; ++i) atomicMax(&amax[lane * 4 + i], a[i]);
    __syncthreads();
    // the lower median: the channel with rank (D - 1) / 2, ties in channel order
    if (tid < D) {
        int rank = 0;
        for (int d = 0; d < D; ++d) rank += amax[d] < amax[tid] || (amax[d] == amax[tid] && d < tid);
        if (rank == (D - 1) / 2) mid = amax[tid];
    }
    __syncthreads();
    if (tid < D) {
        const int e = channel_exponent(amax[tid], mid);
        inv_pow[tid] = exp2_int(-e);
        p.q4.k_exp[ui.cache_unit * D + tid] = (int8_t)e;
    }
    __syncthreads();
    const float4 f = on ? *reinterpret_cast<const float4 *>(inv_pow + lane * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    for (int r = warp; r < n; r += kThreads / 32) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
        if (on) {
            x = load4(k + (int64_t)r * D + lane * 4);
            y = load4(v + (int64_t)r * D + lane * 4);
            x.x *= f.x, x.y *= f.y, x.z *= f.z, x.w *= f.w;
        }
        const int64_t row = ui.cache_unit * p.C + r;
        Q4Row<D, true>(x).store(p.q4.k_codes + row * (D / 2), p.q4.k_scale + row * (D / kQ4Group));
        Q4Row<D, false>(y).store(p.q4.v_codes + row * (D / 2), p.q4.v_scale + row * (D / kQ4Group));
    }
}

struct UnpackParams {
    Q4View q4;
    const int32_t *len;
    void *k_out, *v_out;
    int32_t *status;
    int32_t B, L, Hkv, C, layer_begin, layer_count, first, rows;
};

template <typename T>
__device__ __forceinline__ void store4(T *p, const float (&x)[4]) {
    T y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = Elem<T>::from_f(x[i]);
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(y);
    else
        *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(y);
}

// Row r of the output is slot first + r (from the unit's end if first < 0); zeros where there is none. A warp
// per row, 4 channels per lane.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) q4_unpack_kernel(const UnpackParams p) {
    constexpr int J = D / kQ4Group;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const UnitIdx ui = unit_of(blockIdx.x, p.B, p.L, p.Hkv, p.layer_begin);
    ptx::grid_dependency_wait();
    const int32_t n = p.len[ui.cache_unit];
    if (n < 0 || n > p.C) {
        if (threadIdx.x == 0 && blockIdx.y == 0) raise_status(p.status, VOXZIP_DEV_CAPACITY);
        return;
    }
    if (lane >= D / 4) return;
    const int j = lane >> 3;
    const int64_t out_unit = ((int64_t)ui.b * p.layer_count + ui.l_local) * p.Hkv + ui.h;
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = exp2_int(p.q4.k_exp[ui.cache_unit * D + lane * 4 + i]);
    for (int r = blockIdx.y * (kThreads / 32) + warp; r < p.rows; r += gridDim.y * (kThreads / 32)) {
        const int64_t slot = (int64_t)r + p.first + (p.first < 0 ? n : 0);
        float k[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
        if (slot >= 0 && slot < n) {
            const int64_t row = ui.cache_unit * p.C + slot;
            const uint32_t kw = reinterpret_cast<const uint32_t *>(p.q4.k_codes + row * (D / 2))[((lane >> 1) & 3) * J + j] >>
                                ((lane & 1) * 8);
            const uint32_t vw = reinterpret_cast<const uint16_t *>(p.q4.v_codes + row * (D / 2))[(lane & 7) * J + j];
            const float ks = __bfloat162float(p.q4.k_scale[row * J + j]), vs = __bfloat162float(p.q4.v_scale[row * J + j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                k[i] = (float)((int)(kw >> (4 * (i >> 1) + 16 * (i & 1)) & 15u) - 8) * ks * f[i];
                v[i] = (float)((int)(vw >> (4 * i) & 15u) - 8) * vs;
            }
        }
        const int64_t to = (out_unit * p.rows + r) * D + lane * 4;
        store4(static_cast<T *>(p.k_out) + to, k);
        store4(static_cast<T *>(p.v_out) + to, v);
    }
}

template <typename F>
cudaError_t by_type(const voxzip_cache_desc &d, F &&f) {
    const bool bf16 = d.dtype == VOXZIP_BF16;
    if (d.head_dim == 128) return bf16 ? f((__nv_bfloat16 *)nullptr, std::integral_constant<int, 128>{})
                                       : f((float *)nullptr, std::integral_constant<int, 128>{});
    return bf16 ? f((__nv_bfloat16 *)nullptr, std::integral_constant<int, 64>{})
                : f((float *)nullptr, std::integral_constant<int, 64>{});
}

}  // namespace

cudaError_t launch_q4_pack(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                           const void *k_cache, const void *v_cache, const int32_t *len, int32_t *status,
                           cudaStream_t stream) {
    const PackParams prm{q4, k_cache, v_cache, len, status, d.batch, d.layers, d.kv_heads, d.capacity, layer_begin};
    const unsigned units = (unsigned)(layer_count * d.batch * d.kv_heads);
    return by_type(d, [&](auto t, auto dim) {
        using T = std::remove_pointer_t<decltype(t)>;
        q4_pack_kernel<T, decltype(dim)::value><<<units, kThreads, 0, stream>>>(prm);
        return cudaGetLastError();
    });
}

cudaError_t launch_q4_unpack(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                             const int32_t *len, int32_t first, int32_t rows, void *k_out, void *v_out, int32_t *status,
                             cudaStream_t stream) {
    const UnpackParams prm{q4, len, k_out, v_out, status, d.batch, d.layers, d.kv_heads, d.capacity,
                           layer_begin, layer_count, first, rows};
    const unsigned units = (unsigned)(layer_count * d.batch * d.kv_heads);
    const unsigned tiles = (unsigned)min(1024, (rows + 63) / 64);
    return by_type(d, [&](auto t, auto dim) {
        using T = std::remove_pointer_t<decltype(t)>;
        q4_unpack_kernel<T, decltype(dim)::value><<<dim3(units, tiles), kThreads, 0, stream>>>(prm);
        return cudaGetLastError();
    });
}

}  // namespace voxzip
