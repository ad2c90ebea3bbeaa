// Packing a cache into 4 bits and reading it back (format: q4.cuh).
//
// Packing: the largest magnitude of every channel of K is needed before the first code, so a cluster of CTAs takes a
// unit and reads its K twice, with as many CTAs as it takes for the units at work to stay in L2 in between (DRAM reads
// are those of one pass and a tenth). A lane takes 16 channels, half a group: with fewer, more lanes repeat the scale's
// arithmetic. bf16 rows stay in pairs for their maxima and exponents; codes are rounded by an addition and gathered by
// byte permutations. V's half-words are exchanged between the lanes of neighbouring groups, so that words are stored.
// Reading back: a lane takes 8 channels, so that a warp's stores are whole lines (16 per lane: 255 instead of 218 us).
//
// Both are bound by instructions and latency rather than HBM. 768 units of 2 301 rows, D = 128, bf16: packing 283 us
// (1.16 GB, 0.60 of the measured copy rate, 14 instructions per channel of K or V at 2.3 per cycle), reading back 215 us
// (0.80); fp32 470 (0.65) and 415 us (0.73). Asking rows into L2 ahead gained nothing for bf16 and cost fp32 a fifth.
#include <cooperative_groups.h>

#include <type_traits>

#include "q4.cuh"

namespace cg = cooperative_groups;

namespace voxzip {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr double kL2Share = 72.0 * 1048576.0;  // bytes of K that the units at work may take of L2

struct PackParams {
    Q4View q4;
    const void *k_cache, *v_cache;
    const int32_t *len;
    int32_t *status;
    int32_t B, L, Hkv, C, layer_begin, S;
};

// Exponent of one channel: the power of two nearest to the ratio of its largest magnitude to the unit's median
// one, so that channels of ordinary size (within a factor sqrt 2 of the median) stay as they are.
__device__ __forceinline__ int channel_exponent(uint32_t amax, uint32_t mid) {
    const uint32_t inf = 0x7f800000u;
    if (amax == 0u || amax >= inf || mid == 0u || mid >= inf) return 0;
    const float r = __fmul_rn(__fdiv_rn(__uint_as_float(amax), __uint_as_float(mid)), 1.41421354f);
    return min(max((int)(__float_as_uint(r) >> 23) - 127, -kQ4MaxExp), kQ4MaxExp);
}

// Sixteen channels as they lie in memory: half a group, the eight at p and the eight at p + 16 (two lanes then load
// whole 32-byte sectors).
template <typename T>
struct Half {
    static constexpr int kVecs = (int)sizeof(T);
    uint4 v[kVecs];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = reinterpret_cast<const uint4 *>(p)[i + (i >= kVecs / 2 ? kVecs / 2 : 0)];
    }
    __device__ __forceinline__ const uint32_t *words() const { return reinterpret_cast<const uint32_t *>(v); }
    __device__ __forceinline__ uint32_t *words() { return reinterpret_cast<uint32_t *>(v); }
    __device__ __forceinline__ float at(int i) const {
        if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? words()[i / 2] & 0xffff0000u : words()[i / 2] << 16);
        else return __uint_as_float(words()[i]);
    }
};

__device__ __forceinline__ __nv_bfloat162 as_pair(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); }
__device__ __forceinline__ uint32_t as_word(__nv_bfloat162 x) { return *reinterpret_cast<const uint32_t *>(&x); }

// The magnitude key (q4.cuh) of the group that this lane and the next share, of values as in memory.
__device__ __forceinline__ uint32_t group_key(const Half<__nv_bfloat16> &x) {
    const uint32_t *w = x.words();
    __nv_bfloat162 hi = as_pair(w[0]), lo = hi;
#pragma unroll
    for (int i = 1; i < 8; ++i) hi = __hmax2_nan(hi, as_pair(w[i])), lo = __hmin2_nan(lo, as_pair(w[i]));
    // 16-bit keys of both halves: the magnitude's 15 bits, then "positive"
    auto keys = [](uint32_t u) { return ((u << 1 & 0xfffefffeu) | (u >> 15 & 0x00010001u)) ^ 0x00010001u; };
    const uint32_t k2 = __vmaxu2(keys(as_word(hi)), keys(as_word(lo)));
    uint32_t k = max(k2 & 0xffffu, k2 >> 16);
    k = max(k, __shfl_xor_sync(0xffffffffu, k, 1));
    return (k & 0xfffeu) << 16 | (k & 1u);
}
__device__ __forceinline__ uint32_t group_key(const Half<float> &x) {
    uint32_t k = 0u;
#pragma unroll
    for (int i = 0; i < 16; ++i) k = max(k, magnitude_key(x.at(i)));
    return max(k, __shfl_xor_sync(0xffffffffu, k, 1));
}

// a + b and a b on two fp32 values in one instruction each.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\t"
        "mov.b64 {%0, %1}, z;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\t"
        "mov.b64 {%0, %1}, z;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// Order of the channels in a word's bytes: byte k holds channel low(k) in its lower nibble, high(k) in its upper one.
template <bool kIsK>
struct WordOrder {
    static __host__ __device__ constexpr int low(int k) { return kIsK ? (k & 1) * 4 + (k >> 1) : 2 * k; }
    static __host__ __device__ constexpr int high(int k) { return low(k) + (kIsK ? 2 : 1); }
};

// Codes of eight values under the scale's reciprocal, as a word. A value is rounded by adding 1.5 2^23 + 8, whose unit
// is 1 and even, so that ties go to even codes; 8 (1 + 2^-8), the most a value over its scale comes to, leaves only the
// upper end to clamp. The code + 8 is then the sum's lowest byte.
template <bool kIsK, typename X>
__device__ __forceinline__ uint32_t eight_codes(X &&x, float inv) {
    using O = WordOrder<kIsK>;
    const float2 inv2 = make_float2(inv, inv), round = make_float2(12582920.f, 12582920.f);
    uint32_t n[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const float2 t = mul2(make_float2(x(i), x(i + 1)), inv2);
        const float2 u = add2(make_float2(fminf(t.x, 7.f), fminf(t.y, 7.f)), round);
        n[i] = __float_as_uint(u.x), n[i + 1] = __float_as_uint(u.y);
    }
    const uint32_t lo = __byte_perm(__byte_perm(n[O::low(0)], n[O::low(1)], 0x40), __byte_perm(n[O::low(2)], n[O::low(3)], 0x40), 0x5410);
    const uint32_t hi = __byte_perm(__byte_perm(n[O::high(0)], n[O::high(1)], 0x40), __byte_perm(n[O::high(2)], n[O::high(3)], 0x40), 0x5410);
    return inv == 0.f ? 0x88888888u : lo + 16u * hi;  // scale 0 or NaN: no codes
}

template <typename T, int D, bool kCluster>
__global__ void __launch_bounds__(kThreads, 4) q4_pack_kernel(const PackParams p) {
    constexpr int J = D / kQ4Group, kLanes = D / 16, kRows = 32 / kLanes * kWarps;  // rows the CTA takes at a time
    constexpr int kAhead = 2;  // of which so many are on their way
    __shared__ __align__(16) uint32_t amax[D], amax_unit[D];
    __shared__ float inv_pow[D];
    __shared__ uint32_t mid;
    const int tid = threadIdx.x;
    const int S = kCluster ? p.S : 1, rank = kCluster ? (int)cg::this_cluster().block_rank() : 0;
    const UnitIdx ui = unit_of((int)(blockIdx.x / (unsigned)S), p.B, p.L, p.Hkv, p.layer_begin);
    for (int d = tid; d < D; d += kThreads) amax[d] = 0u;
    if (tid == 0) mid = 0u;
    ptx::grid_dependency_wait();
    const int32_t n = p.len[ui.cache_unit];
    if (n < 0 || n > p.C) {  // the same decision in every CTA of the cluster
        if (tid == 0 && rank == 0) raise_status(p.status, VOXZIP_DEV_CAPACITY);
        return;
    }
    __syncthreads();
    // This CTA's rows are [first, last).
    const int share = ((n + S - 1) / S + kRows - 1) / kRows * kRows, first = min(n, rank * share), last = min(n, first + share);
    const int j = tid % kLanes >> 1, half = tid & 1, r0 = first + tid / kLanes;
    const T *k = static_cast<const T *>(p.k_cache) + ui.cache_unit * p.C * D + 32 * j + 8 * half;
    const T *v = static_cast<const T *>(p.v_cache) + ui.cache_unit * p.C * D + 32 * j + 8 * half;
    auto in_cache = [&](int r) { return VOXZIP_IN_RANGE(p.status, r >= 0 && r < p.C); };  // of a row of the unit
    auto channel = [&](int i) { return 32 * j + 8 * half + i + (i & 8); };  // of the lane's i-th value
    // Largest magnitudes: of bf16 as pairs of 16-bit integers (the order of magnitudes is that of their bits).
    constexpr int kTop = 4 * Half<T>::kVecs;
    uint32_t top[kTop];
#pragma unroll
    for (int i = 0; i < kTop; ++i) top[i] = 0u;
    for (int r = r0; r < last; r += kAhead * kRows) {
        Half<T> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            x[u] = Half<T>{};
            if (r + u * kRows < last && in_cache(r + u * kRows)) x[u].load(k + (int64_t)(r + u * kRows) * D);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int i = 0; i < kTop; ++i) {
                const uint32_t w = x[u].words()[i];
                top[i] = sizeof(T) == 2 ? __vmaxu2(top[i], w & 0x7fff7fffu) : max(top[i], w & 0x7fffffffu);
            }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t t = sizeof(T) == 2 ? (i & 1 ? top[i / 2] & 0xffff0000u : top[i / 2] << 16) : top[i % kTop];
        atomicMax(&amax[channel(i)], t);
    }
    if constexpr (kCluster) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        for (int d = tid; d < D; d += kThreads) {
            uint32_t t = 0u;
            for (int q = 0; q < S; ++q) t = max(t, *cluster.map_shared_rank(&amax[d], q));
            amax_unit[d] = t;
        }
        ptx::cluster_arrive();  // done reading the others: they may leave
    } else {
        __syncthreads();
        for (int d = tid; d < D; d += kThreads) amax_unit[d] = amax[d];
    }
    __syncthreads();
    // the lower median: the channel with rank (D - 1) / 2, ties in channel order
    if (tid < D) {
        int before = 0;
        const uint32_t own = amax_unit[tid];
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
            const uint4 x = *reinterpret_cast<const uint4 *>(amax_unit + d);
            before += (x.x < own + (d < tid)) + (x.y < own + (d + 1 < tid)) + (x.z < own + (d + 2 < tid)) + (x.w < own + (d + 3 < tid));
        }
        if (before == (D - 1) / 2) mid = own;
    }
    __syncthreads();
    if (tid < D) {
        const int e = channel_exponent(amax_unit[tid], mid);
        inv_pow[tid] = exp2_int(-e);
        if (rank == 0) p.q4.k_exp[ui.cache_unit * D + tid] = (int8_t)e;
    }
    __syncthreads();
    auto f = [&](int i) { return inv_pow[channel(i)]; };
    uint32_t f2[8];  // as bf16 pairs
#pragma unroll
    for (int i = 0; i < 8; ++i) f2[i] = ptx::pack_bf16(f(2 * i), f(2 * i + 1));

    const int rounds = (last - first + kRows - 1) / kRows;  // the same for the warp's lanes: shuffles
    constexpr int kBoth = kAhead / 2;
    for (int i0 = 0; i0 < rounds; i0 += kBoth) {
        Half<T> a[kBoth], b[kBoth];
#pragma unroll
        for (int u = 0; u < kBoth; ++u) {
            const int r = r0 + (i0 + u) * kRows;
            a[u] = b[u] = Half<T>{};
            if (r < last && in_cache(r)) {
                a[u].load(k + (int64_t)r * D);
                b[u].load(v + (int64_t)r * D);
            }
        }
#pragma unroll
        for (int u = 0; u < kBoth; ++u) {
            const int r = r0 + (i0 + u) * kRows;
            const int64_t row = ui.cache_unit * p.C + r;
            uint32_t kw[2], vw[2];
            float ks, vs;
            {
                // x = k 2^-e: exact, except for bf16 products below the smallest normal number
                Half<T> x = a[u];
#pragma unroll
                for (int i = 0; i < kTop; ++i) {
                    if constexpr (sizeof(T) == 2) x.words()[i] = as_word(__hmul2(as_pair(x.words()[i]), as_pair(f2[i])));
                    else x.words()[i] = __float_as_uint(x.at(i) * f(i));
                }
                ks = q4_scale(group_key(x));
                const float inv = q4_inverse(ks);
                if (sizeof(T) == 2 && fabsf(ks) < 0x1p-118f)  // where those would be codes
#pragma unroll
                    for (int h = 0; h < 2; ++h) kw[h] = eight_codes<true>([&](int i) { return a[u].at(8 * h + i) * f(8 * h + i); }, inv);
                else
#pragma unroll
                    for (int h = 0; h < 2; ++h) kw[h] = eight_codes<true>([&](int i) { return x.at(8 * h + i); }, inv);
            }
            {
                vs = q4_scale(group_key(b[u]));
                const float inv = q4_inverse(vs);
#pragma unroll
                for (int h = 0; h < 2; ++h)  // half-words g = 2 half + 4 h, + 1
                    vw[h] = eight_codes<false>([&](int i) { return b[u].at(8 * h + i); }, inv);
            }
            // Words of V pair the groups 2 i and 2 i + 1: the even one's lane takes the first two g, the odd one's the others.
            const uint32_t other = __shfl_xor_sync(0xffffffffu, j & 1 ? vw[0] : vw[1], 2);
            const uint32_t even = j & 1 ? other : vw[0], odd = j & 1 ? vw[1] : other;
            if (r < last && in_cache(r)) {
                uint32_t *kc = reinterpret_cast<uint32_t *>(p.q4.k_codes + row * (D / 2)) + half * J + j;
                uint32_t *vc = reinterpret_cast<uint32_t *>(p.q4.v_codes + row * (D / 2)) + (2 * half + 4 * (j & 1)) * (J / 2) + (j >> 1);
                kc[0] = kw[0];
                kc[2 * J] = kw[1];
                vc[0] = __byte_perm(even, odd, 0x5410);
                vc[J / 2] = __byte_perm(even, odd, 0x7632);
                if (half == 0) {
                    p.q4.k_scale[row * J + j] = __float2bfloat16_rn(ks);
                    p.q4.v_scale[row * J + j] = __float2bfloat16_rn(vs);
                }
            }
        }
    }
    if constexpr (kCluster) ptx::cluster_wait();  // the others have read this CTA's magnitudes
}

struct UnpackParams {
    Q4View q4;
    const int32_t *len;
    void *k_out, *v_out;
    int32_t *status;
    int32_t B, L, Hkv, C, layer_begin, layer_count, first, rows;
};

template <typename T>
__device__ __forceinline__ void store8(T *p, const float2 (&x)[4]) {
    if constexpr (sizeof(T) == 2) {
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(ptx::pack_bf16(x[0].x, x[0].y), ptx::pack_bf16(x[1].x, x[1].y),
                                                        ptx::pack_bf16(x[2].x, x[2].y), ptx::pack_bf16(x[3].x, x[3].y)));
    } else {
        __stcs(reinterpret_cast<float4 *>(p), make_float4(x[0].x, x[0].y, x[1].x, x[1].y));
        __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(x[2].x, x[2].y, x[3].x, x[3].y));
    }
}

// The eight channels of a word: code times scale, for K (an eighth of) it and then 2^(e + 3): neither factor nor the
// product between is infinite or inexact, whatever the scale (one times 2^e may be, where the code is 0). A code's byte
// becomes 2^23 + c + 8 by one byte permutation.
template <bool kIsK>
__device__ __forceinline__ void eight_values(uint32_t w, float2 scale, const float2 (&pow)[4], float2 (&x)[4]) {
    using O = WordOrder<kIsK>;
    const uint32_t lo = w & 0x0f0f0f0fu, hi = w >> 4 & 0x0f0f0f0fu;
    float y[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        y[O::low(k)] = __uint_as_float(__byte_perm(lo, 0x4b000000u, 0x7540 | k));
        y[O::high(k)] = __uint_as_float(__byte_perm(hi, 0x4b000000u, 0x7540 | k));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = mul2(add2(make_float2(y[2 * i], y[2 * i + 1]), make_float2(-8388616.f, -8388616.f)), scale);
        if constexpr (kIsK) x[i] = mul2(x[i], pow[i]);
    }
}

// Row r of the output is slot first + r (from the unit's end if first < 0); zeros where there is none. A lane takes 8
// channels, so that a warp's stores are whole lines: a word of K, and of V the half-words of its group from two words
// that it shares with the next group's lane. A CTA takes kAhead times kRows rows of a unit.
template <int D>
struct Unpack {
    static constexpr int kLanes = D / 8, kRows = kThreads / kLanes, kAhead = 2;
};
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 6) q4_unpack_kernel(const UnpackParams p) {
    using U = Unpack<D>;
    constexpr int J = D / kQ4Group, kRows = U::kRows, kAhead = U::kAhead;
    const int c8 = threadIdx.x % U::kLanes, j = c8 >> 2, q = c8 & 3;
    const UnitIdx ui = unit_of(blockIdx.x, p.B, p.L, p.Hkv, p.layer_begin);
    ptx::grid_dependency_wait();
    const int32_t n = p.len[ui.cache_unit];
    const int2 exps = *reinterpret_cast<const int2 *>(p.q4.k_exp + ui.cache_unit * D + c8 * 8);
    if (n < 0 || n > p.C) {
        if (threadIdx.x == 0 && blockIdx.y == 0) raise_status(p.status, VOXZIP_DEV_CAPACITY);
        return;
    }
    float2 f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = (i < 2 ? exps.x : exps.y) >> (16 * (i & 1));
        f[i] = make_float2(exp2_int((int)(int8_t)e + 3), exp2_int((int)(int8_t)(e >> 8) + 3));
    }
    const int64_t out_unit = ((int64_t)ui.b * p.layer_count + ui.l_local) * p.Hkv + ui.h;
    const int64_t shift = (int64_t)p.first + (p.first < 0 ? n : 0);
    T *k_out = static_cast<T *>(p.k_out) + out_unit * p.rows * D + c8 * 8;
    T *v_out = static_cast<T *>(p.v_out) + out_unit * p.rows * D + c8 * 8;
    const uint32_t *kc = reinterpret_cast<const uint32_t *>(p.q4.k_codes + ui.cache_unit * p.C * (D / 2)) + q * J + j;
    const uint32_t *vc = reinterpret_cast<const uint32_t *>(p.q4.v_codes + ui.cache_unit * p.C * (D / 2)) + (2 * q + (j & 1)) * (J / 2) + (j >> 1);
    const __nv_bfloat16 *ks0 = p.q4.k_scale + ui.cache_unit * p.C * J + j, *vs0 = p.q4.v_scale + ui.cache_unit * p.C * J + j;
    // every lane of a warp goes round as often: shuffles
    for (int base = blockIdx.y * (kAhead * kRows); base < p.rows; base += gridDim.y * (kAhead * kRows)) {
        const int r0 = base + (int)threadIdx.x / U::kLanes;
        uint32_t kw[kAhead], vw[kAhead];
        float ks[kAhead], vs[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t slot = r0 + u * kRows + shift;
            kw[u] = vw[u] = 0u;
            ks[u] = vs[u] = 0.f;
            if (r0 + u * kRows < p.rows && slot >= 0 && slot < n && VOXZIP_IN_RANGE(p.status, slot < p.C)) {
                kw[u] = kc[slot * (D / 8)];
                vw[u] = vc[slot * (D / 8)];
                ks[u] = __bfloat162float(ks0[slot * J]);
                vs[u] = __bfloat162float(vs0[slot * J]);
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            // even groups' lanes hold half-words g = 2 q of both, odd ones' g = 2 q + 1
            const uint32_t other = __shfl_xor_sync(0xffffffffu, vw[u], 4);
            const uint32_t v = j & 1 ? __byte_perm(other, vw[u], 0x7632) : __byte_perm(vw[u], other, 0x5410);
            const int r = r0 + u * kRows;
            if (r < p.rows && VOXZIP_IN_RANGE(p.status, r >= 0)) {
                float2 x[4];
                eight_values<true>(kw[u], make_float2(ks[u] * 0.125f, ks[u] * 0.125f), f, x);
                store8(k_out + (int64_t)r * D, x);
                eight_values<false>(v, make_float2(vs[u], vs[u]), f, x);
                store8(v_out + (int64_t)r * D, x);
            }
        }
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

// A launch that starts while the kernel before it drains (its kernels wait before their first read), in clusters of S.
template <typename P>
cudaError_t launch(void (*kern)(P), dim3 grid, int S, const P &prm, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)S;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t err = cudaLaunchKernelEx(&cfg, kern, prm);
    if (err == cudaErrorNotSupported || err == cudaErrorInvalidValue) {  // no programmatic launch here
        cudaGetLastError();
        cfg.numAttrs = 1;
        err = cudaLaunchKernelEx(&cfg, kern, prm);
    }
    return err;
}

}  // namespace

cudaError_t launch_q4_pack(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                           const void *k_cache, const void *v_cache, const int32_t *len, int32_t *status,
                           cudaStream_t stream) {
    const int64_t units = (int64_t)layer_count * d.batch * d.kv_heads;
    // CTAs per unit: enough to fill the GPU (four per SM), and for the units at work to fit L2 between their two reads.
    const double unit_bytes = (double)d.capacity * d.head_dim * (d.dtype == VOXZIP_BF16 ? 2 : 4);
    const int ctas = 4 * sm_count();
    int S = 1;
    while (S < 8 && (units * S < ctas || ctas / S * unit_bytes > kL2Share) && S * 32 < d.capacity) S *= 2;
    if (units * S > INT32_MAX) S = 1;
    const PackParams prm{q4, k_cache, v_cache, len, status, d.batch, d.layers, d.kv_heads, d.capacity, layer_begin, S};
    return by_type(d, [&](auto t, auto dim) {
        using T = std::remove_pointer_t<decltype(t)>;
        constexpr int D = decltype(dim)::value;
        return launch(S > 1 ? q4_pack_kernel<T, D, true> : q4_pack_kernel<T, D, false>, dim3((unsigned)(units * S)), S, prm, stream);
    });
}

cudaError_t launch_q4_unpack(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                             const int32_t *len, int32_t first, int32_t rows, void *k_out, void *v_out, int32_t *status,
                             cudaStream_t stream) {
    const UnpackParams prm{q4, len, k_out, v_out, status, d.batch, d.layers, d.kv_heads, d.capacity,
                           layer_begin, layer_count, first, rows};
    const unsigned units = (unsigned)(layer_count * d.batch * d.kv_heads);
    return by_type(d, [&](auto t, auto dim) {
        using T = std::remove_pointer_t<decltype(t)>;
        using U = Unpack<decltype(dim)::value>;
        const unsigned tiles = (unsigned)min(65535, (rows + U::kAhead * U::kRows - 1) / (U::kAhead * U::kRows));
        return launch(q4_unpack_kernel<T, decltype(dim)::value>, dim3(units, tiles), 1, prm, stream);
    });
}

}  // namespace voxzip
