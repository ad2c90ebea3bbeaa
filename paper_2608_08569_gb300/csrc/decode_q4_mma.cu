// Decode step on a cache held in 4 bits (format: q4.cuh): append (Eq. 1), GQA attention (Eq. 2) and the
// decayed-score update (Eq. 6), reading each packed K and V row once.
//
//   l_h[t] = scale sum_j s[t][j] sum_{d in j} (q_hd 2^e_d) c[t][d]        (groups j of 32 channels)
//   out_h[d] = sum_t (p_h[t] s[t][j(d)]) c[t][d] / sum_t p_h[t]
// The codes are small integers, so they go to the tensor cores (mma.sync m16n8k16, bf16) as they are: exact, and
// without a multiplication by their scale. For K the scale multiplies the fp32 sum of a group (two k-steps); for V
// it multiplies the weight before that is rounded to bf16. A nibble becomes an operand by one AND: as a bf16 bit
// pattern, the integer v in 0..255 is v 2^-133 (a subnormal or in the first binade above, one straight line), so a
// code in bits 0-3 is c 2^-133 and one in bits 4-7 is 16 c 2^-133; q and p carry 2^84 (q of the odd pairs 2^80), and
// what is left, 2^-49, goes into factors that are applied anyway. The stored code is c + 8: for K the accumulators
// start from -8 sum q; for V eight is subtracted from the operands (an output may be far smaller than its weights'
// sum, so that a correction afterwards would cancel: with one, outputs of 1e-6 were off by as much).
// fp32 activations are split into three bf16 parts (24 bits), of which each makes a product of its own, so that
// only fp32 sums round.
//
// Grid: S CTAs per (layer, sequence, kv-head) unit, a thread-block cluster where S > 1; CTA r owns a run of 32-token
// tiles, and its warp w every fourth of them. Every warp streams its own K tiles and then its V tiles through a ring
// of its own, filled by bulk copies that its lane 0 issues, so nothing in the streaming waits for another warp: the
// weights are taken relative to the warp's own maximum. The logits, then the weights, stay in shared memory until
// the unit's maximum and normaliser are known (a sum over warps, then over the cluster through distributed shared
// memory), when each warp rewrites the scores of its own tokens.
#include <cooperative_groups.h>

#include <type_traits>

#include "q4.cuh"

namespace cg = cooperative_groups;

namespace voxzip {
namespace {

#ifndef VOXZIP_Q4_WP
#define VOXZIP_Q4_WP 2
#endif
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 32;   // tokens per stage
constexpr int kStages = 4;  // of a warp's ring
constexpr int kMaxCluster = 16;
constexpr size_t kMaxSmem = 227 * 1024;
constexpr uint32_t kWaitLimit = 1u << 24;
constexpr float kCarry = 0x1p84f, kUncarry = 0x1p49f;

struct MmaQ4Params {
    Q4View q4;
    const void *q, *k_new, *v_new;
    const int32_t *new_pos;
    float *score;
    int32_t *pos, *len;
    void *out;
    int32_t *status;
    int32_t B, L, Hq, Hkv, G, C, layer_begin, S, chunk_cap, max_rows;
    float gamma, scale_log2;  // scale_log2: logits in units of log 2, times kUncarry
};

template <int D, int NT, int kParts>
struct Layout {
    static constexpr int J = D / kQ4Group;
    static constexpr int kGP = 8 * NT;
    static constexpr int kCodeBytes = kTile * D / 2;
    static constexpr int kStageBytes = kCodeBytes + kTile * J * 2;
    static constexpr int kWarpRing = kStages * kStageBytes;
    static constexpr int kOStride = D + 4;  // a warp's outputs take its drained ring: [kGP][kOStride] fp32
    static_assert(kGP * kOStride * 4 <= kWarpRing, "outputs fit the ring");
    static constexpr int kBarOff = kWarps * kWarpRing;  // full[kWarps][kStages], the scores' barrier
    static constexpr int kStatOff = kBarOff + (kWarps * kStages + 2) * 8;
    // m_w, z_w, f_w [kWarps][kGP]; mz [kGP] and mz_all [kMaxCluster][kGP] pairs
    static constexpr int kStatFloats = (3 * kWarps + 2 + 2 * kMaxCluster) * kGP;
    static constexpr int kQOff = kStatOff + kStatFloats * 4;  // fp32: q's operands [parts][NT][2 J][32] pairs
    static constexpr int kQBytes = kParts == 1 ? 0 : kParts * NT * 2 * J * 32 * 8;
    static constexpr int kLgOff = kQOff + kQBytes;  // [NT][chunk_cap][8] logits, then weights; [chunk_cap] old scores
    static size_t bytes(int chunk_cap) { return (size_t)kLgOff + (size_t)chunk_cap * (kGP + 1) * 4; }
};

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float low_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high_bf16(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// A pair of fp32 values as kParts pairs of bf16 whose sums they are (one part: rounded; three: exactly).
template <int kParts>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&part)[kParts]) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        part[i] = ptx::pack_bf16(a, b);
        if (i + 1 < kParts) a -= low_bf16(part[i]), b -= high_bf16(part[i]);
    }
}

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint2 b) {
    ptx::mma_bf16_16816(d, a0, a1, a2, a3, b.x, b.y);
}

// Both bf16 halves of x less the one with bit pattern c (integers below 256 in units of 2^-133: exact).
__device__ __forceinline__ uint32_t minus(uint32_t x, uint16_t c) {
    const uint32_t cc = (uint32_t)c << 16 | c;
    __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&cc));
    return *reinterpret_cast<uint32_t *>(&r);
}

template <int N>
struct Words {
    uint32_t w[N];
};
template <int N>  // N consecutive 4-byte words of shared memory, aligned to their size
__device__ __forceinline__ Words<N> load_words(const uint8_t *p) {
    Words<N> r;
    if constexpr (N == 4) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        r.w[0] = v.x, r.w[1] = v.y, r.w[2] = v.z, r.w[3] = v.w;
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        r.w[0] = v.x, r.w[1] = v.y;
    } else {
        r.w[0] = *reinterpret_cast<const uint32_t *>(p);
    }
    return r;
}

template <int D, int NT, int kParts, bool kCluster>
__global__ void __launch_bounds__(kThreads) decode_q4_mma_kernel(const MmaQ4Params p) {
    using Lay = Layout<D, NT, kParts>;
    using T = std::conditional_t<kParts == 1, __nv_bfloat16, float>;
    constexpr int J = Lay::J, GP = Lay::kGP, OS = Lay::kOStride;
    constexpr int kWeightParts = kParts == 1 ? VOXZIP_Q4_WP : 3;
    constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;

    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, qd = lane & 3;
    uint8_t *ring = smem + warp * Lay::kWarpRing;
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + Lay::kBarOff) + warp * kStages;
    uint64_t *score_bar = reinterpret_cast<uint64_t *>(smem + Lay::kBarOff) + kWarps * kStages;
    float *m_w = reinterpret_cast<float *>(smem + Lay::kStatOff);  // the warps' maxima
    float *z_w = m_w + kWarps * GP;                                // and sums
    float *f_w = z_w + kWarps * GP;                                // what turns a warp's weights into softmax mass
    float2 *mz = reinterpret_cast<float2 *>(f_w + kWarps * GP);    // this CTA's maximum and sum
    float2 *mz_all = mz + GP;                                      // [S][GP]: every CTA's
    float *lg = reinterpret_cast<float *>(smem + Lay::kLgOff);
    float *s_old = lg + (size_t)p.chunk_cap * GP;

    const int S = kCluster ? p.S : 1;
    const int rank = kCluster ? (int)(blockIdx.x % (unsigned)S) : 0;
    const UnitIdx ui = unit_of((int)(blockIdx.x / (unsigned)S), p.B, p.L, p.Hkv, p.layer_begin);
    const int64_t act = (int64_t)ui.l_local * p.B + ui.b, row_base = ui.cache_unit * p.C;

    if (lane == 0) {
        for (int s = 0; s < kStages; ++s) ptx::mbar_init(&full[s], 1);
        if (warp == 0) ptx::mbar_init(score_bar, 1);
        ptx::fence_mbar_init();
    }
    __syncwarp();
    ptx::grid_dependency_wait();

    const int32_t n_old = p.len[ui.cache_unit], n = n_old + 1;
    if (n_old < 0 || n > p.C || n > p.max_rows) {  // the same decision in every CTA of the cluster
        if (rank == 0 && tid == 0)
            raise_status(p.status, n_old < 0 || n > p.C ? VOXZIP_DEV_CAPACITY : VOXZIP_DEV_LEN_HINT);
        return;
    }
    const int tiles = (n + kTile - 1) / kTile, share = (tiles + S - 1) / S;
    const int tile0 = min(tiles, rank * share), mine = min(tiles, tile0 + share) - tile0;  // this CTA's tiles
    const int j0 = tile0 * kTile, cnt = min(n, j0 + mine * kTile) - j0;                    // and tokens
    const int m = (mine - warp + kWarps - 1) / kWarps;                                     // this warp's tiles
    const int items = 2 * m;                                                               // K tiles, then V tiles

    // Stage i of the warp: tile warp + kWarps (i mod m), rows up to the length, in fours (as the capacity is).
    auto issue = [&](int i) {
        const bool v = i >= m;
        const int tile = tile0 + warp + kWarps * (v ? i - m : i);
        const int rows = min(kTile, (n - tile * kTile + 3) & ~3);
        const int64_t row = row_base + (int64_t)tile * kTile;
        uint8_t *stage = ring + i % kStages * Lay::kStageBytes;
        uint64_t *bar = &full[i % kStages];
        if (!VOXZIP_IN_RANGE(p.status, tile >= 0 && tile * kTile + rows <= p.C && rows > 0)) return;
        ptx::mbar_arrive_expect_tx(bar, (uint32_t)rows * (D / 2 + J * 2));
        ptx::bulk_load(stage, (v ? p.q4.v_codes : p.q4.k_codes) + row * (D / 2), (uint32_t)rows * (D / 2), bar);
        ptx::bulk_load(stage + Lay::kCodeBytes, (v ? p.q4.v_scale : p.q4.k_scale) + row * J, (uint32_t)rows * (J * 2), bar);
    };
    if (lane == 0) {
        for (int i = 0; i < min(kStages, items); ++i) issue(i);
        if (warp == 0 && cnt > 0) {
            const uint32_t bytes = (uint32_t)((cnt + 3) & ~3) * 4;
            ptx::mbar_arrive_expect_tx(score_bar, bytes);
            ptx::bulk_load(s_old, p.score + row_base + j0, bytes, score_bar);
        }
    }

    // The appended row lies in the last tile; the warp that has it packs the row over what the ring brought in,
    // and into the cache.
    const bool appends = mine > 0 && tile0 + mine == tiles && (mine - 1) % kWarps == warp;
    const int8_t *ke = p.q4.k_exp + ui.cache_unit * D;
    float4 kn = make_float4(0.f, 0.f, 0.f, 0.f), vn = kn;
    if (appends && lane < D / 4) {
        const int64_t at = (act * p.Hkv + ui.h) * D + lane * 4;
        kn = load4(static_cast<const T *>(p.k_new) + at);
        vn = load4(static_cast<const T *>(p.v_new) + at);
        const char4 e = *reinterpret_cast<const char4 *>(ke + lane * 4);
        kn.x *= exp2_int(-e.x), kn.y *= exp2_int(-e.y), kn.z *= exp2_int(-e.z), kn.w *= exp2_int(-e.w);
        if (lane == 0) p.pos[row_base + n_old] = p.new_pos[ui.b];
    }
    const int row_new = n_old % kTile;

    // q's operands: lane (g, qd) holds channels 32 j + 8 qd .. + 7 of head g, times 2^e; the pairs that meet codes in
    // bits 4-7 a sixteenth of it. c_init: what the accumulators of heads 2 qd, 2 qd + 1 start from.
    uint2 qb[kParts == 1 ? NT : 1][kParts == 1 ? 2 * J : 1];
    uint2 *q_smem = reinterpret_cast<uint2 *>(smem + Lay::kQOff);
    float c_init[NT][J][2];
    {
        const T *qg = static_cast<const T *>(p.q) + (act * p.Hq + (int64_t)ui.h * p.G) * D;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int head = nt * 8 + g, d = 32 * j + 8 * qd;
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (head < p.G) v = load4(qg + head * D + d + i);
                    const char4 e = *reinterpret_cast<const char4 *>(ke + d + i);
                    x[i] = v.x * exp2_int(e.x), x[i + 1] = v.y * exp2_int(e.y);
                    x[i + 2] = v.z * exp2_int(e.z), x[i + 3] = v.w * exp2_int(e.w);
                }
                float sum = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                sum *= -8.f * (kCarry * 0x1p-133f);
                c_init[nt][j][0] = __shfl_sync(0xffffffffu, sum, 8 * qd);
                c_init[nt][j][1] = __shfl_sync(0xffffffffu, sum, 8 * qd + 4);
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    uint32_t b0[kParts], b1[kParts];
                    split_pair<kParts>(x[4 * ks] * kCarry, x[4 * ks + 1] * kCarry, b0);
                    split_pair<kParts>(x[4 * ks + 2] * (kCarry / 16), x[4 * ks + 3] * (kCarry / 16), b1);
                    if constexpr (kParts == 1) {
                        qb[nt][2 * j + ks] = make_uint2(b0[0], b1[0]);
                    } else if (warp == 0) {
#pragma unroll
                        for (int i = 0; i < kParts; ++i)
                            q_smem[((i * NT + nt) * 2 * J + 2 * j + ks) * 32 + lane] = make_uint2(b0[i], b1[i]);
                    }
                }
            }
    }
    if constexpr (kParts > 1) __syncthreads();
    auto q_operand = [&](int part, int nt, int step) {
        if constexpr (kParts == 1) return qb[nt][step];
        else return q_smem[((part * NT + nt) * 2 * J + step) * 32 + lane];
    };

    bool ok = true;
    int done = 0;  // stages seen to land
    auto wait = [&](int i) {
        ok = ok && __all_sync(0xffffffffu, ptx::mbar_wait_bounded(&full[i % kStages], (i / kStages) & 1, kWaitLimit));
        done = ok ? i + 1 : done;
        return ok;
    };
    auto refill = [&](int i, bool wrote) {  // stage i has been read by every lane
        if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0 && i + kStages < items) issue(i + kStages);
    };

    // Phase K: logits and the warp's maxima.
    float mx[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) mx[nt][0] = mx[nt][1] = -INFINITY;
    for (int i = 0; i < m && wait(i); ++i) {
        uint8_t *stage = ring + i % kStages * Lay::kStageBytes;
        const int local = warp + kWarps * i;  // the CTA's tile
        const int valid = cnt - local * kTile;
        const bool last = appends && i == m - 1;
        if (last) {
            const Q4Row<D, true> row(kn);
            row.store(stage + row_new * (D / 2), reinterpret_cast<__nv_bfloat16 *>(stage + Lay::kCodeBytes) + row_new * J);
            row.store(p.q4.k_codes + (row_base + n_old) * (D / 2), p.q4.k_scale + (row_base + n_old) * J);
            __syncwarp();
        }
#pragma unroll
        for (int mb = 0; mb < 2; ++mb) {
            const int r0 = 16 * mb + g, r1 = r0 + 8;
            const Words<J> w0 = load_words<J>(stage + r0 * (D / 2) + qd * (J * 4));
            const Words<J> w1 = load_words<J>(stage + r1 * (D / 2) + qd * (J * 4));
            const Words<J / 2> s0 = load_words<J / 2>(stage + Lay::kCodeBytes + r0 * (J * 2));
            const Words<J / 2> s1 = load_words<J / 2>(stage + Lay::kCodeBytes + r1 * (J * 2));
            float sum[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[nt][k] = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                float acc[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    acc[nt][0] = acc[nt][2] = c_init[nt][j][0];
                    acc[nt][1] = acc[nt][3] = c_init[nt][j][1];
                }
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const uint32_t x0 = w0.w[j] >> (8 * ks), x1 = w1.w[j] >> (8 * ks);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i2 = 0; i2 < kParts; ++i2)
                            mma(acc[nt], x0 & kLow, x1 & kLow, x0 & kHigh, x1 & kHigh, q_operand(i2, nt, 2 * j + ks));
                }
                const float a = j & 1 ? high_bf16(s0.w[j / 2]) : low_bf16(s0.w[j / 2]);
                const float b = j & 1 ? high_bf16(s1.w[j / 2]) : low_bf16(s1.w[j / 2]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    sum[nt][0] += a * acc[nt][0], sum[nt][1] += a * acc[nt][1];
                    sum[nt][2] += b * acc[nt][2], sum[nt][3] += b * acc[nt][3];
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    sum[nt][k] *= p.scale_log2;
                    if ((k < 2 ? r0 : r1) >= valid) sum[nt][k] = -INFINITY;  // past the length: whatever lies there
                    mx[nt][k & 1] = fmaxf(mx[nt][k & 1], sum[nt][k]);
                }
                float *to = lg + ((size_t)nt * p.chunk_cap + local * kTile) * 8 + 2 * qd;
                *reinterpret_cast<float2 *>(to + r0 * 8) = make_float2(sum[nt][0], sum[nt][1]);
                *reinterpret_cast<float2 *>(to + r1 * 8) = make_float2(sum[nt][2], sum[nt][3]);
            }
        }
        refill(i, last);
    }
    // The warp's maxima: to shared memory for heads 2 qd, 2 qd + 1, to lane (g, .) for head g.
    float mg[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) mx[nt][k] = fmaxf(mx[nt][k], __shfl_xor_sync(0xffffffffu, mx[nt][k], o));
        if (g == 0) {
            m_w[warp * GP + nt * 8 + 2 * qd] = mx[nt][0];
            m_w[warp * GP + nt * 8 + 2 * qd + 1] = mx[nt][1];
        }
        const float even = __shfl_sync(0xffffffffu, mx[nt][0], g >> 1), odd = __shfl_sync(0xffffffffu, mx[nt][1], g >> 1);
        mg[nt] = g & 1 ? odd : even;
    }
    __syncwarp();  // the logits that other lanes stored

    // Phase V. Lane (g, qd) takes tokens 4 i + qd of every 16 and channels 32 j + 4 g .. + 3.
    float o[2 * J][NT][4], z[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        z[nt] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[2 * j][nt][k] = o[2 * j + 1][nt][k] = 0.f;
    }
    for (int i = m; i < items && wait(i); ++i) {
        uint8_t *stage = ring + i % kStages * Lay::kStageBytes;
        const int local = warp + kWarps * (i - m);
        const int valid = cnt - local * kTile;
        const bool last = appends && i == items - 1;
        if (last) {
            const Q4Row<D, false> row(vn);
            row.store(stage + row_new * (D / 2), reinterpret_cast<__nv_bfloat16 *>(stage + Lay::kCodeBytes) + row_new * J);
            row.store(p.q4.v_codes + (row_base + n_old) * (D / 2), p.q4.v_scale + (row_base + n_old) * J);
            __syncwarp();
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            Words<J / 2> w[4], s[4];
            float pr[NT][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 16 * kb + 4 * k + qd;
                w[k] = load_words<J / 2>(stage + t * (D / 2) + g * (J * 2));
                s[k] = load_words<J / 2>(stage + Lay::kCodeBytes + t * (J * 2));
                if (t >= valid) s[k] = Words<J / 2>{};  // past the length a scale may be anything, a NaN too
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float *l = lg + ((size_t)nt * p.chunk_cap + local * kTile + t) * 8 + g;
                    const float x = fast_exp2(*l - mg[nt]);
                    *l = x;
                    z[nt] += x;
                    pr[nt][k] = x * kCarry;
                }
            }
#pragma unroll
            for (int j = 0; j < J; ++j) {
                float sc[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) sc[k] = j & 1 ? high_bf16(s[k].w[j / 2]) : low_bf16(s[k].w[j / 2]);
                const uint32_t x01 = __byte_perm(w[0].w[j / 2], w[1].w[j / 2], j & 1 ? 0x7632 : 0x5410);
                const uint32_t x23 = __byte_perm(w[2].w[j / 2], w[3].w[j / 2], j & 1 ? 0x7632 : 0x5410);
                const uint32_t y01 = x01 >> 8, y23 = x23 >> 8;
                const uint32_t a0 = minus(x01 & kLow, 0x0008), a1 = minus(x01 & kHigh, 0x0080);
                const uint32_t a2 = minus(x23 & kLow, 0x0008), a3 = minus(x23 & kHigh, 0x0080);
                const uint32_t c0 = minus(y01 & kLow, 0x0008), c1 = minus(y01 & kHigh, 0x0080);
                const uint32_t c2 = minus(y23 & kLow, 0x0008), c3 = minus(y23 & kHigh, 0x0080);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    uint32_t b0[kWeightParts], b1[kWeightParts];
                    split_pair<kWeightParts>(pr[nt][0] * sc[0], pr[nt][1] * sc[1], b0);
                    split_pair<kWeightParts>(pr[nt][2] * sc[2], pr[nt][3] * sc[3], b1);
#pragma unroll
                    for (int i2 = 0; i2 < kWeightParts; ++i2) {
                        const uint2 b = make_uint2(b0[i2], b1[i2]);
                        mma(o[2 * j][nt], a0, a1, a2, a3, b);
                        mma(o[2 * j + 1][nt], c0, c1, c2, c3, b);
                    }
                }
            }
        }
        refill(i, last);
    }
    if (!ok) {  // a wait gave up: outputs are not valid; let what is still in flight land (bounded)
        raise_status(p.status, VOXZIP_DEV_TIMEOUT);
        for (int i = done; i < min(items, done + kStages); ++i)
            (void)ptx::mbar_wait_bounded(&full[i % kStages], (i / kStages) & 1, kWaitLimit);
    }
    ptx::launch_dependents();

    // The warp's sums and outputs (in units of 2^-49), the latter over its drained ring.
    float *ow = reinterpret_cast<float *>(ring);
    __syncwarp();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        z[nt] += __shfl_xor_sync(0xffffffffu, z[nt], 1);
        z[nt] += __shfl_xor_sync(0xffffffffu, z[nt], 2);
        if (qd == 0) z_w[warp * GP + nt * 8 + g] = z[nt];
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                *reinterpret_cast<float4 *>(ow + (nt * 8 + 2 * qd + k) * OS + 32 * j + 4 * g) =
                    make_float4(o[2 * j][nt][k], o[2 * j][nt][2 + k] * 0.0625f, o[2 * j + 1][nt][k],
                                o[2 * j + 1][nt][2 + k] * 0.0625f);
    }
    __syncthreads();
    // Per head: the CTA's maximum, its sum, and 2^(m_w - m).
    auto warp_factors = [&](int h, float (&f)[kWarps]) {
        float mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, f[w] = m_w[w * GP + h]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) f[w] = f[w] == -INFINITY ? 0.f : fast_exp2(f[w] - mm);
        return mm;
    };
    T *og = static_cast<T *>(p.out) + (act * p.Hq + (int64_t)ui.h * p.G) * D;
    float *o_cta = reinterpret_cast<float *>(smem);  // warp 0's place
    if (tid < GP) {
        float f[kWarps], zz = 0.f;
        const float mm = warp_factors(tid, f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) zz += f[w] * z_w[w * GP + tid];
        if constexpr (kCluster) mz[tid] = make_float2(mm, zz);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) f_w[w * GP + tid] = kCluster ? f[w] : tid < p.G ? f[w] / zz : 0.f;
    }
    for (int e = tid; e < (kCluster ? GP : p.G) * D / 4; e += kThreads) {
        const int h = e / (D / 4), at = h * OS + e % (D / 4) * 4;
        float f[kWarps];
        warp_factors(h, f);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float zz = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float4 x = *reinterpret_cast<const float4 *>(smem + w * Lay::kWarpRing + at * 4);
            v.x += f[w] * x.x, v.y += f[w] * x.y, v.z += f[w] * x.z, v.w += f[w] * x.w;
            zz += f[w] * z_w[w * GP + h];
        }
        if constexpr (kCluster) {
            *reinterpret_cast<float4 *>(o_cta + at) = v;
        } else {
            const float r = kUncarry / zz;
            T *to = og + h * D + e % (D / 4) * 4;
            to[0] = Elem<T>::from_f(v.x * r), to[1] = Elem<T>::from_f(v.y * r);
            to[2] = Elem<T>::from_f(v.z * r), to[3] = Elem<T>::from_f(v.w * r);
        }
    }
    if constexpr (kCluster) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();  // every CTA's mz and o_cta are final
        auto combine = [&](auto ss_tag) {
            constexpr int SS = decltype(ss_tag)::value;
            constexpr int E = (GP * D / SS + kThreads - 1) / kThreads;
            const int total = p.G * D, per = (total + SS - 1) / SS;
            const int lo = rank * per, hi = min(total, lo + per);
            float part[E][SS];
            for (int t = tid; t < SS * GP; t += kThreads) mz_all[t] = *cluster.map_shared_rank(mz + t % GP, t / GP);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = lo + tid + e * kThreads;
                const int at = i < hi ? (i / D) * OS + i % D : 0;
#pragma unroll
                for (int r = 0; r < SS; ++r) part[e][r] = i < hi ? *cluster.map_shared_rank(&o_cta[at], r) : 0.f;
            }
            __syncthreads();
            if (tid < GP) {  // mz_all[r][h].x becomes 2^(m_r - m) / Z
                float2 x[SS];
                float mm = -INFINITY, zz = 0.f;
#pragma unroll
                for (int r = 0; r < SS; ++r) {
                    x[r] = mz_all[r * GP + tid];
                    mm = fmaxf(mm, x[r].x);
                }
#pragma unroll
                for (int r = 0; r < SS; ++r) {
                    x[r].x = x[r].x == -INFINITY ? 0.f : fast_exp2(x[r].x - mm);
                    zz += x[r].x * x[r].y;
                }
                const float rz = tid < p.G ? 1.f / zz : 0.f;
#pragma unroll
                for (int r = 0; r < SS; ++r) {
                    mz_all[r * GP + tid].x = x[r].x * rz;
                    if (r == rank)
#pragma unroll
                        for (int w = 0; w < kWarps; ++w) f_w[w * GP + tid] *= x[r].x * rz;
                }
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = lo + tid + e * kThreads;
                if (i < hi) {
                    float x = 0.f;
#pragma unroll
                    for (int r = 0; r < SS; ++r) x += mz_all[r * GP + i / D].x * part[e][r];
                    og[i] = Elem<T>::from_f(x * kUncarry);
                }
            }
        };
        switch (S) {
            case 2: combine(std::integral_constant<int, 2>{}); break;
            case 4: combine(std::integral_constant<int, 4>{}); break;
            case 8: combine(std::integral_constant<int, 8>{}); break;
            default: combine(std::integral_constant<int, 16>{}); break;
        }
        ptx::cluster_arrive_relaxed();  // this CTA is done reading its peers' shared memory
    } else {
        __syncthreads();
    }
    // Eq. 6 for the warp's own tokens.
    if (m > 0) {
        float f[GP];
#pragma unroll
        for (int h = 0; h < GP; ++h) f[h] = f_w[warp * GP + h];
        if (!ptx::mbar_wait_bounded(score_bar, 0, kWaitLimit)) raise_status(p.status, VOXZIP_DEV_TIMEOUT);
        for (int i = warp * kTile + lane; i < cnt; i += kThreads) {
            float add = 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float4 *w = reinterpret_cast<const float4 *>(lg + ((size_t)nt * p.chunk_cap + i) * 8);
                const float4 a = w[0], b = w[1];
                add += ((a.x * f[nt * 8] + a.y * f[nt * 8 + 1]) + (a.z * f[nt * 8 + 2] + a.w * f[nt * 8 + 3])) +
                       ((b.x * f[nt * 8 + 4] + b.y * f[nt * 8 + 5]) + (b.z * f[nt * 8 + 6] + b.w * f[nt * 8 + 7]));
            }
            if (VOXZIP_IN_RANGE(p.status, j0 + i < p.C))
                p.score[row_base + j0 + i] = j0 + i == n_old ? add : p.gamma * s_old[i] + add;
        }
    }
    if (rank == 0 && tid == 0) p.len[ui.cache_unit] = n;
    if constexpr (kCluster) ptx::cluster_wait();  // no CTA leaves while a peer may still read its shared memory
}

// ---------------------------------------------------------------- host side
using KernelFn = void (*)(MmaQ4Params);

template <int D, int NT, int kParts>
struct Kernels {
    using Lay = Layout<D, NT, kParts>;
    static KernelFn of(int S) {
        return S == 1 ? decode_q4_mma_kernel<D, NT, kParts, false> : decode_q4_mma_kernel<D, NT, kParts, true>;
    }
};

template <typename K>
cudaError_t configure() {
    static std::atomic<uint64_t> done{0};
    return once_per_device(done, [] {
        for (KernelFn kern : {K::of(1), K::of(2)}) {
            cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxSmem);
            if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            if (e != cudaSuccess) return e;
        }
        return cudaSuccess;
    });
}

template <typename F>
auto by_shape(const voxzip_cache_desc &d, F &&f) {
    const bool two = d.q_heads / d.kv_heads > 8, bf16 = d.dtype == VOXZIP_BF16;
    if (d.head_dim == 128) {
        if (two) return bf16 ? f(Kernels<128, 2, 1>{}) : f(Kernels<128, 2, 3>{});
        return bf16 ? f(Kernels<128, 1, 1>{}) : f(Kernels<128, 1, 3>{});
    }
    if (two) return bf16 ? f(Kernels<64, 2, 1>{}) : f(Kernels<64, 2, 3>{});
    return bf16 ? f(Kernels<64, 1, 1>{}) : f(Kernels<64, 1, 3>{});
}

#ifndef VOXZIP_Q4_FORCE_S
#define VOXZIP_Q4_FORCE_S 0
#endif

// CTAs per unit.
int plan(const voxzip_cache_desc &d, int units, int nmax, int *chunk_cap) {
    const int tiles = (nmax + kTile - 1) / kTile;
    for (int S = 1; S <= kMaxCluster; S <<= 1) {
        const int cap = (tiles + S - 1) / S * kTile;
        const size_t smem = by_shape(d, [&](auto k) { return decltype(k)::Lay::bytes(cap); });
        *chunk_cap = cap;
        if (smem > kMaxSmem) continue;
        if (VOXZIP_Q4_FORCE_S ? S >= VOXZIP_Q4_FORCE_S
                              : S == kMaxCluster || cap <= kTile * kWarps || (units * S >= 3 * sm_count() && smem <= kMaxSmem / 3))
            return (int64_t)units * S <= INT32_MAX ? S : 0;
    }
    return 0;
}

}  // namespace

cudaError_t launch_decode_q4(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                             const void *q, const void *k_new, const void *v_new, const int32_t *new_pos, float *score,
                             int32_t *pos, int32_t *len, float gamma, float sm_scale, int32_t max_len, void *out,
                             int32_t *status, cudaStream_t stream) {
    const int nmax = (max_len > 0 && max_len < d.capacity) ? max_len : d.capacity;
    const int units = layer_count * d.batch * d.kv_heads;
    int chunk_cap = 0;
    const int S = plan(d, units, nmax, &chunk_cap);
    if (S == 0)
        return launch_decode_q4_rows(d, q4, layer_begin, layer_count, q, k_new, v_new, new_pos, score, pos, len, gamma,
                                     sm_scale, max_len, out, status, stream);
    const float scale = sm_scale > 0.f ? sm_scale : 1.0f / sqrtf((float)d.head_dim);
    const MmaQ4Params prm{q4, q, k_new, v_new, new_pos, score, pos, len, out, status, d.batch, d.layers, d.q_heads,
                          d.kv_heads, d.q_heads / d.kv_heads, d.capacity, layer_begin, S, chunk_cap, nmax, gamma,
                          scale * 1.4426950408889634f * kUncarry};
    return by_shape(d, [&](auto k) {
        using K = decltype(k);
        const cudaError_t set = configure<K>();
        if (set != cudaSuccess) return set;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)units * (unsigned)S, 1, 1);
        cfg.blockDim = dim3(kThreads, 1, 1);
        cfg.dynamicSmemBytes = K::Lay::bytes(chunk_cap);
        cfg.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)S;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // overlap the previous kernel's tail
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        cudaError_t err = cudaLaunchKernelEx(&cfg, K::of(S), prm);
        if (err == cudaErrorNotSupported || err == cudaErrorInvalidValue) {  // no programmatic launch here
            cudaGetLastError();
            cfg.numAttrs = 1;
            err = cudaLaunchKernelEx(&cfg, K::of(S), prm);
        }
        return err;
    });
}

}  // namespace voxzip
