// Decode step on a cache held in 4 bits (format: q4.cuh): append (Eq. 1), GQA attention (Eq. 2) and the
// decayed-score update (Eq. 6), reading each packed K and V row once.
//
//   l_h[t] = scale sum_j s[t][j] sum_{d in j} (q_hd 2^e_d) c[t][d]        (groups j of 32 channels)
//   out_h[d] = sum_t (p_h[t] s[t][j(d)]) c[t][d] / sum_t p_h[t]
// The codes are small integers, so they go to the tensor cores (mma.sync m16n8k16, bf16) as they are: exact, and
// without a multiplication by their scale. For K the scale multiplies the fp32 sum of a group (two k-steps); for V
// it multiplies the weight before that is split. A nibble becomes an operand by one AND: as a bf16 bit pattern, the
// integer v in 0..255 is v 2^-133 (a subnormal or in the first binade above, one straight line), so a code in bits
// 0-3 is c 2^-133 and one in bits 4-7 is 16 c 2^-133; q and p carry 2^84 (q of the odd pairs 2^80), and what is left,
// 2^-49, goes into factors that are applied anyway. The stored code is c + 8: for K the accumulators start from
// -8 sum q; for V (and for K of fp32 activations) eight is subtracted from the operands, since an output may be far
// smaller than its weights' sum, so that a correction afterwards would cancel.
// Roundings: a bf16 weight times scale is two bf16 parts (15 bits at least; one part's 8 bits would make the output's
// rounding error 1.36 times as large, for a tenth of the time), fp32 activations and their weights three (24 bits). Sums
// are fp32.
//
// Grid: S CTAs per (layer, sequence, kv-head) unit, a thread-block cluster where S > 1; CTA r owns a run of 32-token
// tiles, and its warp w every fourth of them. Every warp streams its own K tiles and then its V tiles through a ring
// of its own (cp.async by all lanes: bulk copies issued by one lane, with their barriers, cost four times the
// instructions per tile), so nothing in the streaming waits for another warp: the weights are taken relative to the
// warp's own maximum. The logits, then the weights, stay in shared memory until the unit's maximum and normaliser are
// known: each CTA sends its statistics and outputs to the cluster's CTAs and meets them at one barrier, after which
// each writes a slice of the outputs and every warp the scores of its own tokens.
//
// What bounds it: instructions and the chain of latencies at a CTA's start and end, not HBM. A row of 152 bytes is 6.3
// cycles of an SM's share of HBM and 28 warp instructions (K 6, V 12, the rest start, end and tiles); of a CTA's 14 us
// at 768 units of 2 317 rows, 6 to 7 stream. Measured, bf16, G = 8, D = 128, back to back: 768 units of 2 317 rows 80 us
// (3.4 TB/s, 0.50 of the measured copy rate; the same rows in bf16 take 148), of 11 522 389 us (0.51); 192 units of 416
// 8.4 us; 6 144 of 1 564 355 us (0.61). fp32: 116, 550 and 11 us of the first three. A call per layer, from a graph: 5.3
// us for 4 units of 416 rows, 7.6 for 16 of 2 317. Asking the whole range into L2 at the start gained nothing, nor did
// starting the first CTAs apart, five CTAs per SM (96 registers), or fp16 weights (whose range loses the least ones).
#include <cooperative_groups.h>

#include <type_traits>

#include "decode_q4_plan.cuh"
#include "q4.cuh"

namespace cg = cooperative_groups;

namespace voxzip {
namespace {

using namespace q4;
static_assert(kGroup == kQ4Group, "the plan counts the format's groups");

constexpr float kCarry = 0x1p84f, kUncarry = 0x1p49f;
constexpr float kLeast = -3.402823466e38f;

struct MmaQ4Params {
    Q4View q4;
    const void *q, *k_new, *v_new;
    const int32_t *new_pos;
    float *score;
    int32_t *pos, *len;
    void *out;
    int32_t *status;
    int32_t B, L, Hq, Hkv, G, C, layer_begin, chunk_cap, max_rows;
    int32_t S, stages, slice;               // CTAs per unit; each writes this many float4 of its G D outputs
    int32_t next_h, next_b, next_l; // how far the unit lies whose CTAs take these ones' place (next_l < 0: none)
    uint32_t inv_s, inv_slice;      // ceil(2^32 / S), ceil(2^32 / slice): quotients by __umulhi
    float gamma, scale_log2;  // scale_log2: logits in units of log 2, times kUncarry
};

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float low_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high_bf16(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

__device__ __forceinline__ float2 times(float2 a, float2 b) {  // both products in one instruction
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\t"
        "mov.b64 {%0, %1}, z;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 less(float2 a, float2 b) {  // a - b, both in one instruction
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tsub.rn.f32x2 z, x, y;\n\t"
        "mov.b64 {%0, %1}, z;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// A pair of fp32 values as kParts pairs of bf16: each takes the upper half of what is left (8 bits), one pair
// alone is rounded. Two leave 2^-15 of a value, three nothing.
template <int kParts>
__device__ __forceinline__ void split_pair(float2 a, uint32_t (&part)[kParts]) {
    if constexpr (kParts == 1) {
        part[0] = ptx::pack_bf16(a.x, a.y);
    } else {
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            part[i] = __byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x7632);
            if (i + 1 < kParts)
                a = less(a, make_float2(high_bf16(__float_as_uint(a.x)), high_bf16(__float_as_uint(a.y))));
        }
    }
}

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint2 b) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y));
}
// Half of it: the first operands of A's rows, 8 of the 16 terms.
__device__ __forceinline__ void mma_half(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(b));
}
// The same, from c: an accumulator that stays as it is.
__device__ __forceinline__ void mma_from(float (&d)[4], const float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint2 b) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// Both bf16 halves of x less the one with bit pattern c (integers below 256 in units of 2^-133: exact).
__device__ __forceinline__ uint32_t minus(uint32_t x, uint16_t c) {
    const uint32_t cc = (uint32_t)c << 16 | c;
    __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&cc));
    return *reinterpret_cast<uint32_t *>(&r);
}
// kBytes from global to shared memory, asynchronously (of this thread's current group).
template <int kBytes>
__device__ __forceinline__ void copy_async(void *dst, const void *src) {
    if constexpr (kBytes == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(dst)), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(ptx::smem_u32(dst)), "l"(src), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {  // all but this thread's last N groups have landed
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Eight consecutive elements of q and their channels' exponents, as loaded.
template <typename T>
struct RawQ {
    uint4 v[sizeof(T) / 2];
    int2 e;
    __device__ __forceinline__ void load(const T *q, const int8_t *exps) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = reinterpret_cast<const uint4 *>(q)[i];
        e = *reinterpret_cast<const int2 *>(exps);
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const {  // times 2^e
        const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[2 * i] = low_bf16(w[i]), x[2 * i + 1] = high_bf16(w[i]);
        } else {
            const uint32_t w2[4] = {v[sizeof(T) / 2 - 1].x, v[sizeof(T) / 2 - 1].y, v[sizeof(T) / 2 - 1].z, v[sizeof(T) / 2 - 1].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]), x[4 + i] = __uint_as_float(w2[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= exp2_int((int)(int8_t)((i < 4 ? e.x : e.y) >> (8 * (i & 3))));
    }
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_index() {  // of the cluster, along x
    uint32_t r;
    asm("mov.u32 %0, %%clusterid.x;" : "=r"(r));
    return r;
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
__global__ void __launch_bounds__(kThreads, NT == 1 && kParts == 1 ? 4 : 3) decode_q4_mma_kernel(const MmaQ4Params p) {
    using Lay = Layout<D, NT, kParts>;
    using T = std::conditional_t<kParts == 1, __nv_bfloat16, float>;
    constexpr int J = Lay::J, GP = Lay::kGP, OS = Lay::kOStride;
    constexpr int kWeightParts = kParts == 1 ? 2 : 3;  // one part (8 bits) would double the output's rounding error
    constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;

    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, qd = lane & 3;
    const int stages = p.stages, ring_bytes = Lay::warp_ring(stages), wrap = (stages - 1) * Lay::kStageBytes;
    uint8_t *ring = smem + warp * ring_bytes, *rest = smem + kWarps * ring_bytes;
    float *m_w = reinterpret_cast<float *>(rest + Lay::kStatOff);  // the warps' maxima
    float *z_w = m_w + kWarps * GP;                                // and sums
    float *f_w = z_w + kWarps * GP;                                // what turns a warp's weights into softmax mass
    float2 *mz_rx = reinterpret_cast<float2 *>(rest + Lay::kMzOff);  // [S][GP] maxima and sums of the cluster's CTAs
    const int S = kCluster ? p.S : 1;
    float4 *o_rx = reinterpret_cast<float4 *>(mz_rx + S * GP);       // [S][slice] their outputs, this CTA's slice
    float *lg = reinterpret_cast<float *>(rest + Lay::lg_off(S));
    const int rank = kCluster ? (int)cluster_rank() : 0;
    UnitIdx ui;  // the grid is [layers][B][Hkv S]
    ui.h = kCluster ? (int)cluster_index() : (int)blockIdx.x;
    ui.b = (int)blockIdx.y;
    ui.l_local = (int)blockIdx.z;
    ui.l = p.layer_begin + ui.l_local;
    ui.cache_unit = ((int64_t)ui.b * p.L + ui.l) * p.Hkv + ui.h;
    const int64_t act = (int64_t)ui.l_local * p.B + ui.b, row_base = ui.cache_unit * p.C;

    ptx::grid_dependency_wait();
    // The length first, then the warp's share of q (which does not depend on it): one memory latency for both.
    const int32_t n_old = *static_cast<const volatile int32_t *>(p.len + ui.cache_unit);
    const int8_t *ke = p.q4.k_exp + ui.cache_unit * D;
    const T *qg = static_cast<const T *>(p.q) + (act * p.Hq + (int64_t)ui.h * p.G) * D;
    constexpr int kShare = (NT * J + kWarps - 1) / kWarps;
    RawQ<T> q_raw[kShare];
#pragma unroll
    for (int it = 0; it < kShare; ++it) {
        const int nj = it * kWarps + warp, head = nj / J * 8 + g, d = 32 * (nj % J) + 8 * qd;
        q_raw[it] = RawQ<T>{};
        if (nj < NT * J && head < p.G) q_raw[it].load(qg + head * D + d, ke + d);
    }
    if (n_old < 0 || n_old >= min(p.C, p.max_rows)) {  // the same decision in every CTA of the cluster
        if (rank == 0 && tid == 0)
            raise_status(p.status, n_old < 0 || n_old >= p.C ? VOXZIP_DEV_CAPACITY : VOXZIP_DEV_LEN_HINT);
        return;
    }
    const int32_t n = n_old + 1;
    const int tiles = (n + kTile - 1) / kTile, share = kCluster ? (int)__umulhi(tiles + S - 1, p.inv_s) : tiles;
    const int tile0 = min(tiles, rank * share), mine = min(tiles, tile0 + share) - tile0;  // this CTA's tiles
    const int j0 = tile0 * kTile, cnt = min(n, j0 + mine * kTile) - j0;                    // and tokens
    const int m = (mine - warp + kWarps - 1) / kWarps;                                     // this warp's tiles
    const int items = 2 * m;                                                               // K tiles, then V tiles

    // The ring: item i of the warp (tile warp + kWarps (i mod m) of the CTA) goes to slot i mod `stages`. Each lane
    // copies 16-byte pieces of the codes and one row's scales; of the last tile, rows up to the length in fours (as
    // the capacity is). One copy group per item, empty past the last.
    constexpr int kPieces = Lay::kCodeBytes / 512;  // per lane
    const int64_t first = row_base + j0 + warp * kTile;
    const uint8_t *next_codes = p.q4.k_codes + first * (D / 2) + lane * 16;
    const __nv_bfloat16 *next_scale = p.q4.k_scale + (first + lane) * J;
    int next = 0, next_slot = 0, next_left = n - j0 - warp * kTile;  // the item, its slot, rows from its tile's first on
    auto issue = [&]() {
        if (next < items) {
            uint8_t *stage = ring + next_slot;
            const int rows = (next_left + 3) & ~3;
            if (VOXZIP_IN_RANGE(p.status, next_left > 0 && n - next_left + min(rows, kTile) <= p.C)) {
#pragma unroll
                for (int k = 0; k < kPieces; ++k)
                    if (lane / (D / 32) + k * (kTile / kPieces) < rows) copy_async<16>(stage + lane * 16 + k * 512, next_codes + k * 512);
                if (lane < rows) copy_async<J * 2>(stage + Lay::kCodeBytes + lane * (J * 2), next_scale);
            }
            if (++next == m) {
                next_codes = p.q4.v_codes + first * (D / 2) + lane * 16;
                next_scale = p.q4.v_scale + (first + lane) * J;
                next_left = n - j0 - warp * kTile;
            } else {
                next_codes += kWarps * Lay::kCodeBytes;
                next_scale += kWarps * kTile * J;
                next_left -= kWarps * kTile;
            }
            next_slot = next_slot == wrap ? 0 : next_slot + Lay::kStageBytes;
        }
        copy_commit();
    };
    if (tid == 0 && cnt > 0) ptx::prefetch_l2(p.score + row_base + j0, (uint32_t)((cnt + 3) & ~3) * 4);
    for (int i = 0; i < stages - 1; ++i) issue();

    // The appended row lies in the last tile; the warp that has it packs the row over what the ring brought in,
    // and into the cache.
    const bool appends = mine > 0 && tile0 + mine == tiles && (mine - 1) % kWarps == warp;
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
    // bits 4-7 a sixteenth of it. The warps make a share each, and of the sums that the accumulators start from.
    uint2 *q_smem = reinterpret_cast<uint2 *>(rest + Lay::kQOff);
    float *c_smem = reinterpret_cast<float *>(rest + Lay::kCOff);
#pragma unroll
    for (int it = 0; it < kShare; ++it) {
        const int nj = it * kWarps + warp;
        if (nj < NT * J) {
            const int nt = nj / J, j = nj % J;
            float x[8];
            q_raw[it].widen(x);
            float sum = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            if (qd == 0) c_smem[nj * 8 + g] = kParts == 1 ? sum * (-8.f * (kCarry * 0x1p-133f)) : 0.f;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                uint32_t b0[kParts], b1[kParts];
                split_pair<kParts>(make_float2(x[4 * ks] * kCarry, x[4 * ks + 1] * kCarry), b0);
                split_pair<kParts>(make_float2(x[4 * ks + 2] * (kCarry / 16), x[4 * ks + 3] * (kCarry / 16)), b1);
#pragma unroll
                for (int i = 0; i < kParts; ++i)
                    q_smem[((i * NT + nt) * 2 * J + 2 * j + ks) * 32 + lane] = make_uint2(b0[i], b1[i]);
            }
        }
    }
    __syncthreads();
    uint2 qb[kParts == 1 ? NT : 1][kParts == 1 ? 2 * J : 1];
    if constexpr (kParts == 1) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int step = 0; step < 2 * J; ++step) qb[nt][step] = q_smem[(nt * 2 * J + step) * 32 + lane];
    }
    float c_init[NT][J][4];  // heads 2 qd, 2 qd + 1, for the two rows of an accumulator
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const float2 c = *reinterpret_cast<const float2 *>(c_smem + (nt * J + j) * 8 + 2 * qd);
            c_init[nt][j][0] = c_init[nt][j][2] = c.x;
            c_init[nt][j][1] = c_init[nt][j][3] = c.y;
        }
    if constexpr (kCluster) {  // this CTA runs, and has q: the others may send to it once all its warps say so
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    }
    auto q_operand = [&](int part, int nt, int step) {
        if constexpr (kParts == 1) return qb[nt][step];
        else return q_smem[((part * NT + nt) * 2 * J + step) * 32 + lane];
    };

    int slot = 0;
    auto stage_of_next = [&]() {  // the next item's stage, landed, and every lane done with the one before
        if (stages == 2) copy_wait<0>();
        else copy_wait<1>();
        __syncwarp();
        uint8_t *stage = ring + slot;
        slot = slot == wrap ? 0 : slot + Lay::kStageBytes;
        issue();
        return stage;
    };

    // Phase K: logits (before the softmax scale, in units of 2^-49) and the warp's maxima.
    float mx[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) mx[nt][0] = mx[nt][1] = -INFINITY;
    auto k_tile = [&](auto full_tag, const uint8_t *stage, int local, int valid) {
        constexpr bool kFull = decltype(full_tag)::value;
#pragma unroll
        for (int mb = 0; mb < kTile / 16; ++mb) {
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
                uint32_t x[2][4];
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const uint32_t x0 = w0.w[j] >> (8 * ks), x1 = w1.w[j] >> (8 * ks);
                    x[ks][0] = x0 & kLow, x[ks][1] = x1 & kLow, x[ks][2] = x0 & kHigh, x[ks][3] = x1 & kHigh;
                    if constexpr (kParts > 1)  // codes without their offset: sums of smaller terms round less
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[ks][k] = minus(x[ks][k], k < 2 ? 0x0008 : 0x0080);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if constexpr (kParts == 1) {
                        mma_from(acc[nt], c_init[nt][j], x[0][0], x[0][1], x[0][2], x[0][3], q_operand(0, nt, 2 * j));
                        mma(acc[nt], x[1][0], x[1][1], x[1][2], x[1][3], q_operand(0, nt, 2 * j + 1));
                    } else {
                        // The tensor cores cut off what an addition does not hold: the lesser parts' sum first, and the
                        // greatest part's products added to it with rounding.
                        float hi[2][4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[nt][k] = hi[0][k] = hi[1][k] = 0.f;
#pragma unroll
                        for (int part = kParts - 1; part >= 0; --part)
#pragma unroll
                            for (int ks = 0; ks < 2; ++ks)
                                mma(part ? acc[nt] : hi[ks], x[ks][0], x[ks][1], x[ks][2], x[ks][3], q_operand(part, nt, 2 * j + ks));
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[nt][k] += hi[0][k] + hi[1][k];
                    }
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
                    if (!kFull && (k < 2 ? r0 : r1) >= valid) sum[nt][k] = -INFINITY;  // past the length: whatever lies there
                    mx[nt][k & 1] = fmaxf(mx[nt][k & 1], sum[nt][k]);
                }
                float *to = lg + ((size_t)nt * p.chunk_cap + local * kTile) * 8 + 2 * qd;
                *reinterpret_cast<float2 *>(to + r0 * 8) = make_float2(sum[nt][0], sum[nt][1]);
                *reinterpret_cast<float2 *>(to + r1 * 8) = make_float2(sum[nt][2], sum[nt][3]);
            }
        }
    };
    for (int i = 0; i < m; ++i) {
        uint8_t *stage = stage_of_next();
        const int local = warp + kWarps * i;  // the CTA's tile
        const int valid = cnt - local * kTile;
        const bool last = appends && i == m - 1;
        if (last) {
            const Q4Row<D, true> row(kn);
            row.store(stage + row_new * (D / 2), reinterpret_cast<__nv_bfloat16 *>(stage + Lay::kCodeBytes) + row_new * J);
            row.store(p.q4.k_codes + (row_base + n_old) * (D / 2), p.q4.k_scale + (row_base + n_old) * J);
            __syncwarp();
        }
        if (valid >= kTile) k_tile(std::true_type{}, stage, local, valid);
        else k_tile(std::false_type{}, stage, local, valid);
    }
    // The warp's maxima: to shared memory for heads 2 qd, 2 qd + 1, to lane (g, .) for head g.
    float mg[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) mx[nt][k] = fmaxf(mx[nt][k], __shfl_xor_sync(0xffffffffu, mx[nt][k], o));
#pragma unroll
        for (int k = 0; k < 2; ++k) mx[nt][k] *= p.scale_log2;
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
    float *sc_w = reinterpret_cast<float *>(rest + Lay::kScOff) + warp * (J * kTile);  // [J][32] a tile's scales
    for (int i = 0; i < m; ++i) {
        uint8_t *stage = stage_of_next();
        const int local = warp + kWarps * i;
        const int valid = cnt - local * kTile;
        if (appends && i == m - 1) {
            const Q4Row<D, false> row(vn);
            row.store(stage + row_new * (D / 2), reinterpret_cast<__nv_bfloat16 *>(stage + Lay::kCodeBytes) + row_new * J);
            row.store(p.q4.v_codes + (row_base + n_old) * (D / 2), p.q4.v_scale + (row_base + n_old) * J);
            __syncwarp();
        }
        {  // Lane t widens the scales of token t; zero past the length, where a scale may be anything, a NaN too.
            Words<J / 2> s = load_words<J / 2>(stage + Lay::kCodeBytes + lane * (J * 2));
#pragma unroll
            for (int k = 0; k < J / 2; ++k) {
                if (lane >= valid) s.w[k] = 0u;
                float *to = sc_w + 2 * k * kTile + ((lane & 16) | (lane & 3) << 2 | (lane >> 2 & 3));
                to[0] = low_bf16(s.w[k]);
                to[kTile] = high_bf16(s.w[k]);
            }
            __syncwarp();
        }
#pragma unroll
        for (int kb = 0; kb < kTile / 16; ++kb) {
            Words<J / 2> w[4];
            float2 p01[NT], p23[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float *l = lg + ((size_t)nt * p.chunk_cap + local * kTile + 16 * kb + qd) * 8 + g;
                float x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    x[k] = fast_exp2(fmaf(l[k * 32], p.scale_log2, -mg[nt]));
                    l[k * 32] = x[k];
                }
                z[nt] += (x[0] + x[1]) + (x[2] + x[3]);
                p01[nt] = make_float2(x[0] * kCarry, x[1] * kCarry);
                p23[nt] = make_float2(x[2] * kCarry, x[3] * kCarry);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = load_words<J / 2>(stage + (16 * kb + 4 * k + qd) * (D / 2) + g * (J * 2));
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const float4 sc = *reinterpret_cast<const float4 *>(sc_w + j * kTile + 16 * kb + 4 * qd);
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
                    split_pair<kWeightParts>(times(p01[nt], make_float2(sc.x, sc.y)), b0);
                    split_pair<kWeightParts>(times(p23[nt], make_float2(sc.z, sc.w)), b1);
                    if constexpr (kParts == 1) {
#pragma unroll
                        for (int part = kWeightParts - 1; part >= 0; --part) {
                            const uint2 b = make_uint2(b0[part], b1[part]);
                            mma(o[2 * j][nt], a0, a1, a2, a3, b);
                            mma(o[2 * j + 1][nt], c0, c1, c2, c3, b);
                        }
                    } else {
                        // The tensor cores cut off, of every term, what their sum does not hold: the lesser parts apart,
                        // the greatest part 8 tokens at a time, and rounding between.
                        float t[2][4], u[2][2][4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) t[0][k] = t[1][k] = u[0][0][k] = u[0][1][k] = u[1][0][k] = u[1][1][k] = 0.f;
#pragma unroll
                        for (int part = kWeightParts - 1; part > 0; --part) {
                            const uint2 b = make_uint2(b0[part], b1[part]);
                            mma(t[0], a0, a1, a2, a3, b);
                            mma(t[1], c0, c1, c2, c3, b);
                        }
                        mma_half(u[0][0], a0, a1, b0[0]);
                        mma_half(u[0][1], a2, a3, b1[0]);
                        mma_half(u[1][0], c0, c1, b0[0]);
                        mma_half(u[1][1], c2, c3, b1[0]);
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                            for (int k = 0; k < 4; ++k) o[2 * j + mt][nt][k] += (t[mt][k] + u[mt][0][k]) + u[mt][1][k];
                    }
                }
            }
        }
    }
    // The CTA that will take this one's place: its rows are asked into L2 now, so that HBM works on while this one
    // puts its results together and that one starts.
    if (warp == kWarps - 1 && p.next_l >= 0) {
        int h2 = ui.h + p.next_h, b2 = ui.b + p.next_b, l2 = ui.l_local + p.next_l;
        if (h2 >= p.Hkv) h2 -= p.Hkv, ++b2;
        if (b2 >= p.B) b2 -= p.B, ++l2;
        if (l2 < (int)gridDim.z) {
            const int64_t unit2 = ((int64_t)b2 * p.L + p.layer_begin + l2) * p.Hkv + h2;
            const int n2 = min(max(ptx::load_relaxed(p.len + unit2), 0), p.C - 1) + 1;  // only aims: it may be about to change
            const int tiles2 = (n2 + kTile - 1) / kTile, share2 = kCluster ? (int)__umulhi(tiles2 + S - 1, p.inv_s) : tiles2;
            const int first2 = min(tiles2, rank * share2) * kTile;
            const int rows2 = (min(n2, first2 + share2 * kTile) - first2 + 3) & ~3;
            if (lane == 0 && rows2 > 0 && VOXZIP_IN_RANGE(p.status, first2 + rows2 <= p.C)) {
                const int64_t row = unit2 * p.C + first2;
                ptx::prefetch_l2(p.q4.k_codes + row * (D / 2), (uint32_t)rows2 * (D / 2));
                ptx::prefetch_l2(p.q4.k_scale + row * J, (uint32_t)rows2 * (J * 2));
            }
        }
    }
    // The old scores of the first tokens travel while the CTA and the cluster put their statistics together.
    constexpr int kAhead = 6;
    float old[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        const int i = warp * kTile + lane + k * kThreads;
        old[k] = i < cnt ? p.score[row_base + j0 + i] : 0.f;
    }
    ptx::launch_dependents();

    // The warp's sums and outputs, the latter over its drained ring.
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
                    make_float4(o[2 * j][nt][k] * kUncarry, o[2 * j][nt][2 + k] * (kUncarry / 16), o[2 * j + 1][nt][k] * kUncarry,
                                o[2 * j + 1][nt][2 + k] * (kUncarry / 16));
    }
    __syncthreads();
    // Per head: the CTA's maximum, and 2^(m_w - m). A warp without tiles has -inf: 0 for any finite m.
    auto warp_factors = [&](int h, float (&f)[kWarps]) {
        float mm = kLeast;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, f[w] = m_w[w * GP + h]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) f[w] = fast_exp2(f[w] - mm);
        return mm;
    };
    auto warp_sum = [&](int h, const float (&f)[kWarps]) {
        float zz = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) zz += f[w] * z_w[w * GP + h];
        return zz;
    };
    T *og = static_cast<T *>(p.out) + (act * p.Hq + (int64_t)ui.h * p.G) * D;
    auto store_out = [&](int e, const float4 &v, float r) {  // float4 e of the unit's outputs
        T *to = og + 4 * e;
        to[0] = Elem<T>::from_f(v.x * r), to[1] = Elem<T>::from_f(v.y * r);
        to[2] = Elem<T>::from_f(v.z * r), to[3] = Elem<T>::from_f(v.w * r);
    };
    if constexpr (kCluster) {
        ptx::cluster_wait();  // every CTA of the cluster runs
        cg::cluster_group cluster = cg::this_cluster();
        for (int t = tid; t < S * GP; t += kThreads) {
            const int h = t % GP;
            float f[kWarps];
            const float mm = warp_factors(h, f);
            *cluster.map_shared_rank(mz_rx + rank * GP + h, t / GP) = make_float2(mm, warp_sum(h, f));
        }
    }
    for (int e = tid; e < p.G * D / 4; e += kThreads) {
        const int h = e / (D / 4), at = h * OS + e % (D / 4) * 4;
        float f[kWarps];
        warp_factors(h, f);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float4 x = *reinterpret_cast<const float4 *>(smem + w * ring_bytes + at * 4);
            v.x += f[w] * x.x, v.y += f[w] * x.y, v.z += f[w] * x.z, v.w += f[w] * x.w;
        }
        if constexpr (kCluster) {  // to the CTA that writes it
            const int to = (int)__umulhi(e, p.inv_slice);
            *cg::this_cluster().map_shared_rank(o_rx + rank * p.slice + (e - to * p.slice), to) = v;
        } else {
            store_out(e, v, 1.f / warp_sum(h, f));
        }
    }
    // What turns weights into softmax mass: 2^(m_r - m) / Z for CTA r of the unit.
    auto unit_stats = [&](int h, float &mm) {  // returns 1 / Z
        float zz = 0.f;
        mm = kLeast;
        for (int r = 0; r < S; ++r) mm = fmaxf(mm, mz_rx[r * GP + h].x);
        for (int r = 0; r < S; ++r) zz += fast_exp2(mz_rx[r * GP + h].x - mm) * mz_rx[r * GP + h].y;
        return 1.f / zz;
    };
    if constexpr (kCluster) {
        // What the others sent has landed, and nobody touches another's memory from here on.
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        for (int i = tid; i < p.slice; i += kThreads) {
            const int e = rank * p.slice + i;
            if (e >= p.G * D / 4) break;
            const int h = e / (D / 4);
            float mm;
            const float rz = unit_stats(h, mm);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int r = 0; r < S; ++r) {
                const float f = fast_exp2(mz_rx[r * GP + h].x - mm);
                const float4 x = o_rx[r * p.slice + i];
                v.x += f * x.x, v.y += f * x.y, v.z += f * x.z, v.w += f * x.w;
            }
            store_out(e, v, rz);
        }
    }
    // Eq. 6 for the warp's own tokens.
    if (m > 0) {
        if (lane < GP) {
            float f[kWarps], mm, r;
            const float m_cta = warp_factors(lane, f);
            if constexpr (kCluster) {
                r = unit_stats(lane, mm);
                r *= fast_exp2(m_cta - mm);
            } else {
                r = 1.f / warp_sum(lane, f);
            }
#pragma unroll
            for (int w = 0; w < kWarps; ++w)
                if (w == warp) f_w[w * GP + lane] = lane < p.G ? f[w] * r : 0.f;
        }
        __syncwarp();
        float f[GP];
#pragma unroll
        for (int h = 0; h < GP; ++h) f[h] = f_w[warp * GP + h];
        auto mass = [&](int i) {
            float add = 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float4 *w = reinterpret_cast<const float4 *>(lg + ((size_t)nt * p.chunk_cap + i) * 8);
                const float4 a = w[0], b = w[1];
                add += ((a.x * f[nt * 8] + a.y * f[nt * 8 + 1]) + (a.z * f[nt * 8 + 2] + a.w * f[nt * 8 + 3])) +
                       ((b.x * f[nt * 8 + 4] + b.y * f[nt * 8 + 5]) + (b.z * f[nt * 8 + 6] + b.w * f[nt * 8 + 7]));
            }
            return add;
        };
        auto update = [&](int i, float before, float add) {
            if (i < cnt && VOXZIP_IN_RANGE(p.status, j0 + i < p.C))
                p.score[row_base + j0 + i] = j0 + i == n_old ? add : p.gamma * before + add;
        };
        const int i0 = warp * kTile + lane;  // below the weights' room, whatever cnt is
        float add[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) add[k] = mass(i0 + k * kThreads < cnt ? i0 + k * kThreads : i0);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) update(i0 + k * kThreads, old[k], add[k]);
        for (int i = i0 + kAhead * kThreads; i < cnt; i += kThreads) update(i, p.score[row_base + j0 + i], mass(i));
    }
    if (rank == 0 && tid == 0) p.len[ui.cache_unit] = n;
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

// How many clusters of S CTAs with `smem` bytes each fit the GPU at once.
template <typename K>
cudaError_t resident_clusters(int S, size_t smem, int *n) {
    *n = 0;
    const cudaError_t set = configure<K>();
    if (set != cudaSuccess) return set;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)S, 1024, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)S;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaOccupancyMaxActiveClusters(n, K::of(S), &cfg);
    if (err == cudaSuccess) return err;
    cudaGetLastError();
    *n = 0;
    return err == cudaErrorInvalidClusterSize ? cudaSuccess : err;  // such clusters do not fit
}

cudaError_t plan(const voxzip_cache_desc &d, int units, int nmax, Plan *best) {
    const q4::Shape shape{d.head_dim, d.dtype == VOXZIP_F32, d.q_heads / d.kv_heads > 8};
    return q4::choose_plan(
        shape, sm_count(), units, nmax,
        [&](int cap, int S, int stages) {
            return by_shape(d, [&](auto k) { return decltype(k)::Lay::bytes(cap, S, stages); });
        },
        [&](int S, size_t smem, int *n) {
            return by_shape(d, [&](auto k) { return resident_clusters<decltype(k)>(S, smem, n); });
        },
        best);
}

}  // namespace

cudaError_t launch_decode_q4(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                             const void *q, const void *k_new, const void *v_new, const int32_t *new_pos, float *score,
                             int32_t *pos, int32_t *len, float gamma, float sm_scale, int32_t max_len, void *out,
                             int32_t *status, cudaStream_t stream) {
    const int nmax = (max_len > 0 && max_len < d.capacity) ? max_len : d.capacity;
    const int units = layer_count * d.batch * d.kv_heads;
    // Plans are kept per device and shape (lengths in tiles).
    struct Entry {
        int device, dim, dtype, two, units, tiles;
        Plan plan;
    };
    thread_local Entry cache[16];
    thread_local int cache_next = 0;
    const int G = d.q_heads / d.kv_heads, tiles = (nmax - 1) / kTile + 1;
    int device = 0;
    const cudaError_t got = cudaGetDevice(&device);
    if (got != cudaSuccess) return got;
    Plan pl{0, 0, 0, 0};
    bool found = false;
    for (const Entry &e : cache)
        if (e.tiles == tiles && e.units == units && e.device == device && e.dim == d.head_dim && e.dtype == d.dtype && e.two == (G > 8)) {
            pl = e.plan;
            found = true;
        }
    if (!found) {
        const cudaError_t err = plan(d, units, nmax, &pl);
        if (err != cudaSuccess) return err;  // (no plan is kept)
        cache[cache_next] = Entry{device, d.head_dim, d.dtype, G > 8, units, tiles, pl};
        cache_next = (cache_next + 1) % 16;
    }
    const int S = pl.S;
    if (S == 0 || d.batch > 65535 || layer_count > 65535)  // more rows than a cluster holds the logits of, or than a grid's extent
        return launch_decode_q4_rows(d, q4, layer_begin, layer_count, q, k_new, v_new, new_pos, score, pos, len, gamma,
                                     sm_scale, max_len, out, status, stream);
    const int slice = max(2, (G * d.head_dim / 4 + S - 1) / S);
    auto inverse = [](int x) { return x <= 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + x - 1) / x); };
    const float scale = sm_scale > 0.f ? sm_scale : 1.0f / sqrtf((float)d.head_dim);
    const int resident = pl.resident;
    const bool later = resident > 0 && resident < units;
    const MmaQ4Params prm{q4, q, k_new, v_new, new_pos, score, pos, len, out, status, d.batch, d.layers, d.q_heads,
                          d.kv_heads, G, d.capacity, layer_begin, pl.chunk_cap, nmax, S, pl.stages, slice,
                          later ? resident % d.kv_heads : 0, later ? resident / d.kv_heads % d.batch : 0,
                          later ? resident / d.kv_heads / d.batch : -1, inverse(S), inverse(slice), gamma,
                          scale * 1.4426950408889634f * kUncarry};
    return by_shape(d, [&](auto k) {
        using K = decltype(k);
        const cudaError_t set = configure<K>();
        if (set != cudaSuccess) return set;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(d.kv_heads * S), (unsigned)d.batch, (unsigned)layer_count);
        cfg.blockDim = dim3(kThreads, 1, 1);
        cfg.dynamicSmemBytes = K::Lay::bytes(pl.chunk_cap, S, pl.stages);
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
