// Budgeted eviction from a cache held in 4 bits (format: q4.cuh): the policies of voxzip_evict_ex.
//
// One CTA per unit. Selection: MSB-first radix selects (four passes of 8 bits over order-preserving 32-bit keys)
// give the N-th best history score and, where that score is tied and not all tied rows fit, the position up to
// which its rows stay. Compaction: the kept rows that move are listed in shared memory, a segment at a time, and
// go through registers a batch of rows at a time. A batch is loaded whole before any of it is stored: in the
// ordered compaction a destination may be a source of the same batch, never of a later one (a row's destination
// is its rank among the kept rows, which no source of a higher rank lies below); when holes are filled, sources
// lie at or above the budget and destinations below it.
#include "q4.cuh"

namespace voxzip {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kSegment = 1024;  // pairs listed at a time

struct EvictQ4Params {
    Q4View q4;
    float *score;
    int32_t *pos, *len;
    const int32_t *budget;
    int32_t *status;
    int32_t B, L, Hkv, C, layer_begin, sink;
    int32_t budget_stride_b, budget_stride_l, history;
    float recent_frac;
};

__device__ __forceinline__ uint32_t score_order(float s) {  // uint32 order of fp32 values
    const uint32_t b = __float_as_uint(s);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct Scratch {
    uint32_t hist[256];
    int warp_sums[kWarps];
    uint32_t prefix;
    int rank, ties;
};

// Ranks of the set flags of a block, in thread order; `total` their number.
__device__ __forceinline__ int block_rank(bool flag, int &total, Scratch &s) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t votes = __ballot_sync(0xffffffffu, flag);
    __syncthreads();  // the sums of the call before are read
    if (lane == 0) s.warp_sums[warp] = __popc(votes);
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        before += w < warp ? s.warp_sums[w] : 0;
        total += s.warp_sums[w];
    }
    return before + __popc(votes & ((1u << lane) - 1u));
}

struct Cut {
    uint32_t key;  // the rank-th smallest key
    int left;      // how many keys equal to it are among the first `rank`
    int ties;      // how many there are
};

// The rank-th smallest (from 1) key over the j in [lo, hi) for which key_of(j, key) is true. rank is at most
// their number.
template <typename KeyOf>
__device__ Cut select_kth(int lo, int hi, int rank, KeyOf key_of, Scratch &s) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0u;
    int ties = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        s.hist[tid] = 0u;
        __syncthreads();
        const uint32_t above = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
        for (int j = lo + tid; j < hi; j += kThreads) {
            uint32_t key;
            if (key_of(j, key) && (key & above) == prefix) atomicAdd(&s.hist[key >> shift & 255u], 1u);
        }
        __syncthreads();
        if (tid < 32) {  // lane l holds bins 8 l .. 8 l + 7
            int c[8], sum = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += c[k] = (int)s.hist[tid * 8 + k];
            int upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, upto, o);
                if (tid >= o) upto += y;
            }
            int before = upto - sum;
            if (before < rank && rank <= upto) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (before < rank && rank <= before + c[k]) {
                        s.prefix = prefix | (uint32_t)(tid * 8 + k) << shift;
                        s.rank = rank - before;
                        s.ties = c[k];
                    }
                    before += c[k];
                }
            }
        }
        __syncthreads();
        prefix = s.prefix;
        rank = s.rank;
        ties = s.ties;
    }
    return Cut{prefix, rank, ties};
}

template <int D, bool kFill>
__global__ void __launch_bounds__(kThreads) evict_q4_kernel(const EvictQ4Params p) {
    constexpr int VPR = D / 32;  // 16-byte vectors of a row's K (or V) codes
    constexpr int kVecs = 4;     // of them per thread and batch
    constexpr int kBatch = kThreads * kVecs / (2 * VPR);
    constexpr int kSmall = kBatch * 4 / kThreads;  // K scales, V scales, score, position of a row
    using Scale = std::conditional_t<D == 128, uint2, uint32_t>;
    __shared__ Scratch scratch;
    __shared__ int32_t src_list[kSegment + kThreads], dst_list[kSegment];
    const int tid = threadIdx.x;
    const UnitIdx ui = unit_of(blockIdx.x, p.B, p.L, p.Hkv, p.layer_begin);
    ptx::grid_dependency_wait();
    const int32_t n = p.len[ui.cache_unit];
    const int32_t bud = p.budget[(int64_t)ui.b * p.budget_stride_b + (int64_t)ui.l * p.budget_stride_l];
    const int32_t T = p.sink;
    const int32_t M = p.history ? (int32_t)floor((double)p.recent_frac * (double)bud) : bud - T;
    const int32_t N = bud - T - M;
    if (bud < 0 || N < 0 || M < 0) {
        if (tid == 0) raise_status(p.status, VOXZIP_DEV_BAD_BUDGET);
        return;
    }
    if (n <= bud) return;
    if (n > p.C) {
        if (tid == 0) raise_status(p.status, VOXZIP_DEV_CAPACITY);
        return;
    }
    if (tid == 0) scratch.prefix = 0u, scratch.rank = 1, scratch.ties = 0;  // what a select that finds no key returns
    const int64_t base = ui.cache_unit * p.C;
    float *sc = p.score + base;
    int32_t *ps = p.pos + base;

    // The rows that stay whatever their score: by slot, or (the cache not being in time order) by position.
    uint32_t p_lo = 0u, p_hi = 0xffffffffu;
    auto pos_key = [&](int j, uint32_t &key) {
        key = (uint32_t)ps[j];
        return true;
    };
    if constexpr (kFill) {
        if (T > 0) p_lo = select_kth(0, n, T, pos_key, scratch).key;
        if (M > 0) p_hi = select_kth(0, n, n - M + 1, pos_key, scratch).key;
    }
    auto history = [&](int j) {
        if constexpr (!kFill) return j >= T && j < n - M;
        const uint32_t q = (uint32_t)ps[j];
        return !(T > 0 && q <= p_lo) && !(M > 0 && q >= p_hi);
    };
    // Eq. 9: the N best of the history; keys ascend as scores descend.
    uint32_t thr = 0u, pos_thr = 0xffffffffu;
    if (N > 0) {
        const Cut cut = select_kth(0, n, N, [&](int j, uint32_t &key) {
            key = ~score_order(sc[j]);
            return history(j);
        }, scratch);
        thr = cut.key;
        if (cut.left < cut.ties)
            pos_thr = select_kth(0, n, cut.left, [&](int j, uint32_t &key) {
                key = (uint32_t)ps[j];
                return history(j) && ~score_order(sc[j]) == thr;
            }, scratch).key;
    }
    auto kept = [&](int j) {
        if (!history(j)) return true;
        if (N == 0) return false;
        const uint32_t key = ~score_order(sc[j]);
        return key < thr || (key == thr && (uint32_t)ps[j] <= pos_thr);
    };

    auto move = [&](int rows) {  // src_list[i] to dst_list[i]
        for (int r0 = 0; r0 < rows; r0 += kBatch) {
            uint4 x[kVecs];
            uint64_t y[kSmall];
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const int v = tid + k * kThreads, r = r0 + v / (2 * VPR), w = v % (2 * VPR);
                if (r < rows && VOXZIP_IN_RANGE(p.status, src_list[r] >= 0 && src_list[r] < n)) {
                    const int64_t at = (base + src_list[r]) * VPR + w % VPR;
                    x[k] = reinterpret_cast<const uint4 *>(w < VPR ? p.q4.k_codes : p.q4.v_codes)[at];
                }
            }
#pragma unroll
            for (int k = 0; k < kSmall; ++k) {
                const int v = tid + k * kThreads, r = r0 + v % kBatch, w = v / kBatch;
                if (r < rows && VOXZIP_IN_RANGE(p.status, src_list[r] >= 0 && src_list[r] < n)) {
                    const int64_t at = base + src_list[r];
                    if (w < 2) {
                        const Scale s = reinterpret_cast<const Scale *>(w == 0 ? p.q4.k_scale : p.q4.v_scale)[at];
                        memcpy(&y[k], &s, sizeof(s));
                    } else {
                        y[k] = w == 2 ? __float_as_uint(p.score[at]) : (uint32_t)p.pos[at];
                    }
                }
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const int v = tid + k * kThreads, r = r0 + v / (2 * VPR), w = v % (2 * VPR);
                if (r < rows && VOXZIP_IN_RANGE(p.status, dst_list[r] >= 0 && dst_list[r] < bud)) {
                    const int64_t at = (base + dst_list[r]) * VPR + w % VPR;
                    reinterpret_cast<uint4 *>(w < VPR ? p.q4.k_codes : p.q4.v_codes)[at] = x[k];
                }
            }
#pragma unroll
            for (int k = 0; k < kSmall; ++k) {
                const int v = tid + k * kThreads, r = r0 + v % kBatch, w = v / kBatch;
                if (r < rows && VOXZIP_IN_RANGE(p.status, dst_list[r] >= 0 && dst_list[r] < bud)) {
                    const int64_t at = base + dst_list[r];
                    if (w < 2) {
                        Scale s;
                        memcpy(&s, &y[k], sizeof(s));
                        reinterpret_cast<Scale *>(w == 0 ? p.q4.k_scale : p.q4.v_scale)[at] = s;
                    } else if (w == 2) {
                        p.score[at] = __uint_as_float((uint32_t)y[k]);
                    } else {
                        p.pos[at] = (int32_t)y[k];
                    }
                }
            }
        }
    };

    if constexpr (!kFill) {
        int rank0 = 0;
        for (int cursor = 0; cursor < n;) {
            int listed = 0;
            while (cursor < n && listed + kThreads <= kSegment) {
                const int j = cursor + tid;
                const bool keep = j < n && kept(j);
                int total;
                const int r = block_rank(keep, total, scratch);
                // rows before the first evicted slot stay where they are
                const bool moves = keep && j != rank0 + r;
                int moving;
                const int at = block_rank(moves, moving, scratch);
                if (moves) {
                    src_list[listed + at] = j;
                    dst_list[listed + at] = rank0 + r;
                }
                listed += moving;
                rank0 += total;
                cursor += kThreads;
            }
            __syncthreads();
            // Later slots are classified by their own scores, which lie above every destination so far.
            move(listed);
            __syncthreads();
        }
        if (tid == 0) p.len[ui.cache_unit] = rank0;
    } else {
        int hcur = 0, mcur = bud, spare = 0;  // movers found beyond the holes so far
        bool unequal = false;
        while (true) {
            int nh = 0;
            while (hcur < bud && nh + kThreads <= kSegment) {
                const int j = hcur + tid;
                const bool hole = j < bud && !kept(j);
                int total;
                const int r = block_rank(hole, total, scratch);
                if (hole) dst_list[nh + r] = j;
                nh += total;
                hcur += kThreads;
            }
            while (spare < nh && mcur < n) {
                const int j = mcur + tid;
                const bool mover = j < n && kept(j);
                int total;
                const int r = block_rank(mover, total, scratch);
                if (mover) src_list[spare + r] = j;
                spare += total;
                mcur += kThreads;
            }
            __syncthreads();
            const int pairs = min(nh, spare);
            unequal = unequal || pairs < nh;
            move(pairs);
            __syncthreads();
            const int left = spare - pairs;  // below kThreads
            const int keep = tid < left ? src_list[pairs + tid] : 0;
            __syncthreads();
            if (tid < left) src_list[tid] = keep;
            spare = left;
            if (hcur >= bud) break;
        }
        // A kept row left over, or a hole, means that the unit's positions were not unique.
        int extra = spare > 0 || unequal;
        for (int j = mcur + tid; j < n; j += kThreads) extra |= kept(j) ? 1 : 0;
        if (__syncthreads_or(extra) && tid == 0) raise_status(p.status, VOXZIP_DEV_BAD_POSITIONS);
        if (tid == 0) p.len[ui.cache_unit] = bud;
    }
}

}  // namespace

cudaError_t launch_evict_q4(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                            float *score, int32_t *pos, int32_t *len, const int32_t *budget,
                            const voxzip_evict_policy &pol, int32_t *status, cudaStream_t stream) {
    const EvictQ4Params prm{q4, score, pos, len, budget, status, d.batch, d.layers, d.kv_heads, d.capacity, layer_begin,
                            pol.sink, pol.budget_stride_b, pol.budget_stride_l, pol.history, pol.recent_frac};
    const unsigned units = (unsigned)(layer_count * d.batch * d.kv_heads);
    const bool fill = pol.compaction == VOXZIP_COMPACT_FILL;
    if (d.head_dim == 128) {
        if (fill) evict_q4_kernel<128, true><<<units, kThreads, 0, stream>>>(prm);
        else evict_q4_kernel<128, false><<<units, kThreads, 0, stream>>>(prm);
    } else {
        if (fill) evict_q4_kernel<64, true><<<units, kThreads, 0, stream>>>(prm);
        else evict_q4_kernel<64, false><<<units, kThreads, 0, stream>>>(prm);
    }
    return cudaGetLastError();
}

}  // namespace voxzip
