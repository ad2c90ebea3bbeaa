// Budgeted eviction from a cache held in 4 bits (format: q4.cuh): the policies of voxzip_evict_ex.
//
// One CTA per unit. Selection: MSB-first radix selects (passes of 8 bits over order-preserving 32-bit keys, the scores,
// and to fill holes the positions, held in shared memory) give the N-th best history score and, where that score is
// tied and not all tied rows fit, the position up to which its rows stay. Compaction: the kept rows are listed in shared
// memory, a segment at a time, and go through a cp.async ring in batches. A batch is stored when all of it has
// landed: in the ordered compaction a destination may be a source of the same batch, never of a later one (a row's
// destination is its rank among the kept rows, which no source of a higher rank lies below); when holes are filled,
// sources lie at or above the budget and destinations below it.
//
// The ordered compaction moves nearly every row (the first to leave is early) and is bound by memory, as far as three
// CTAs per SM keep it busy: 768 units of 2 333 rows down to 2 301 take 107 us (0.73 of the measured copy rate), 192 units
// of 11 554 to 11 522 163 us (0.60: 192 CTAs on 152 SMs). Hole filling moves 32 rows of those and is bound by the
// selection's passes: 39 and 62 us. 192 units of 189 rows to 157: 8 us.
// The room for scores and positions goes by the capacity, which the host knows: hole filling takes 96 us for the 768 units
// in a capacity of 20 480 (one CTA per SM), and 99 for the 192 in one of 47 048, where they are read where they lie.
#include <type_traits>

#include "q4.cuh"

namespace voxzip {
namespace {

constexpr int kNT = 256;           // threads of a CTA
constexpr int kSegment = 1024;   // pairs listed at a time
// Shared memory that may hold a unit's scores (and, to fill holes, its positions) while it selects, in the ring's
// place; those of longer units are read where they lie.
constexpr int kHeldBytes = 160 * 1024;

struct EvictQ4Params {
    Q4View q4;
    float *score;
    int32_t *pos, *len;
    const int32_t *budget;
    int32_t *status;
    int32_t B, L, Hkv, C, layer_begin, sink;
    int32_t held_rows;  // what the launch's shared memory holds
    int32_t budget_stride_b, budget_stride_l, history;
    float recent_frac;
};

__device__ __forceinline__ uint32_t score_order(float s) {  // uint32 order of fp32 values
    const uint32_t b = __float_as_uint(s);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int NT>
struct Scratch {
    uint32_t hist[256];
    int warp_sums[NT / 32];
    uint32_t prefix;
    int rank, ties;
};

// Exclusive sums of a count per thread, in thread order; `total` their sum.
template <int NT>
__device__ __forceinline__ int block_sum(int count, int &total, Scratch<NT> &s) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int upto = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
    }
    __syncthreads();  // the sums of the call before are read
    if (lane == 31) s.warp_sums[warp] = upto;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        before += w < warp ? s.warp_sums[w] : 0;
        total += s.warp_sums[w];
    }
    return before + upto - count;
}

struct Cut {
    uint32_t key;  // the rank-th smallest key
    int left;      // how many keys equal to it are among the first `rank`
    int ties;      // how many there are
};

// The rank-th smallest (from 1) key over the j in [lo, hi) for which key_of(j, key) is true. rank is at most
// their number, and no key has a bit above the digit at top_shift.
template <int NT, typename KeyOf>
__device__ Cut select_kth(int lo, int hi, int rank, KeyOf key_of, Scratch<NT> &s, int top_shift = 24) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0u;
    int ties = 0;
    for (int shift = top_shift; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = tid; i < 256; i += NT) s.hist[i] = 0u;
        __syncthreads();
        const uint32_t above = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
        if (shift == 24) {
            // Scores share their highest digit: the first lane's bin is counted for its whole warp at once (an add
            // per lane to the same bin would go one after another).
            for (int j0 = lo; j0 < hi; j0 += NT) {
                const int j = j0 + tid;
                uint32_t key = 0u;
                const bool counts = j < hi && key_of(j, key);
                const uint32_t bin = key >> 24, voters = __ballot_sync(0xffffffffu, counts);
                if (voters == 0u) continue;
                const int first = __ffs(voters) - 1;
                const uint32_t common = __shfl_sync(0xffffffffu, bin, first);
                const uint32_t same = __ballot_sync(0xffffffffu, counts && bin == common);
                if ((tid & 31) == first) atomicAdd(&s.hist[common], (uint32_t)__popc(same));
                else if (counts && bin != common) atomicAdd(&s.hist[bin], 1u);
            }
        } else {
            for (int j = lo + tid; j < hi; j += NT) {
                uint32_t key;
                if (key_of(j, key) && (key & above) == prefix) atomicAdd(&s.hist[key >> shift & 255u], 1u);
            }
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

// The compaction's ring: kDepth batches of rows, each thread its own vectors (codes) and small pieces (two scales,
// score, position of a row).
template <int D, int NT, bool kFill>
struct Ring {
    static constexpr int VPR = D / 32;  // 16-byte vectors of a row's K (or V) codes
    static constexpr int kVecs = kFill ? 2 : 4;  // of them per thread and batch
    static constexpr int kBatch = NT * kVecs / (2 * VPR);
    static constexpr int kSmall = kBatch * 4 / NT;
    static constexpr int kDepth = kFill ? 2 : 3;
    static constexpr int kStageBytes = NT * (kVecs * 16 + kSmall * 8);
    static constexpr int kBytes = kDepth * kStageBytes;
};

template <int kBytes>
__device__ __forceinline__ void copy_async(void *dst, const void *src) {
    if constexpr (kBytes == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(dst)), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(ptx::smem_u32(dst)), "l"(src), "n"(kBytes) : "memory");
}

template <int D, int NT, bool kFill>
__global__ void __launch_bounds__(NT, 1024 / NT) evict_q4_kernel(const EvictQ4Params p) {
    using R = Ring<D, NT, kFill>;
    constexpr int VPR = R::VPR, kVecs = R::kVecs, kBatch = R::kBatch, kSmall = R::kSmall, kDepth = R::kDepth;
    using Scale = std::conditional_t<D == 128, uint2, uint32_t>;
    __shared__ Scratch<NT> scratch;
    __shared__ int32_t src_list[kSegment + 4 * NT], dst_list[kFill ? kSegment : 1];
    extern __shared__ __align__(16) uint8_t ring[];
    float *held = reinterpret_cast<float *>(ring);
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
    // The selection reads every score (and, to fill holes, every position) several times.
    const float *scores = sc;
    const int32_t *places = ps;
    if (n <= p.held_rows) {
        int32_t *held_ps = reinterpret_cast<int32_t *>(held + p.held_rows);
        for (int j = tid; j < n; j += NT) {
            held[j] = sc[j];
            if constexpr (kFill) held_ps[j] = ps[j];
        }
        scores = held;
        if constexpr (kFill) places = held_ps;
        __syncthreads();
    }

    // The rows that stay whatever their score: by slot, or (the cache not being in time order) by position.
    uint32_t p_lo = 0u, p_hi = 0xffffffffu;
    int pos_shift = 24;  // of the highest digit that any position sets
    if constexpr (kFill) {
        uint32_t any = 0u;
        for (int j = tid; j < n; j += NT) any |= (uint32_t)places[j];
        any = __reduce_or_sync(0xffffffffu, any);
        if ((tid & 31) == 0) scratch.warp_sums[tid >> 5] = (int)any;
        __syncthreads();
        any = 0u;
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) any |= (uint32_t)scratch.warp_sums[w];
        pos_shift = any >> 24 ? 24 : any >> 16 ? 16 : any >> 8 ? 8 : 0;
        auto pos_key = [&](int j, uint32_t &key) {
            key = (uint32_t)places[j];
            return true;
        };
        if (T > 0) p_lo = select_kth<NT>(0, n, T, pos_key, scratch, pos_shift).key;
        if (M > 0) p_hi = select_kth<NT>(0, n, n - M + 1, pos_key, scratch, pos_shift).key;
    }
    auto history = [&](int j) {
        if constexpr (!kFill) return j >= T && j < n - M;
        const uint32_t q = (uint32_t)places[j];
        return !(T > 0 && q <= p_lo) && !(M > 0 && q >= p_hi);
    };
    // Eq. 9: the N best of the history; keys ascend as scores descend.
    uint32_t thr = 0u, pos_thr = 0xffffffffu;
    if (N > 0) {
        const Cut cut = select_kth<NT>(0, n, N, [&](int j, uint32_t &key) {
            key = ~score_order(scores[j]);
            return history(j);
        }, scratch);
        thr = cut.key;
        if (cut.left < cut.ties)
            pos_thr = select_kth<NT>(0, n, cut.left, [&](int j, uint32_t &key) {
                key = (uint32_t)places[j];
                return history(j) && ~score_order(scores[j]) == thr;
            }, scratch, pos_shift).key;
    }
    auto kept = [&](int j) {
        if (!history(j)) return true;
        if (N == 0) return false;
        const uint32_t key = ~score_order(sc[j]);
        return key < thr || (key == thr && (uint32_t)ps[j] <= pos_thr);
    };

    // Rows src_list[i] go to dst(i), by way of the ring: a batch is stored when all of it has landed, with the next
    // ones on their way.
    auto move = [&](int rows, auto dst) {
        auto moves = [&](int r) {
            return r < rows && src_list[r] != dst(r) && VOXZIP_IN_RANGE(p.status, src_list[r] >= 0 && src_list[r] < n && dst(r) >= 0 && dst(r) < bud);
        };
        auto vec_of = [&](uint8_t *stage, int k) { return reinterpret_cast<uint4 *>(stage) + k * NT + tid; };
        auto small_of = [&](uint8_t *stage, int k) { return reinterpret_cast<uint2 *>(stage + NT * kVecs * 16) + k * NT + tid; };
        auto load = [&](int batch) {
            uint8_t *stage = ring + batch % kDepth * R::kStageBytes;
            const int r0 = batch * kBatch;
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const int v = tid + k * NT, r = r0 + v / (2 * VPR), w = v % (2 * VPR);
                if (moves(r))
                    copy_async<16>(vec_of(stage, k), (w < VPR ? p.q4.k_codes : p.q4.v_codes) + ((base + src_list[r]) * VPR + w % VPR) * 16);
            }
#pragma unroll
            for (int k = 0; k < kSmall; ++k) {
                const int v = tid + k * NT, r = r0 + v % kBatch, w = v / kBatch;
                if (moves(r)) {
                    const int64_t at = base + src_list[r];
                    if (w < 2) copy_async<sizeof(Scale)>(small_of(stage, k), reinterpret_cast<const Scale *>(w == 0 ? p.q4.k_scale : p.q4.v_scale) + at);
                    else copy_async<4>(small_of(stage, k), w == 2 ? reinterpret_cast<const int32_t *>(p.score) + at : p.pos + at);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        auto store = [&](int batch) {
            uint8_t *stage = ring + batch % kDepth * R::kStageBytes;
            const int r0 = batch * kBatch;
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const int v = tid + k * NT, r = r0 + v / (2 * VPR), w = v % (2 * VPR);
                if (moves(r))
                    reinterpret_cast<uint4 *>(w < VPR ? p.q4.k_codes : p.q4.v_codes)[(base + dst(r)) * VPR + w % VPR] = *vec_of(stage, k);
            }
#pragma unroll
            for (int k = 0; k < kSmall; ++k) {
                const int v = tid + k * NT, r = r0 + v % kBatch, w = v / kBatch;
                if (moves(r)) {
                    const int64_t at = base + dst(r);
                    const uint2 x = *small_of(stage, k);
                    if (w < 2) {
                        Scale *to = reinterpret_cast<Scale *>(w == 0 ? p.q4.k_scale : p.q4.v_scale) + at;
                        if constexpr (D == 128) *to = x;
                        else *to = x.x;
                    } else if (w == 2) {
                        p.score[at] = __uint_as_float(x.x);
                    } else {
                        p.pos[at] = (int32_t)x.x;
                    }
                }
            }
        };
        const int batches = (rows + kBatch - 1) / kBatch;
#pragma unroll
        for (int i = 0; i < kDepth - 1; ++i) load(i);
        for (int i = 0; i < batches; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 2) : "memory");
            __syncthreads();  // the batch has landed, everybody's: none of its sources is read again
            store(i);
            load(i + kDepth - 1);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    };
    scores = sc;  // the ring takes the held scores' place
    places = ps;
    __syncthreads();

    if constexpr (!kFill) {
        // Four slots per thread at a time: kept rows are listed by rank, those before the first evicted slot too
        // (they stay: their rank is their slot).
        int rank0 = 0;
        for (int cursor = 0; cursor < n;) {
            int listed = 0;
            while (cursor < n && listed < kSegment) {
                const int j0 = cursor + 4 * tid;
                uint32_t flags = 0u;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j0 + k < n && kept(j0 + k)) flags |= 1u << k;
                int total;
                int at = listed + block_sum(__popc(flags), total, scratch);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (flags >> k & 1u) src_list[at++] = j0 + k;
                listed += total;
                cursor += 4 * NT;
            }
            __syncthreads();
            // Later slots are classified by their own scores and positions, which lie above every destination so far.
            move(listed, [&](int r) { return rank0 + r; });
            rank0 += listed;
            __syncthreads();
        }
        if (tid == 0) p.len[ui.cache_unit] = rank0;
    } else {
        int hcur = 0, mcur = bud, spare = 0;  // movers found beyond the holes so far
        bool unequal = false;
        while (true) {
            int nh = 0;
            while (hcur < bud && nh + NT <= kSegment) {
                const int j = hcur + tid;
                const bool hole = j < bud && !kept(j);
                int total;
                const int r = block_sum(hole, total, scratch);
                if (hole) dst_list[nh + r] = j;
                nh += total;
                hcur += NT;
            }
            while (spare < nh && mcur < n) {
                const int j = mcur + tid;
                const bool mover = j < n && kept(j);
                int total;
                const int r = block_sum(mover, total, scratch);
                if (mover) src_list[spare + r] = j;
                spare += total;
                mcur += NT;
            }
            __syncthreads();
            const int pairs = min(nh, spare);
            unequal = unequal || pairs < nh;
            move(pairs, [&](int r) { return dst_list[min(r, kSegment - 1)]; });
            __syncthreads();
            const int left = spare - pairs;  // below NT
            const int keep = tid < left ? src_list[pairs + tid] : 0;
            __syncthreads();
            if (tid < left) src_list[tid] = keep;
            spare = left;
            if (hcur >= bud) break;
        }
        // A kept row left over, or a hole, means that the unit's positions were not unique.
        int extra = spare > 0 || unequal;
        for (int j = mcur + tid; j < n; j += NT) extra |= kept(j) ? 1 : 0;
        if (__syncthreads_or(extra) && tid == 0) raise_status(p.status, VOXZIP_DEV_BAD_POSITIONS);
        if (tid == 0) p.len[ui.cache_unit] = bud;
    }
}

template <int D, bool kFill>
cudaError_t launch_t(EvictQ4Params prm, unsigned units, cudaStream_t stream) {
    using R = Ring<D, kNT, kFill>;
    void (*kern)(EvictQ4Params) = evict_q4_kernel<D, kNT, kFill>;
    static std::atomic<uint64_t> done{0};
    const cudaError_t set = once_per_device(done, [&] {
        return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, max(kHeldBytes, R::kBytes));
    });
    if (set != cudaSuccess) return set;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(units, 1, 1);
    cfg.blockDim = dim3(kNT, 1, 1);
    constexpr int kRowBytes = kFill ? 8 : 4;
    const int64_t held = (int64_t)((prm.C + 3) & ~3) * kRowBytes;
    cfg.dynamicSmemBytes = held <= kHeldBytes && held > R::kBytes ? (size_t)held : R::kBytes;
    prm.held_rows = (int32_t)(cfg.dynamicSmemBytes / kRowBytes);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // the kernel waits before its first read
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t err = cudaLaunchKernelEx(&cfg, kern, prm);
    if (err == cudaErrorNotSupported || err == cudaErrorInvalidValue) {  // no programmatic launch here
        cudaGetLastError();
        cfg.numAttrs = 0;
        err = cudaLaunchKernelEx(&cfg, kern, prm);
    }
    return err;
}

}  // namespace

cudaError_t launch_evict_q4(const voxzip_cache_desc &d, const Q4View &q4, int32_t layer_begin, int32_t layer_count,
                            float *score, int32_t *pos, int32_t *len, const int32_t *budget,
                            const voxzip_evict_policy &pol, int32_t *status, cudaStream_t stream) {
    const EvictQ4Params prm{q4, score, pos, len, budget, status, d.batch, d.layers, d.kv_heads, d.capacity, layer_begin,
                            pol.sink, 0, pol.budget_stride_b, pol.budget_stride_l, pol.history, pol.recent_frac};
    const unsigned units = (unsigned)(layer_count * d.batch * d.kv_heads);
    const bool fill = pol.compaction == VOXZIP_COMPACT_FILL;
    auto by_dim = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        return fill ? launch_t<D, true>(prm, units, stream) : launch_t<D, false>(prm, units, stream);
    };
    return d.head_dim == 128 ? by_dim(std::integral_constant<int, 128>{}) : by_dim(std::integral_constant<int, 64>{});
}

}  // namespace voxzip
