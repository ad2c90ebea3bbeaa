// Rotary positions and the append of a prompt's rows.
//
//   th = position[axis_i] freq_i;   lo' = lo cos th - hi sin th,   hi' = hi cos th + lo sin th
//
// of pairs i < R / 2 of a head's first R channels, in fp32 and rounded once. A warp takes a token of a layer: it
// computes the token's angles once (each lane two of them) for all heads, and streams the heads' rows past them, q to
// q_out, k and v to the cache rows behind the unit's own. Bound by memory: each row is read and written once.
#include <algorithm>

#include "evict_policy.cuh"  // sm_count
#include "prompt.cuh"
#include "ptx.cuh"

namespace voxzip {
namespace {

constexpr int kWarps = 4;

struct RowsParams {
    RotaryTable rot;  // rot.half = 0: rows as they are
    RowsView q, k, v;
    void *q_out, *k_out;  // k_out: rotated rows as they lie in k (no cache)
    const int32_t *positions;  // [axes][T]
    const int32_t *seq_off, *new_pos, *start;
    CacheRows cache;
    float *score;
    int32_t *pos, *status;
    int32_t T, B, L, Hq, Hkv, C, D;
    int32_t layer_begin, layer_count;
    int32_t heads;        // heads of a token: Hq (if q) + Hkv + Hkv (if a cache)
    int32_t warp_heads;   // heads that one warp takes
    int32_t chunks;       // warps per token
};

// sin and cos of a fraction of a turn, of which the upper 32 bits are kept. The nearest quarter-turn is taken off in
// integers, so the argument of the functions is small and rounded by 2^-28 of a turn at most.
__device__ __forceinline__ float2 turn_cos_sin(uint64_t turns) {
    const int32_t t = (int32_t)(turns >> 32);  // [-1/2, 1/2) turns
    const uint32_t quarter = ((uint32_t)t + (1u << 29)) >> 30;
    const int32_t rest = (int32_t)((uint32_t)t - (quarter << 30));  // [-1/8, 1/8) turns
    float s, c;
    sincospif((float)rest * 4.656612873077393e-10f, &s, &c);  // 2^-31: half-turns
    const float2 r0 = (quarter & 1) ? make_float2(-s, c) : make_float2(c, s);
    return (quarter & 2) ? make_float2(-r0.x, -r0.y) : r0;
}

template <typename T> struct Vec;  // 16 bytes of a row
template <> struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(const uint4 &u, float (&x)[4]) {
        x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(const uint4 &u, float (&x)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 put(const float (&x)[8]) {
        return make_uint4(ptx::pack_bf16(x[0], x[1]), ptx::pack_bf16(x[2], x[3]), ptx::pack_bf16(x[4], x[5]),
                          ptx::pack_bf16(x[6], x[7]));
    }
};

// The sequence that packed token t belongs to, -1 for none. All lanes of a warp; 32 candidates per round.
__device__ __forceinline__ int32_t sequence_of(const int32_t *off, int32_t B, int32_t t) {
    const int lane = threadIdx.x & 31;
    int32_t lo = 0, n = B + 1;  // the last entry at or below t is in [lo - 1, lo + n)
    while (n > 0) {
        const int32_t step = (n + 31) / 32, at = lo + lane * step;
        const int c = __popc(__ballot_sync(0xffffffffu, lane * step < n && off[min(at, B)] <= t));
        if (c == 0) break;
        const int32_t next = lo + (c - 1) * step + 1;
        n = min(lo + n, lo + c * step) - next;
        lo = next;
    }
    const int32_t b = lo - 1;
    return b >= 0 && b < B && off[b] >= 0 && off[b] <= t && t < off[b + 1] ? b : -1;
}

// A lane's part of its token's rows: two vectors, and the angles of their pairs. A warp has kLanes rows in hand at once.
template <typename T, int D> struct Part {
    using V = Vec<T>;
    static constexpr int kItems = D / V::N / 2;  // pairs of vectors in a row
    static constexpr int kLanes = 32 / kItems;
    int va, vb;  // in vectors
    bool rotated;
    float2 cs[V::N];

    __device__ __forceinline__ Part(const RotaryTable &rot, const float2 *angles) {
        const int j = (threadIdx.x & 31) % kItems, rot_items = rot.half / V::N;
        rotated = j < rot_items;
        va = rotated ? j : 2 * rot_items + 2 * (j - rot_items);
        vb = rotated ? j + rot_items : va + 1;
#pragma unroll
        for (int i = 0; i < V::N; ++i) {  // (of pairs side by side each vector has half as many)
            const int pair = !rot.adjacent ? j * V::N + i
                             : i < V::N / 2 ? va * (V::N / 2) + i
                                            : vb * (V::N / 2) + i - V::N / 2;
            cs[i] = rotated ? angles[pair] : make_float2(1.f, 0.f);
        }
    }
    __device__ __forceinline__ void rotate(bool adjacent, uint4 &a, uint4 &c) const {
        float x[V::N], y[V::N];
        V::get(a, x);
        V::get(c, y);
        if (!adjacent) {
#pragma unroll
            for (int i = 0; i < V::N; ++i) {
                const float lo = x[i], hi = y[i];
                x[i] = lo * cs[i].x - hi * cs[i].y;
                y[i] = hi * cs[i].x + lo * cs[i].y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V::N / 2; ++i) {
                float lo = x[2 * i], hi = x[2 * i + 1];
                const float2 u = cs[i], w = cs[V::N / 2 + i];
                x[2 * i] = lo * u.x - hi * u.y;
                x[2 * i + 1] = hi * u.x + lo * u.y;
                lo = y[2 * i], hi = y[2 * i + 1];
                y[2 * i] = lo * w.x - hi * w.y;
                y[2 * i + 1] = hi * w.x + lo * w.y;
            }
        }
        a = V::put(x);
        c = V::put(y);
    }
};

// The angles of token t, by a warp.
__device__ __forceinline__ void token_angles(const RowsParams &p, int32_t t, float2 *angles) {
    for (int i = threadIdx.x & 31; i < p.rot.half; i += 32)
        angles[i] = turn_cos_sin((uint64_t)(int64_t)p.positions[(int64_t)p.rot.axis[i] * p.T + t] * p.rot.turns[i]);
    __syncwarp();
}

// Where row `head` ([q heads][k heads][v heads]) of token t comes from and goes to; false for a unit that is skipped.
// start(h): the length before of the unit of kv-head h (kCache).
template <typename T, int D, bool kCache, typename S>
__device__ __forceinline__ bool locate(const RowsParams &p, int l, int32_t t, int32_t b, int32_t row, int head, int Hq,
                                       S start, const T *&from, T *&to, bool &turn) {
    const bool is_q = head < Hq, is_v = head >= Hq + p.Hkv;
    const int h = is_q ? head : is_v ? head - Hq - p.Hkv : head - Hq;
    const RowsView &src = is_q ? p.q : is_v ? p.v : p.k;
    from = static_cast<const T *>(src.data) + l * src.layer_stride + t * src.token_stride + (int64_t)h * D;
    turn = !is_v;
    if (is_q) {
        to = static_cast<T *>(p.q_out) + (((int64_t)l * p.T + t) * p.Hq + h) * D;
    } else if (!kCache) {
        to = static_cast<T *>(p.k_out) + (((int64_t)l * p.T + t) * p.Hkv + h) * D;
    } else {
        const int64_t cu = ((int64_t)b * p.L + p.layer_begin + l) * p.Hkv + h;
        const int32_t at = start(h);
        if (at < 0) return false;
        const int32_t slot = at + row;
        const int64_t r = p.cache.pv.table ? paged_row(p.cache.pv, cu, slot) : cu * p.C + slot;
        if (p.cache.pv.table && (r < 0 || r >= p.cache.pool_rows)) {  // a page that the pool does not have
            raise_status(p.status, VOXZIP_DEV_CAPACITY);
            return false;
        }
        if (!VOXZIP_IN_RANGE(p.status, slot < p.C && r >= 0 && r < p.cache.pool_rows)) return false;
        to = static_cast<T *>(is_v ? p.cache.v : p.cache.k) + r * D;
        if (!is_v && (threadIdx.x & 31) % Part<T, D>::kItems == 0) {
            if (p.score) p.score[cu * p.C + slot] = 0.f;
            if (p.pos) p.pos[cu * p.C + slot] = p.new_pos[t];
        }
    }
    return true;
}

// Rows head(0), head(1), ... below n of a token, kUnroll of them on their way at once.
template <typename T, int D, bool kCache, int kUnroll, typename S, typename F>
__device__ __forceinline__ void move_rows(const RowsParams &p, const Part<T, D> &part, int l, int32_t t, int32_t b,
                                          int32_t row, int Hq, S start, int n, F head) {
    const int sub = (threadIdx.x & 31) / Part<T, D>::kItems;
    for (int i0 = sub; i0 < n; i0 += kUnroll * Part<T, D>::kLanes) {
        uint4 a[kUnroll], c[kUnroll];
        T *to[kUnroll];
        bool turn[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int i = i0 + u * Part<T, D>::kLanes;
            const T *from = nullptr;
            to[u] = nullptr;
            turn[u] = false;
            if (i < n && locate<T, D, kCache>(p, l, t, b, row, head(i), Hq, start, from, to[u], turn[u])) {
                a[u] = reinterpret_cast<const uint4 *>(from)[part.va];
                c[u] = reinterpret_cast<const uint4 *>(from)[part.vb];
            } else {
                to[u] = nullptr;
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (to[u] == nullptr) continue;
            if (turn[u] && part.rotated) part.rotate(p.rot.adjacent, a[u], c[u]);
            reinterpret_cast<uint4 *>(to[u])[part.va] = a[u];
            reinterpret_cast<uint4 *>(to[u])[part.vb] = c[u];
        }
    }
}

template <typename T, int D, bool kCache>
__global__ void __launch_bounds__(32 * kWarps, 8) rows_kernel(const RowsParams p) {
    __shared__ float2 angles[kWarps][kMaxPairs];
    const int warp = threadIdx.x >> 5;
    const int64_t item = (int64_t)blockIdx.x * kWarps + warp;
    ptx::grid_dependency_wait();
    const int64_t total = (int64_t)p.layer_count * p.T * p.chunks;
    if (item >= total) return;
    const int chunk = (int)(item % p.chunks);
    const int32_t t = (int32_t)(item / p.chunks % p.T);
    const int l = (int)(item / p.chunks / p.T);
    int32_t b = 0, row = 0;
    if (kCache) {
        b = sequence_of(p.seq_off, p.B, t);
        if (b < 0) return;  // behind the last sequence: left as it is
        row = t - p.seq_off[b];
    }
    token_angles(p, t, angles[warp]);
    const Part<T, D> part(p.rot, angles[warp]);
    const int h0 = chunk * p.warp_heads;
    const int32_t *start = kCache ? p.start + ((int64_t)l * p.B + b) * p.Hkv : nullptr;
    move_rows<T, D, kCache, 2>(p, part, l, t, b, row, p.q.data ? p.Hq : 0, [=](int h) { return start[h]; },
                               min(p.heads, h0 + p.warp_heads) - h0, [=](int i) { return h0 + i; });
}

struct PlanParams {
    const int32_t *seq_off;
    PageView pv;
    int32_t *len, *start, *status;
    int32_t B, L, Hkv, C, T, layer_begin, units;
};

// Takes `want` pages off the free stack, all or none: the stack index of the first, or -1.
__device__ __forceinline__ int32_t take_pages(const PageView &pv, int32_t want) {
    int32_t have = *reinterpret_cast<volatile int32_t *>(pv.free_count);
    while (have >= want) {  // a failed exchange means that another unit took its pages: at most one per unit
        const int32_t was = atomicCAS(pv.free_count, have, have - want);
        if (was == have) return have - want;
        have = was;
    }
    return -1;
}

// What the page table holds, from the plan of an append to its last launch, where the unit's next slot wants a page. It is
// taken when all units have those of their rows, so that no unit goes without for another one's next slot.
constexpr int32_t kWantedPage = -2;

// A warp: whether unit ui takes its sequence's m rows behind its n, and the pages that they need. 0, or the error.
__device__ __forceinline__ uint32_t plan_unit(const PlanParams &p, int64_t cu, int32_t n, int32_t m) {
    const int lane = threadIdx.x & 31;
    if (n < 0 || n > p.C || m > p.C - n) return VOXZIP_DEV_CAPACITY;
    if (!p.pv.table || m == 0) return 0;
    // pages of slots [n, n + m) that the unit does not hold
    int32_t *table = p.pv.table + cu * p.pv.max_pages;
    const int32_t p0 = n / kPageTokens, p1 = (n + m - 1) / kPageTokens + 1;
    int32_t missing = 0;
    for (int32_t base = p0; base < p1; base += 32)
        missing += __popc(__ballot_sync(0xffffffffu, base + lane < p1 && table[base + lane] < 0));
    if (missing > 0) {
        int32_t at = lane == 0 ? take_pages(p.pv, missing) : 0;
        at = __shfl_sync(0xffffffffu, at, 0);
        if (at < 0) return VOXZIP_DEV_CAPACITY;
        int32_t done = 0;  // the highest stack entry first, as take_page does
        for (int32_t base = p0; base < p1; base += 32) {
            const bool none = base + lane < p1 && table[base + lane] < 0;
            const unsigned who = __ballot_sync(0xffffffffu, none);
            if (none) table[base + lane] = p.pv.free_pages[at + missing - 1 - done - __popc(who & ((1u << lane) - 1u))];
            done += __popc(who);
        }
    }
    if (lane == 0 && (n + m) % kPageTokens == 0 && p1 < p.pv.max_pages && table[p1] < 0) table[p1] = kWantedPage;
    return 0;
}

// A warp: whether the sequences' offsets are in order.
__device__ __forceinline__ bool offsets_ok(const int32_t *off, int32_t B, int32_t T) {
    bool bad = false;
    for (int32_t b = threadIdx.x & 31; b < B; b += 32) bad |= off[b] < 0 || off[b + 1] < off[b] || off[b + 1] > T;
    return !__any_sync(0xffffffffu, bad);
}

// A warp per unit: where its rows go (start, -1 where it is skipped), the pages that they need, and its new length.
__global__ void __launch_bounds__(128) append_plan_kernel(const PlanParams p) {
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    const int32_t u = blockIdx.x * 4 + (threadIdx.x >> 5);
    if (u >= p.units) return;
    const UnitIdx ui = unit_of(u, p.B, p.L, p.Hkv, p.layer_begin);
    const bool ok = offsets_ok(p.seq_off, p.B, p.T);
    const int32_t m = ok ? p.seq_off[ui.b + 1] - p.seq_off[ui.b] : 0;
    const int32_t n = p.len[ui.cache_unit];
    const uint32_t error = ok ? plan_unit(p, ui.cache_unit, n, m) : VOXZIP_DEV_BAD_SPANS;
    if ((threadIdx.x & 31) == 0) {
        if (error) raise_status(p.status, error);
        p.start[u] = error ? -1 : n;
        if (!error && m > 0) p.len[ui.cache_unit] = n + m;
    }
}

// A thread per unit, behind the rows: the pages of the next append's slots, as far as there are any.
__global__ void __launch_bounds__(128) append_next_page_kernel(const PlanParams p) {
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    const int32_t u = blockIdx.x * 128 + threadIdx.x;
    if (u >= p.units) return;
    const UnitIdx ui = unit_of(u, p.B, p.L, p.Hkv, p.layer_begin);
    const int32_t n = p.len[ui.cache_unit];
    if (n <= 0 || n % kPageTokens != 0 || n / kPageTokens >= p.pv.max_pages) return;
    int32_t *entry = p.pv.table + ui.cache_unit * p.pv.max_pages + n / kPageTokens;
    if (*entry != kWantedPage) return;
    const int32_t at = take_pages(p.pv, 1);  // (never below the count that an append beside this one reads)
    *entry = at >= 0 ? p.pv.free_pages[at] : -1;
}

// The same and the rows in one launch, for short sequences of few units: a cluster per unit has its k and v rows and its
// query heads', a token per warp. Its first CTA plans; the others read from its shared memory where the rows go.
constexpr int kUnitWarps = 8, kUnitCtas = 8;
template <typename T, int D>
__global__ void __launch_bounds__(32 * kUnitWarps) append_unit_kernel(const PlanParams pp, const RowsParams p, int ctas) {
    __shared__ float2 angles[kUnitWarps][kMaxPairs];
    __shared__ int32_t plan[2];  // the unit's length before (-1: it is skipped), its rows
    const int warp = threadIdx.x >> 5, rank = blockIdx.x % ctas;
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    const UnitIdx ui = unit_of(blockIdx.x / ctas, p.B, p.L, p.Hkv, p.layer_begin);
    const int32_t t0 = p.seq_off[ui.b], t1 = p.seq_off[ui.b + 1], first = rank * kUnitWarps + warp;
    // (the first token's angles while the plan is made; the offsets may be anything, their difference too)
    if (0 <= t0 && t0 <= t1 && t1 <= p.T && first < t1 - t0) token_angles(p, t0 + first, angles[warp]);
    if (rank == 0 && warp == 0) {
        const int32_t n = pp.len[ui.cache_unit];
        const bool ok = offsets_ok(p.seq_off, p.B, p.T);
        const int32_t m = ok ? t1 - t0 : 0;
        const uint32_t error = ok ? plan_unit(pp, ui.cache_unit, n, m) : VOXZIP_DEV_BAD_SPANS;
        if (threadIdx.x == 0) {
            if (error) raise_status(p.status, error);
            plan[0] = error ? -1 : n;
            plan[1] = m;
            if (!error && m > 0) pp.len[ui.cache_unit] = n + m;
        }
    }
    ptx::cluster_arrive();
    ptx::cluster_wait();
    int32_t start, rows;
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(ptx::smem_u32(plan)));
    asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];" : "=r"(start), "=r"(rows) : "r"(at) : "memory");
    ptx::cluster_arrive();  // the first CTA's memory is read
    const int G = p.Hq / p.Hkv, Hq = p.q.data ? p.Hq : 0, nq = p.q.data ? G : 0;
    for (int32_t row = first; row < rows; row += ctas * kUnitWarps) {
        __syncwarp();
        if (row != first) token_angles(p, t0 + row, angles[warp]);
        const Part<T, D> part(p.rot, angles[warp]);
        move_rows<T, D, true, 2>(
            p, part, ui.l_local, t0 + row, ui.b, row, Hq, [=](int) { return start; }, nq + 2,
            [=](int i) { return i < nq ? ui.h * G + i : Hq + ui.h + (i - nq) * p.Hkv; });
    }
    ptx::cluster_wait();
}

template <typename T>
cudaError_t launch_rows(const RowsParams &p, bool cache, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    const int64_t warps = (int64_t)p.layer_count * p.T * p.chunks;
    cfg.gridDim = dim3((unsigned)((warps + kWarps - 1) / kWarps));
    cfg.blockDim = dim3(32 * kWarps);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (p.D == 128)
        return cache ? cudaLaunchKernelEx(&cfg, rows_kernel<T, 128, true>, p)
                     : cudaLaunchKernelEx(&cfg, rows_kernel<T, 128, false>, p);
    return cache ? cudaLaunchKernelEx(&cfg, rows_kernel<T, 64, true>, p)
                 : cudaLaunchKernelEx(&cfg, rows_kernel<T, 64, false>, p);
}

cudaError_t launch_rows(const voxzip_cache_desc &d, RowsParams &p, bool cache, cudaStream_t stream) {
    p.D = d.head_dim;
    p.Hq = d.q_heads;
    p.Hkv = d.kv_heads;
    // A warp takes all heads of a token, unless there are too few tokens to fill the SMs: then fewer, as long as it
    // has one round of them (a warp has 32 / (D / 2 / vector) heads in hand at once).
    const int vec = d.dtype == VOXZIP_BF16 ? 8 : 4;
    const int round = 32 / (d.head_dim / vec / 2);
    const int64_t tokens = (int64_t)p.layer_count * p.T;
    const int64_t want = (int64_t)sm_count() * 16;
    const int most = (p.heads + round - 1) / round;
    p.chunks = (int)std::min<int64_t>(most, std::max<int64_t>(1, (want + tokens - 1) / tokens));
    p.warp_heads = (p.heads + p.chunks - 1) / p.chunks;
    p.warp_heads = (p.warp_heads + round - 1) / round * round;
    p.chunks = (p.heads + p.warp_heads - 1) / p.warp_heads;
    return d.dtype == VOXZIP_BF16 ? launch_rows<__nv_bfloat16>(p, cache, stream) : launch_rows<float>(p, cache, stream);
}

}  // namespace

cudaError_t launch_rotary(const voxzip_cache_desc &d, const RotaryTable &table, int32_t layer_count, int32_t tokens,
                          RowsView q, RowsView k, const int32_t *positions, void *q_out, void *k_out,
                          cudaStream_t stream) {
    RowsParams p = {};
    p.rot = table;
    p.q = q;
    p.k = k;
    p.q_out = q_out;
    p.k_out = k_out;
    p.positions = positions;
    p.T = tokens;
    p.layer_count = layer_count;
    p.heads = (q.data ? d.q_heads : 0) + (k.data ? d.kv_heads : 0);
    return launch_rows(d, p, false, stream);
}

// CTAs of a unit's cluster where an append is one launch, 0 where it is a plan and the rows. One launch is 10 us less of an
// eager call and needs no workspace, for sequences of up to a token per warp of a cluster (with several a warp it takes twice
// as long) and units that all start at once: each computes its tokens' angles anew, and where clusters wait for places that
// shows. 32/4 heads, D = 128, us of the GPU in one launch and in two: one layer of four sequences of 57 to 64 tokens (128
// CTAs) 8.0 and 8.1; two layers 8.0 and 8.7; four 14.3 and 10.4; 12 of them 37 and 15; 48 of them 151 and 52.
inline int unit_ctas(const voxzip_cache_desc &d, int32_t layer_count, int32_t tokens, int32_t max_rows) {
    const int32_t bound = max_rows > 0 && max_rows < tokens ? max_rows : tokens;
    if (bound > kUnitCtas * kUnitWarps) return 0;
    int ctas = 1;
    while (ctas * kUnitWarps < bound) ctas *= 2;
    return (int64_t)d.batch * layer_count * d.kv_heads * ctas <= 2 * sm_count() ? ctas : 0;
}

size_t append_workspace_bytes(const voxzip_cache_desc &d, int32_t layer_count, int32_t tokens, int32_t max_rows) {
    if (unit_ctas(d, layer_count, tokens, max_rows) > 0) return 0;
    return ((size_t)d.batch * layer_count * d.kv_heads * sizeof(int32_t) + 255) / 256 * 256;
}

cudaError_t launch_append(const voxzip_cache_desc &d, const RotaryTable *table, int32_t layer_begin,
                          int32_t layer_count, RowsView q, RowsView k, RowsView v, const int32_t *positions,
                          const int32_t *new_pos, const int32_t *seq_off, int32_t tokens, int32_t max_rows,
                          const CacheRows &cache, float *score, int32_t *pos, int32_t *len, void *q_out,
                          void *workspace, int32_t *status, cudaStream_t stream) {
    PlanParams pp = {};
    pp.seq_off = seq_off;
    pp.pv = cache.pv;
    pp.len = len;
    pp.start = static_cast<int32_t *>(workspace);
    pp.status = status;
    pp.B = d.batch;
    pp.L = d.layers;
    pp.Hkv = d.kv_heads;
    pp.C = d.capacity;
    pp.T = tokens;
    pp.layer_begin = layer_begin;
    pp.units = d.batch * layer_count * d.kv_heads;
    RowsParams p = {};
    if (table) p.rot = *table;
    p.q = q;
    p.k = k;
    p.v = v;
    p.q_out = q_out;
    p.positions = positions;
    p.seq_off = seq_off;
    p.new_pos = new_pos;
    p.start = pp.start;
    p.cache = cache;
    p.score = score;
    p.pos = pos;
    p.status = status;
    p.T = tokens;
    p.B = d.batch;
    p.L = d.layers;
    p.Hq = d.q_heads;
    p.Hkv = d.kv_heads;
    p.C = d.capacity;
    p.D = d.head_dim;
    p.layer_begin = layer_begin;
    p.layer_count = layer_count;
    p.heads = (q.data ? d.q_heads : 0) + 2 * d.kv_heads;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e;
    if (const int ctas = unit_ctas(d, layer_count, tokens, max_rows)) {
        cfg.gridDim = dim3(pp.units * ctas);
        cfg.blockDim = dim3(32 * kUnitWarps);
        cudaLaunchAttribute both[2] = {attr[0], {}};
        both[1].id = cudaLaunchAttributeClusterDimension;
        both[1].val.clusterDim.x = ctas;
        both[1].val.clusterDim.y = both[1].val.clusterDim.z = 1;
        cfg.attrs = both;
        cfg.numAttrs = 2;
        if (d.dtype == VOXZIP_BF16)
            e = d.head_dim == 128 ? cudaLaunchKernelEx(&cfg, append_unit_kernel<__nv_bfloat16, 128>, pp, p, ctas)
                                  : cudaLaunchKernelEx(&cfg, append_unit_kernel<__nv_bfloat16, 64>, pp, p, ctas);
        else
            e = d.head_dim == 128 ? cudaLaunchKernelEx(&cfg, append_unit_kernel<float, 128>, pp, p, ctas)
                                  : cudaLaunchKernelEx(&cfg, append_unit_kernel<float, 64>, pp, p, ctas);
    } else {
        cfg.gridDim = dim3((pp.units + 3) / 4);
        cfg.blockDim = dim3(128);
        e = cudaLaunchKernelEx(&cfg, append_plan_kernel, pp);
        if (e == cudaSuccess) e = launch_rows(d, p, true, stream);
    }
    if (e != cudaSuccess || !cache.pv.table) return e;
    cfg.gridDim = dim3((pp.units + 127) / 128);
    cfg.blockDim = dim3(128);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, append_next_page_kernel, pp);
}

}  // namespace voxzip
