// Causal attention of a prompt's packed bf16 rows on the tensor cores (the mathematics: prompt_attn.cu).
//
// A CTA has 256 rows ((token, head of the group) pairs) of a unit as two tiles of 128, which take turns on the tensor
// cores: while a warpgroup turns one tile's logits into weights, the other tile's products run.
//   S_t = Q_t K_j'           128 x 128, fp32, tensor memory
//   P_t = 2^(c S_t - m - 8)  bf16, over S_t's columns; rounding it costs 2^-8 of each weight, as much as the output's (V is
//                            bf16 and both operands are of one type; a row's sum is of the weights before it)
//   O_t += P_t V_j           128 x D, fp32, tensor memory
// (a tile's products run in the order in which its one warp issues them, so S_t's next logits may overwrite P_t).
// m is a row's reference, not its running maximum: it moves (and O_t with it) only when the maximum has grown by more
// than 2^8 over it, so weights stay at most 1 and nearly every tile leaves O_t to the tensor cores alone.
// A CTA that is done takes the place of one that has not started: the copies and logits of its next tile begin while the
// results of the last are on their way out (10-min prompt without outlier channels of K 380 us against 397, 32 ragged ones 5.0 ms against 5.3; a fixed
// share for each CTA 401 us).
// Warps 0-7 and 8-15: a tile's weights, a quarter of two rows per thread (a thread per row took 1500 cycles, which the
// other tile's 1000 cycles of products cannot hide). Warps 16 and 19: a tile's matrix instructions (one warp for both
// would wait for one tile's weights while the other's lie ready). Warp 17: items, and copies of their tiles into a ring of
// K and V. Warp 18: what the mask hides of V.
// 46 024 tokens, 32/4 heads, D = 128: 11.4 to 12.3 ms by box, up to 1 520 TFLOP/s, 0.78 of the measured burst rate and 0.88
// of the sustained one: the card is then at its power limit (1 390 W at 1 940 MHz, sw_power_cap), the tensor cores busy
// for 63% of the cycles.
#include <algorithm>

#include "evict_policy.cuh"  // once_per_device
#include "prompt.cuh"
#include "ptx.cuh"
#include "tcgen05.cuh"
#include "tmap.cuh"

namespace voxzip {
namespace {

constexpr int kTile = 128;       // rows of a tile, keys of a tile
constexpr int kMatrixWarp = 16, kCopyWarp = 17, kMaskWarp = 18, kMatrixWarp1 = 19;
constexpr int kThreads = 20 * 32;
// Polls of a wait for a few tiles: 4 s by a whole warp (7 850 cycles a poll), 38 ms by one lane, which is not suspended (70).
// The longest, for the results of an item in which the mask hides infinities, takes 0.1 ms.
constexpr uint32_t kPolls = 1u << 20;
// Those of a wait for an item without any step of the copies: 4 s, in checked builds 8 ms, shorter than their tests' items.
#ifdef VOXZIP_CHECKED
constexpr uint32_t kItemPolls = 1u << 11;
#else
constexpr uint32_t kItemPolls = 1u << 20;
#endif
constexpr float kSlack = 8.f;    // growth of a row's maximum that its reference lets pass (log2)

template <int D> struct Cfg {
    static constexpr int kHalves = D / 64;                    // copies of 64 channels
    static constexpr int kHalfBytes = kTile * 128;            // one of them
    static constexpr int kTileBytes = kHalves * kHalfBytes;   // a Q, K or V tile
    static constexpr int kStages = D == 128 ? 5 : 6;
    static constexpr int kBytes = 2 * kTileBytes + kStages * kTileBytes;
    static constexpr uint32_t kColO = 256;                    // S_0, S_1: columns 0 and 128
    static constexpr uint32_t kColumns = 512;
};

// A tile of the launch: 256 rows and the keys of its split.
struct Item {
    int32_t valid;           // 0: there is none left
    int32_t h, l, t0, rows;  // kv-head, layer; first packed token, tokens
    int32_t part;            // where its part goes, -1: all keys are its own
    int32_t first;           // keys that its first token sees (may be < 1)
    int32_t most;            // keys that its last one sees
    int32_t j0, end0, end1;  // key tiles [j0, end0) and [j0, end1) of the two row tiles
    int32_t dirty;           // the mask warp has taken elements out of V
    int64_t cu;              // cache unit

    __device__ __forceinline__ int32_t end() const { return max(end0, end1); }
    // From this key tile on some row does not see all keys.
    __device__ __forceinline__ int32_t masked0() const { return max(j0, max(0, first) / kTile); }
};

template <int D> struct Shared {
    uint64_t item_full[2], item_empty[2], q_full, q_empty, full[Cfg<D>::kStages], empty[Cfg<D>::kStages], s_full[2], p_full[2],
        o_full[2], o_empty[2], sent[2][4], clean[2][4], pair[8], drained[2], next_full;
    alignas(16) uint4 next;  // the hardware's answer: a CTA that need not start
    Item item[2];
    float sum[2][kTile], top[2][kTile];  // of the rows, when they are done
    uint32_t tmem, steps;  // (of the copy warp)
    int dead;
};

// The tiles start on a multiple of 1024 behind Shared; a CTA's memory does too, but for what the compiler puts first.
constexpr size_t kFront = 3 * 1024;
template <int D> constexpr size_t smem_bytes() { return kFront + Cfg<D>::kBytes; }
static_assert(sizeof(Shared<128>) <= kFront && sizeof(Shared<64>) <= kFront && smem_bytes<128>() <= 232448, "what an SM has");

// A bounded wait; once one has given up in a CTA, all do.
template <int D> __device__ __forceinline__ bool wait(Shared<D> &sh, uint64_t *bar, uint32_t parity) {
    for (uint32_t i = 0; i < kPolls; ++i) {
        if (ptx::mbar_try_wait(bar, parity)) return true;
        if ((i & 63) == 63 && *reinterpret_cast<volatile int *>(&sh.dead)) return false;
    }
    *reinterpret_cast<volatile int *>(&sh.dead) = 1;
    return false;
}

// The same for what takes as long as an item: it gives up when the copy warp has not come further for kItemPolls. (A tile's copy
// waits for the products of the one whose place it takes, so while there are copies all warps advance, and an item has so
// many tiles. Every other wait is for a few tiles.)
template <int D> __device__ __forceinline__ bool wait_item(Shared<D> &sh, uint64_t *bar, uint32_t parity) {
    uint32_t steps = 0;  // (before the first one)
    for (uint32_t i = 0; i < kItemPolls / 64; ++i) {
        if (ptx::mbar_wait_bounded(bar, parity, 64)) return true;
        if (*reinterpret_cast<volatile int *>(&sh.dead)) return false;
        const uint32_t now = *reinterpret_cast<volatile uint32_t *>(&sh.steps);
        if (now != steps) steps = now, i = 0;
    }
    *reinterpret_cast<volatile int *>(&sh.dead) = 1;
    return false;
}

// The same by all lanes of a warp, which stay together whatever each of them saw.
template <int D> __device__ __forceinline__ bool wait_warp(Shared<D> &sh, uint64_t *bar, uint32_t parity) {
    return __all_sync(0xffffffffu, wait(sh, bar, parity));
}
template <int D> __device__ __forceinline__ bool wait_item_warp(Shared<D> &sh, uint64_t *bar, uint32_t parity) {
    return __all_sync(0xffffffffu, wait_item(sh, bar, parity));
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
// (a0, a1) b + c and (a0, a1) + (b0, b1), two at a time.
__device__ __forceinline__ float2 fma2(float a0, float a1, float b, float c) {
    float2 y;
    asm("{\n\t.reg .b64 u, v, w;\n\tmov.b64 u, {%2, %3};\n\tmov.b64 v, {%4, %4};\n\tmov.b64 w, {%5, %5};\n\t"
        "fma.rn.f32x2 u, u, v, w;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "=f"(y.x), "=f"(y.y)
        : "f"(a0), "f"(a1), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ void add2(float2 &a, float b0, float b1) {
    asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tadd.rn.f32x2 u, u, v;\n\t"
        "mov.b64 {%0, %1}, u;\n\t}"
        : "+f"(a.x), "+f"(a.y)
        : "f"(b0), "f"(b1));
}

__device__ __forceinline__ void tma_load_4d(void *dst, const CUtensorMap *map, int x, int y, int z, int w, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(ptx::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(ptx::smem_u32(bar))
        : "memory");
}

// Asks for a CTA of this launch that has not started, which then will not; the answer comes by `bar`.
__device__ __forceinline__ void ask_next(uint4 *answer, uint64_t *bar) {
    ptx::mbar_arrive_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                     ptx::smem_u32(answer)),
                 "r"(ptx::smem_u32(bar))
                 : "memory");
}
// Whether there was one, and its blockIdx.x.
__device__ __forceinline__ bool canceled(const uint4 *answer, int64_t *x) {
    uint32_t ok, cta;
    asm volatile(
        "{\n\t.reg .b128 a;\n\t.reg .pred p;\n\t.reg .b64 lo, hi;\n\t"
        "ld.shared.v2.b64 {lo, hi}, [%2];\n\tmov.b128 a, {lo, hi};\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\tselp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, a;\n\t}"
        : "=r"(ok), "=r"(cta)
        : "r"(ptx::smem_u32(answer))
        : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // read before the next answer is written
    *x = cta;
    return ok != 0;
}

template <int D, bool kPaged>
__global__ void __launch_bounds__(kThreads, 1)
prompt_mma_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                  const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PromptAttn p) {
    using C = Cfg<D>;
    extern __shared__ __align__(16) uint8_t raw[];
    Shared<D> &sh = *reinterpret_cast<Shared<D> *>(raw);
    const uint32_t front = (sizeof(Shared<D>) + ptx::smem_u32(raw) + 1023) / 1024 * 1024 - ptx::smem_u32(raw);
    if (front + C::kBytes > smem_bytes<D>()) {  // (never: the memory in front of raw is a multiple of 1024)
        ptx::grid_dependency_wait();
        raise_status(p.status, VOXZIP_DEV_TIMEOUT);
        return;
    }
    uint8_t *tiles = raw + front;
    uint8_t *q_smem = tiles, *ring = tiles + 2 * C::kTileBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // uniform for the compiler too
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(&sh.item_full[i], 1), ptx::mbar_init(&sh.item_empty[i], kMatrixWarp + 3);
            ptx::mbar_init(&sh.s_full[i], 1), ptx::mbar_init(&sh.p_full[i], 8);
            ptx::mbar_init(&sh.o_full[i], 1), ptx::mbar_init(&sh.o_empty[i], 8);
            for (int e = 0; e < 4; ++e) ptx::mbar_init(&sh.sent[i][e], 1), ptx::mbar_init(&sh.clean[i][e], 1);
            ptx::mbar_init(&sh.drained[i], 1);
        }
        ptx::mbar_init(&sh.q_full, 1), ptx::mbar_init(&sh.q_empty, 2), ptx::mbar_init(&sh.next_full, 1);
        for (int i = 0; i < C::kStages; ++i) ptx::mbar_init(&sh.full[i], 1), ptx::mbar_init(&sh.empty[i], 2);
        for (int i = 0; i < 8; ++i) ptx::mbar_init(&sh.pair[i], 2);
        ptx::fence_mbar_init();
        sh.dead = 0;
        sh.steps = 0;
    }
    if (warp == kMatrixWarp) tc::alloc(&sh.tmem, C::kColumns);
    if (warp == kCopyWarp && lane == 0) {
        ptx::prefetch_tmap(&map_q);
        ptx::prefetch_tmap(&map_k);
        ptx::prefetch_tmap(&map_v);
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    ptx::grid_dependency_wait();
    ptx::launch_dependents();  // the join may take its place on the SMs
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
    const int tile_tokens = kTile / p.G;
    bool live = true;

    if (warp == kCopyWarp) {
        // ------------------------------------------------------------ items and copies
        const int64_t items = (int64_t)(p.tiles + p.part_tiles * (p.splits - 1)) * p.Hkv * p.layer_count;
        int issued = 0, queries = 0, given = 0;
        // Its own, then those of CTAs that have not started: the hardware gives them out in order.
        int64_t i = blockIdx.x;
        uint32_t asked = 0, steps = 0;
        bool more = true;
        auto step = [&] { *reinterpret_cast<volatile uint32_t *>(&sh.steps) = ++steps; };  // (lane 0)
        for (bool first = true; live; first = false) {
            if (lane == 0) step();
            if (!first) {
                if (!(live = wait_warp(sh, &sh.next_full, (asked - 1) & 1))) break;
                more = canceled(&sh.next, &i);
                __syncwarp();
            }
            if (more) {
                if (lane == 0) ask_next(&sh.next, &sh.next_full);
                ++asked;
            }
            Item w = {};
            if (more) {
                if (i >= items) continue;
                const CtaAt cta = cta_at(p, i);
                TileAt at;
                if (!find_tile(p, cta, at)) continue;
                if (at.n < 0 || at.n > p.C) {
                    if (lane == 0) raise_status(p.status, VOXZIP_DEV_CAPACITY);
                    continue;
                }
                const bool split = in_parts(p, cta.x, at);
                if (!split && cta.split > 0) continue;
                const int splits = split ? p.splits : 1;
                w.valid = 1;
                w.h = cta.h, w.l = cta.l, w.t0 = at.t0, w.rows = at.rows;
                w.part = split ? part_of(p, cta) : -1;
                w.cu = ((int64_t)at.b * p.L + p.layer_begin + cta.l) * p.Hkv + cta.h;
                w.first = at.n - at.m + at.before + 1;
                w.most = max(0, w.first + at.rows - 1);
                // the keys of this split, of those that the last token sees; row tile 0 ends with its own last token's
                const int32_t total = (w.most + kTile - 1) / kTile, per = (total + splits - 1) / splits;
                w.j0 = min(total, cta.split * per);
                const int32_t j1 = min(total, w.j0 + per);
                const int32_t most0 = max(0, w.first + min(tile_tokens, at.rows) - 1);
                w.end0 = max(w.j0, min(j1, (most0 + kTile - 1) / kTile));
                w.end1 = at.rows > tile_tokens ? j1 : w.j0;
            }
            const int place = given & 1;
            if (given >= 2 && !(live = wait_warp(sh, &sh.item_empty[place], (given >> 1 & 1) ^ 1))) break;
            if (lane == 0) {
                sh.item[place] = w;
                ptx::mbar_arrive(&sh.item_full[place]);
            }
            __syncwarp();
            ++given;
            if (!w.valid) break;
            const int32_t end = w.end(), masked0 = w.masked0();
            if (end > w.j0) {
                if (queries > 0 && !(live = wait_warp(sh, &sh.q_empty, (queries - 1) & 1))) break;
                ++queries;
                if (lane == 0) {
                    const uint32_t bytes = p.G * tile_tokens * 128 * C::kHalves;
                    const int both = w.rows > tile_tokens ? 2 : 1;
                    ptx::mbar_arrive_expect_tx(&sh.q_full, bytes * both);
                    for (int t = 0; t < both; ++t)
                        for (int c = 0; c < C::kHalves; ++c)
                            tma_load_4d(q_smem + t * C::kTileBytes + c * C::kHalfBytes, &map_q, 64 * c, w.h * p.G,
                                        w.t0 + t * tile_tokens, w.l, &sh.q_full);
                }
            }
            int32_t pages = 0, pages_at = INT32_MIN;  // this lane's of 32 consecutive page indices
            for (int32_t j = w.j0; j < end && live; ++j) {
                int32_t row[2];
                if constexpr (kPaged) {
                    constexpr int kPages = kTile / kPageTokens;
                    const int32_t first_page = j * kPages;
                    if (pages_at == INT32_MIN || first_page >= pages_at + 32) {
                        pages_at = first_page;
                        const int32_t at_page = first_page + lane;
                        pages = -1;
                        if (at_page * kPageTokens < w.most) {
                            pages = p.cache.pv.table[w.cu * p.cache.pv.max_pages + at_page];
                            if (pages < 0 || (int64_t)pages * kPageTokens >= p.cache.pool_rows) {
                                raise_status(p.status, VOXZIP_DEV_CAPACITY);
                                pages = -1;
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kPages; ++i) {
                        const int32_t page = __shfl_sync(0xffffffffu, pages, first_page - pages_at + i);
                        row[i] = page < 0 ? (int32_t)p.cache.pool_rows : page * kPageTokens;  // outside: zeros
                    }
                } else {
                    row[0] = (int32_t)(w.cu * p.C + (int64_t)j * kTile);
                    row[1] = row[0] + kTile / 2;
                    (void)VOXZIP_IN_RANGE(p.status, row[0] >= 0 && row[0] < p.kv_rows);
                }
                if (lane == 0) {
                    for (int kv = 0; kv < 2 && live; ++kv) {
                        const int slot = issued % C::kStages;
                        live = issued < C::kStages || wait(sh, &sh.empty[slot], (issued / C::kStages & 1) ^ 1);
                        if (!live) break;
                        const CUtensorMap *map = kv ? &map_v : &map_k;
                        uint8_t *to = ring + slot * C::kTileBytes;
                        ptx::mbar_arrive_expect_tx(&sh.full[slot], C::kTileBytes);
                        for (int c = 0; c < C::kHalves; ++c) {
                            ptx::tma_load_2d(to + c * C::kHalfBytes, map, 64 * c, row[0], &sh.full[slot]);
                            if (kPaged)
                                ptx::tma_load_2d(to + c * C::kHalfBytes + C::kHalfBytes / 2, map, 64 * c, row[1],
                                                 &sh.full[slot]);
                        }
                        ++issued;
                        step();
                        if (kv && j >= masked0) ptx::mbar_arrive(&sh.sent[place][j - masked0]);
                    }
                }
                live = __shfl_sync(0xffffffffu, live, 0);
            }
        }
        if (lane == 0 && !live) {  // a wait gave up: no copy is left in flight behind this CTA
            for (int i = max(0, issued - C::kStages); i < issued; ++i)
                ptx::mbar_wait_bounded(&sh.full[i % C::kStages], i / C::kStages & 1, kPolls);
            if (queries > 0) ptx::mbar_wait_bounded(&sh.q_full, (queries - 1) & 1, kPolls);
            if (asked > 0) ptx::mbar_wait_bounded(&sh.next_full, (asked - 1) & 1, kPolls);
        }
    } else if (warp == kMatrixWarp || warp == kMatrixWarp1) {
        // ------------------------------------------------------------ matrix instructions, a warp per row tile
        constexpr uint32_t kInstS = tc::instruction(kTile, false), kInstO = tc::instruction(D, true);
        const int t = warp == kMatrixWarp1;
        const uint32_t q_at = ptx::smem_u32(q_smem) + t * C::kTileBytes, ring_at = ptx::smem_u32(ring);
        const uint32_t s_at = tmem + t * kTile, o_at = tmem + C::kColO + t * D;
        int slot = 0, phase = 0;  // of the ring's next tile
        uint32_t weights_phase = 0, results = 0, queries_phase = 0, clean_phase[2] = {0, 0};
        auto advance = [&] {
            if (++slot == C::kStages) slot = 0, phase ^= 1;
        };
        auto logits = [&](int k_slot) {
            const uint32_t k_at = ring_at + k_slot * C::kTileBytes;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint32_t off = k / 4 * C::kHalfBytes + k % 4 * 32;
                tc::mma(s_at, tc::operand(q_at + off, 0), tc::operand(k_at + off, 0), kInstS, k > 0);
            }
            tc::commit(&sh.s_full[t]);
        };
        // Gives memory back. What this warp has no use for goes back only when it has come: before that, the barrier's
        // phase is that of its last use.
        auto release = [&](uint64_t *bar, bool used) {
            if (used)
                tc::commit(bar);
            else if (lane == 0)
                ptx::mbar_arrive(bar);
        };
        for (int n = 0; live; ++n) {
            const int place = n & 1;
            if (!(live = wait_item_warp(sh, &sh.item_full[place], n >> 1 & 1))) break;
            const Item &w = sh.item[place];
            const int32_t valid = w.valid, j0 = w.j0, t_end = t ? w.end1 : w.end0, end = w.end(), masked0 = w.masked0();
            if (!valid) break;
            if (end == j0) {
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sh.item_empty[place]);
                continue;
            }
            live = wait_warp(sh, &sh.q_full, queries_phase) && wait_warp(sh, &sh.full[slot], phase);
            if (!live) break;
            queries_phase ^= 1;
            tc::fence_after();
            if (j0 < t_end) logits(slot);
            release(&sh.empty[slot], j0 < t_end);
            if (j0 + 1 >= t_end) release(&sh.q_empty, j0 < t_end);
            advance();
            for (int32_t j = j0; j < end; ++j) {
                // V of this key tile and K of the next, before the weights: their copies are long done
                const int v_slot = slot;
                live = wait_warp(sh, &sh.full[slot], phase);
                advance();
                const int k_slot = slot;
                if (live && j + 1 < end) {
                    live = wait_warp(sh, &sh.full[slot], phase);
                    advance();
                }
                if (live && j >= masked0)
                    live = wait_warp(sh, &sh.clean[place][j - masked0], clean_phase[place] >> (j - masked0) & 1);
                if (live && j < t_end) {
                    live = wait_warp(sh, &sh.p_full[t], weights_phase);
                    weights_phase ^= 1;
                    if (live && j == j0 && results > 0) live = wait_warp(sh, &sh.o_empty[t], (results - 1) & 1);
                    if (!live) break;
                    tc::fence_after();
                    const uint32_t v_at = ring_at + v_slot * C::kTileBytes;
#pragma unroll
                    for (int k = 0; k < kTile / 16; ++k)
                        tc::mma_ta(o_at, s_at + k * 8, tc::operand(v_at + k * 16 * 128, C::kHalfBytes), kInstO,
                                   j > j0 || k > 0);
                    if (j + 1 < t_end) logits(k_slot);
                    if (j + 1 == t_end) tc::commit(&sh.o_full[t]);
                }
                if (!live) break;
                release(&sh.empty[v_slot], j < t_end);
                if (j + 1 < end) release(&sh.empty[k_slot], j + 1 < t_end);
                if (j + 2 == t_end) tc::commit(&sh.q_empty);
            }
            if (j0 < t_end) ++results;
            clean_phase[place] ^= (1u << max(0, end - masked0)) - 1;
            if (live && lane == 0) ptx::mbar_arrive(&sh.item_empty[place]);
        }
        if (!live) {  // a wait gave up: what was issued ends before the tensor memory goes
            tc::commit(&sh.drained[t]);
            ptx::mbar_wait_bounded(&sh.drained[t], 0, kPolls);
            raise_status(p.status, VOXZIP_DEV_TIMEOUT);
        }
    } else if (warp == kMaskWarp) {
        // ------------------------------------------------------------ V behind the mask
        // A weight of 0 times an infinity or a NaN would be NaN in rows that do not see the key. Rows that nobody sees
        // become 0. In rows that some see such elements do, and join the result at the end.
        int tiles_before = 0;  // of the ring
        uint32_t sent_phase[2] = {0, 0};
        for (int n = 0; live; ++n) {
            const int place = n & 1;
            if (!(live = wait_item_warp(sh, &sh.item_full[place], n >> 1 & 1))) break;
            Item &w = sh.item[place];
            if (!w.valid) break;
            const int32_t j0 = w.j0, end = w.end(), masked0 = w.masked0();
            for (int32_t j = masked0; j < end && live; ++j) {
                const int i = tiles_before + 2 * (j - j0) + 1, slot = i % C::kStages;
                // only once its copy is asked for is a phase of the slot's barrier this tile's
                live = wait_item_warp(sh, &sh.sent[place][j - masked0], sent_phase[place] >> (j - masked0) & 1) &&
                       wait_warp(sh, &sh.full[slot], i / C::kStages & 1);
                if (!live) break;
                uint8_t *tile = ring + slot * C::kTileBytes;
                const int32_t key0 = j * kTile;
                const int r0 = max(0, w.first - key0), r1 = min(kTile, max(0, w.most - key0));
                bool found = false;
#pragma unroll
                for (int c = 0; c < C::kHalves; ++c) {
                    uint4 *half = reinterpret_cast<uint4 *>(tile + c * C::kHalfBytes);
                    for (int i0 = r0 * 8 + lane; i0 < r1 * 8; i0 += 2 * 32) {  // two at a time on their way
                        uint4 u[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            u[e] = i0 + 32 * e < r1 * 8 ? half[i0 + 32 * e] : make_uint4(0, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            uint32_t *x = &u[e].x;
                            bool bad = false;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                if ((x[k] & 0x7f80u) == 0x7f80u) x[k] &= 0xffff0000u, bad = true;
                                if ((x[k] & 0x7f800000u) == 0x7f800000u) x[k] &= 0x0000ffffu, bad = true;
                            }
                            if (bad) half[i0 + 32 * e] = u[e];
                            found |= bad;
                        }
                    }
                    for (int i = r1 * 8 + lane; i < kTile * 8; i += 32) half[i] = make_uint4(0, 0, 0, 0);
                }
                if (__any_sync(0xffffffffu, found) && lane == 0) *reinterpret_cast<volatile int32_t *>(&w.dirty) = 1;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sh.clean[place][j - masked0]);
            }
            tiles_before += 2 * (end - j0);
            sent_phase[place] ^= (1u << max(0, end - masked0)) - 1;
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sh.item_empty[place]);
        }
    } else {
        // ------------------------------------------------------------ weights, a quarter of two rows per thread
        const int t = warp >> 3, hf = warp >> 2 & 1;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // the 32 lanes that this warp can reach
        const uint32_t s_at = tmem + (lanes | (uint32_t)hf << 20) + t * kTile;  // 16 of them are its own
        const uint32_t o_rows = tmem + (lanes | (uint32_t)hf << 20) + C::kColO + t * D;
        const int own = (warp & 3) * 32 + hf * 16 + lane / 4;  // its first row; the second is 8 on
        uint64_t *pair = &sh.pair[t * 4 + (warp & 3)];  // of the two warps that share the 32 lanes
        uint32_t logits_phase = 0, results_phase = 0;
        for (int n = 0; live; ++n) {
            const int place = n & 1;
            if (!(live = wait_item_warp(sh, &sh.item_full[place], n >> 1 & 1))) break;
            const Item &w = sh.item[place];
            if (!w.valid) break;
            const int32_t t_end = t ? w.end1 : w.end0, j0 = w.j0, masked0 = w.masked0();
            float m[2] = {-INFINITY, -INFINITY};
            float2 sums[2] = {};
            for (int32_t j = j0; j < t_end; ++j) {
                if (!(live = wait_warp(sh, &sh.s_full[t], logits_phase))) break;
                logits_phase ^= 1;
                tc::fence_after();
                float x[2][32];
                tc::ld_rows(s_at, x[0]);
                tc::ld_rows(s_at + 64, x[1]);
                tc::wait_ld();
                if (j >= masked0) {
                    int row0 = own;
                    asm volatile("" : "+r"(row0));  // (what follows is not kept in registers from tile to tile)
                    int32_t lims[2];                // keys that the two rows see
#pragma unroll
                    for (int e = 0; e < 2; ++e) lims[e] = w.first + t * tile_tokens + (row0 + 8 * e) / p.G;
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (64 * c + i / 4 * 8 + (lane & 3) * 2 + (i & 1) >= lims[i >> 1 & 1] - j * kTile) x[c][i] = -INFINITY;
                }
                float top[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float a = fmaxf(x[0][2 * e], x[0][2 * e + 1]), b = fmaxf(x[1][2 * e], x[1][2 * e + 1]);
#pragma unroll
                    for (int i = 4; i < 32; i += 4) {
                        a = max3(a, x[0][i + 2 * e], x[0][i + 2 * e + 1]);
                        b = max3(b, x[1][i + 2 * e], x[1][i + 2 * e + 1]);
                    }
                    top[e] = fmaxf(a, b);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 1));
                    top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 2)) * p.scale_log2;
                }
                const bool grown[2] = {top[0] > m[0] + kSlack, top[1] > m[1] + kSlack};
                if (__any_sync(0xffffffffu, grown[0] || grown[1])) {
                    float keep[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        keep[e] = grown[e] ? ex2(m[e] - top[e]) : 1.f;  // a row does not depend on its neighbours
                        if (grown[e]) m[e] = top[e];
                        sums[e].x *= keep[e], sums[e].y *= keep[e];
                    }
                    if (j > j0) {  // the products of the tiles before are done: the logits' commit came after theirs
                        float o[8];
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {
                            tc::ld_rows16(o_rows + c, o);
                            tc::wait_ld();
#pragma unroll
                            for (int i = 0; i < 8; ++i) o[i] *= keep[i >> 1 & 1];
                            tc::st_rows16(o_rows + c, o);
                        }
                    }
                }
                const float ref[2] = {m[0] == -INFINITY ? 0.f : -m[0] - kSlack, m[1] == -INFINITY ? 0.f : -m[1] - kSlack};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t u[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 e = fma2(x[c][2 * i], x[c][2 * i + 1], p.scale_log2, ref[i & 1]);
                        const float a = ex2(e.x), b = ex2(e.y);
                        add2(sums[i & 1], a, b);
                        u[i] = ptx::pack_bf16(a, b);
                    }
                    tc::st_rows(s_at + 32 * c, u);
                }
                tc::wait_st();
                tc::fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&sh.p_full[t]);
            }
            // ------------------------------------------------------------ results, half a row per thread
            constexpr int kCols = D / 2;
            const uint32_t o_at = tmem + lanes + C::kColO + t * D + hf * kCols;
            int r = threadIdx.x & (kTile - 1);
            asm volatile("" : "+r"(r));  // (nor is this)
            const int32_t token = t * tile_tokens + r / p.G, lim = w.first + token;
            const bool any = t_end > j0;
            float sum = 0.f, m_row = -INFINITY;
            if (live && any) {
                live = wait_warp(sh, &sh.o_full[t], results_phase);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float part = sums[e].x + sums[e].y;
                    part += __shfl_xor_sync(0xffffffffu, part, 1);
                    part += __shfl_xor_sync(0xffffffffu, part, 2);
                    if ((lane & 3) == 0) sh.sum[t][own + 8 * e] = part, sh.top[t][own + 8 * e] = m[e];
                }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(pair);
                live = wait_warp(sh, pair, results_phase) && live;
                results_phase ^= 1;
                sum = sh.sum[t][r], m_row = sh.top[t][r];
            }
            if (!live) break;
            tc::fence_after();
            const bool mine = token < w.rows && r < tile_tokens * p.G;
            const int64_t row = ((int64_t)w.l * p.T + w.t0 + token) * p.Hq + w.h * p.G + r % p.G;
            const bool none = !any || lim <= 0;
            const float inv = none ? 0.f : 1.f / sum;
            const bool dirty = *reinterpret_cast<volatile int32_t *>(&sh.item[place].dirty);
            const bool whole = w.part < 0;
            const int32_t part = w.part * (p.part_tokens * p.G) + token * p.G + r % p.G;
            if (mine && !whole && hf == 0)
                p.part_ml[part] = make_float2(!any || m_row == -INFINITY ? -INFINITY : m_row + kSlack, any ? sum : 0.f);
            if (any) {
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c) {
                    float o[32];
                    tc::ld32(o_at + 32 * c, o);
                    tc::wait_ld();
                    if (c == kCols / 32 - 1) {  // the last of it is in registers: the next item's products may come
                        tc::fence_before();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(&sh.o_empty[t]);
                    }
                    if (!mine) continue;
                    const int col = hf * kCols + 32 * c;
                    if (whole)
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = none ? 0.f : o[i] * inv;
                    if (dirty) {  // the elements of V that the mask warp took out, for the rows that see them
                        const int32_t k0 = max(max(0, w.first), w.j0 * kTile), k1 = min(lim, t_end * kTile);
                        for (int32_t key = k0; key < k1; ++key) {
                            const int64_t at_row = kPaged ? paged_row(p.cache.pv, w.cu, key) : w.cu * p.C + key;
                            if (at_row < 0 || at_row >= p.kv_rows) continue;
                            const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(p.cache.v) + at_row * D + col;
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                const float e = __bfloat162float(v[i]);
                                if (!isfinite(e)) o[i] += e;
                            }
                        }
                    }
                    if (!whole) {
                        float4 *to = reinterpret_cast<float4 *>(p.part_o + (int64_t)part * D + col);
#pragma unroll
                        for (int i = 0; i < 8; ++i) to[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    } else {
                        uint4 *to = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) + row * D + col);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            to[i] = make_uint4(ptx::pack_bf16(o[8 * i], o[8 * i + 1]), ptx::pack_bf16(o[8 * i + 2], o[8 * i + 3]),
                                               ptx::pack_bf16(o[8 * i + 4], o[8 * i + 5]), ptx::pack_bf16(o[8 * i + 6], o[8 * i + 7]));
                    }
                }
            } else if (mine && whole) {
                uint4 *to = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) + row * D + hf * kCols);
                for (int i = 0; i < kCols / 8; ++i) to[i] = make_uint4(0, 0, 0, 0);
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sh.item_empty[place]);
        }
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    __syncwarp();
    if (warp == kMatrixWarp) tc::dealloc(tmem, C::kColumns);
}

bool encode(CUtensorMap *map, const void *base, int rank, const cuuint64_t *dims, const cuuint64_t *strides,
            const cuuint32_t *box) {
    auto enc = tensor_map_encoder();
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void *>(base), dims, strides, box, ones,
                      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool kPaged> cudaError_t launch(const PromptAttn &p, cudaStream_t stream) {
    static std::atomic<uint64_t> done{0};
    cudaError_t e = once_per_device(done, [] {
        return cudaFuncSetAttribute(prompt_mma_kernel<D, kPaged>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)smem_bytes<D>());
    });
    if (e != cudaSuccess) return e;
    CUtensorMap mq, mk, mv;
    // a stride that no second token or layer uses may be anything: the map gets a valid one
    const int64_t ts = p.T > 1 ? p.q.token_stride : (int64_t)p.Hq * D;
    const int64_t ls = p.layer_count > 1 ? p.q.layer_stride : ts * p.T;
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)p.Hq, (cuuint64_t)p.T, (cuuint64_t)p.layer_count};
    const cuuint64_t strides[3] = {(cuuint64_t)D * 2, (cuuint64_t)ts * 2, (cuuint64_t)ls * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)p.G, (cuuint32_t)(kTile / p.G), 1};
    if (!encode(&mq, p.q.data, 4, dims, strides, box)) return cudaErrorInvalidValue;
    const int rows = kPaged ? kPageTokens : kTile;
    if (!make_cache_map(&mk, p.cache.k, p.cache.pool_rows, D, rows) ||
        !make_cache_map(&mv, p.cache.v, p.cache.pool_rows, D, rows))
        return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(pieces(p));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes<D>();
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, prompt_mma_kernel<D, kPaged>, mq, mk, mv, p);
}

}  // namespace

cudaError_t launch_prompt_mma(const PromptAttn &p, int D, cudaStream_t stream) {
    const bool paged = p.cache.pv.table != nullptr;
    if (D == 128) return paged ? launch<128, true>(p, stream) : launch<128, false>(p, stream);
    return paged ? launch<64, true>(p, stream) : launch<64, false>(p, stream);
}

}  // namespace voxzip
