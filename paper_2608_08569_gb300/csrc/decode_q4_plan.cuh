// How a decode step on the 4-bit cache is laid out in shared memory, and the choice of its launch (decode_q4_mma.cu).
// No CUDA in here: the choice is also made, with a GPU's figures put in by hand, where there is none.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>

namespace voxzip {
namespace q4 {

constexpr int kGroup = 32;  // channels of a scale
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 32;   // tokens per stage
constexpr int kMaxStages = 3;  // of a warp's ring: two, or three where they do not cost the SM a CTA
constexpr int kMaxCluster = 16;
constexpr size_t kMaxSmem = 227 * 1024;

template <int D, int NT, int kParts>
struct Layout {
    static constexpr int J = D / kGroup;
    static constexpr int kGP = 8 * NT;
    static constexpr int kCodeBytes = kTile * D / 2;
    static constexpr int kStageBytes = kCodeBytes + kTile * J * 2;
    static constexpr int kOStride = D + 4;  // a warp's outputs take its drained ring: [kGP][kOStride] fp32
    static constexpr int warp_ring(int stages) { return std::max(stages * kStageBytes, kGP * kOStride * 4); }
    // Offsets from the rings' end.
    static constexpr int kStatOff = 0;
    static constexpr int kStatFloats = 3 * kWarps * kGP;                 // m_w, z_w, f_w [kWarps][kGP]
    static constexpr int kScOff = kStatOff + kStatFloats * 4;  // [kWarps][J][kTile] the scales of a V tile
    static constexpr int kCOff = kScOff + kWarps * J * kTile * 4;  // [NT][J][8] what the accumulators start from
    // q's operands [parts][NT][2 J][32] pairs, and in their place, once every CTA of the cluster has them in
    // registers (fp32: beside them), what the cluster's CTAs send: [S][kGP] maxima and sums, [S][slice] float4 of
    // outputs (S slices cover kGP D).
    static constexpr int kQOff = kCOff + NT * J * 8 * 4;
    static constexpr int kQBytes = kParts * NT * 2 * J * 32 * 8;
    static constexpr int kMzOff = kParts == 1 ? kQOff : kQOff + kQBytes;
    static constexpr int rx_bytes(int S) { return S * (kGP * 8 + 16) + kGP * D * 4; }
    static_assert(kParts > 1 || rx_bytes(2) >= kQBytes, "q's operands fit");
    // [NT][chunk_cap][8] logits, then weights
    static constexpr int lg_off(int S) { return S > 1 ? kMzOff + rx_bytes(S) : kQOff + kQBytes; }
    static size_t bytes(int chunk_cap, int S, int stages) {
        return (size_t)kWarps * warp_ring(stages) + lg_off(S) + (size_t)chunk_cap * kGP * 4;
    }
};

struct Plan {
    int S, stages, chunk_cap;
    int resident;  // clusters at once
};

// A time model of a launch, in us, fitted to back-to-back launches of forced plans (4 to 6 144 units of 100 to
// 40 000 rows, groups of 1 to 16 heads, both head dims and types: 22 shapes, S up to 16, two to four stages). The
// plans it picks are 0.6% slower than the best of each shape on average, 4% at worst.
constexpr double kFixed = 3.46, kFixedNeighbour = 0.2;  // a CTA's start and end, more with each CTA on its SM
constexpr double kExchange = 2.51;                      // the cluster's
constexpr double kTileAlone = 1.33, kTileShared = 0.41; // a warp's tile of K and V: by latency, or by CTAs on its SM
constexpr double kTwoStages = 0.18;                     // more per tile with a ring of two, shared by the SM's CTAs
constexpr double kLastRound = 0.75;                     // how far a part-filled last round costs a whole one

struct Shape {
    int dim;
    bool f32, two;  // fp32 activations; groups of more than 8 heads
};

// The plan of least cost for units of up to nmax rows, S = 0 where none fits: where the logits of nmax rows are more
// than the shared memory of a cluster of 16 CTAs. bytes(rows, S, stages) is a CTA's shared memory; resident(S, bytes,
// &n) sets how many such clusters the GPU holds at once, and its failure is the plan's.
template <typename Bytes, typename Resident>
auto choose_plan(const Shape &shape, int sms, int units, int nmax, Bytes &&bytes, Resident &&resident_of, Plan *out) {
    const int tiles = (nmax - 1) / kTile + 1;
    const double weight = (shape.dim == 64 ? 0.70 : 1.0) * (shape.f32 ? 1.24 : 1.0) * (shape.two ? 1.55 : 1.0);
    decltype(resident_of(1, (size_t)0, (int *)nullptr)) err{};
    Plan &best = *out;
    best = Plan{0, 0, 0, 0};
    double best_cost = 0.0;
    for (int S : {1, 2, 3, 4, 5, 6, 8, 12, 16}) {
        if (S > tiles) break;
        const int share = (tiles + S - 1) / S;
        if (share > (int)(kMaxSmem / kTile)) continue;
        const int cap = share * kTile;
        for (int stages = kMaxStages; stages >= 2; --stages) {
            const size_t smem = bytes(cap, S, stages);
            if (smem > kMaxSmem) continue;
            int resident = 0;
            err = resident_of(S, smem, &resident);
            if (err != decltype(err){}) {
                best = Plan{0, 0, 0, 0};
                return err;
            }
            if (resident <= 0) continue;
            const double per_sm = std::min((double)resident, (double)units) * S / sms, neighbours = std::max(1.0, per_sm);
            const double tile = std::max(kTileAlone, kTileShared * neighbours) * weight + (stages == 2 ? kTwoStages / neighbours : 0.0);
            const double cta = kFixed + kFixedNeighbour * neighbours + (S > 1 ? kExchange : 0.0) +
                               tile * ((tiles + kWarps * S - 1) / (kWarps * S));
            const double rounds = (double)units / resident;
            const double cost = cta * (rounds <= 1.0 ? 1.0 : kLastRound * std::ceil(rounds) + (1.0 - kLastRound) * rounds);
            if (best.S == 0 || cost < best_cost) {
                best = Plan{S, stages, cap, resident};
                best_cost = cost;
            }
        }
    }
    return err;
}

}  // namespace q4
}  // namespace voxzip
