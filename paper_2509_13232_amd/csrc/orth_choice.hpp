// Which kernel forms a product of an orthogonalised update, and how many sums of squares it can leave: sizes alone decide, so this
// runs on any host.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "tile_choice.hpp"

namespace spo {

// few: a share of the contraction per wavefront; the others: tiles that the wavefronts of a workgroup share
enum class Kind { few, small, middle, large };
constexpr int64_t kOrthEdge[] = {64, 128, 192, 256};  // by kind
constexpr int kOrthWaves[] = {4, 4, 8, 8};
static inline int64_t edge_of(Kind k) { return kOrthEdge[static_cast<int>(k)]; }
static inline int waves_of(Kind k) { return kOrthWaves[static_cast<int>(k)]; }

// tiles of M x N; of a symmetric product those on and below the diagonal
__host__ __device__ __forceinline__ int64_t orth_tiles(int64_t M, int64_t N, int64_t edge, bool symmetric) {
    const int64_t m = (M + edge - 1) / edge, n = (N + edge - 1) / edge;
    return symmetric ? m * (m + 1) / 2 : m * n;
}

struct ProductSize {
    int64_t M, N, batch;  // padded sides of the output
    int steps;            // of the contraction
    bool pairs, symmetric;
    int addend, stored;   // planes read and written beside the product's operands
};

// Which kernel forms a product?  About what a launch takes, in us (measured on single matrices of 64 to 4096 and stacks of
// four of 1024 x 4096, both kinds of products; within a fifth of it but for launches of a few us):
//   tiles shared by wavefronts: rounds of workgroups on the chip x (steps x time of a step + the tile's ends); a step slows
//   down as the chip fills up.  Half of the time that the addend and the output take from and to memory comes on top.
//   a share of the contraction per wavefront: half rounds of a tile per compute unit, with pairs whole ones.
// So 64 x 64 x 64 (k, L, steps) takes 5 us instead of 7, 1024 x 1024 x 16 8.8 instead of 14 (128), 48 steps 14 instead of 33;
// 2048 x 2048 x 32 24 on tiles of 128 (64: 25, 192: 31), 4096 x 4096 x 64 symmetric 73 on 192 (253 tiles on 256 compute units;
// 85 on 256, 99 on 128), otherwise 118 on 256.
struct OrthTimes {
    Kind kind;
    int64_t slots;
    double start, step, crowd, ends;  // crowd: what a step takes longer on a chip that is full
};
constexpr OrthTimes kSmallTimes{Kind::small, 512, 3.0, 0.57, 0.30, 4.0}, kMiddleTimes{Kind::middle, 256, 3.0, 0.75, 0.25, 4.0},
    kLargeTimes{Kind::large, 256, 3.0, 1.00, 0.40, 9.0};
static inline double product_time(const OrthTimes &t, const ProductSize &p, double steps) {
    const int64_t tiles = orth_tiles(p.M, p.N, edge_of(t.kind), p.symmetric) * p.batch, full = tiles / t.slots, rest = tiles % t.slots;
    // (two small tiles share a compute unit once half of the slots are taken)
    const double fill = t.slots > kChipCUs ? std::max<int64_t>(0, rest - kChipCUs) / 256.0 : static_cast<double>(rest) / static_cast<double>(t.slots);
    const double bytes = static_cast<double>(p.M) * static_cast<double>(p.N) * static_cast<double>(p.batch) * (2 * (p.addend + p.stored));
    return t.start + static_cast<double>(full) * (steps * (t.step + t.crowd) + t.ends) +
           (rest ? steps * (t.step + t.crowd * fill) + t.ends : 0.0) + 0.5 * bytes / 5.0e6;
}
// (tiles of 192 take rows along the contraction only: the symmetric products)
static inline Kind product_kind(const ProductSize &p) {
    const double steps = p.steps * (p.pairs ? 3 : 1);
    const int64_t tiles = orth_tiles(p.M, p.N, edge_of(Kind::few), p.symmetric) * p.batch;
    const double halves = std::max(1.0, static_cast<double>((2 * tiles + kChipCUs - 1) / kChipCUs) * 0.5);
    Kind best = Kind::few;
    double least = p.pairs ? 4.0 + static_cast<double>((tiles + kChipCUs - 1) / kChipCUs) * (p.steps * 0.475 + 2.4)
                           : 4.0 + halves * (steps * 0.2 + 2.4);
    auto offer = [&](const OrthTimes &t) {
        const double time = product_time(t, p, steps);
        if (time < least) {
            least = time;
            best = t.kind;
        }
    };
    offer(kSmallTimes);
    if (p.symmetric) offer(kMiddleTimes);
    offer(kLargeTimes);
    return best;
}

// Sides are rounded up to steps of the contraction.
static inline int64_t padded(int64_t n) { return (n + kStep - 1) / kStep * kStep; }
// Where the smaller side is one step of the contraction, launches are all that counts, and so few roundings do not
// average out (one of 1 x 1: 4e-3): always pairs.
static inline bool as_pairs(int64_t k, bool asked) { return asked || k <= kStep; }

// The products of a step on X of k x L (padded): A = X X^T, B = c A A + ..., X <- B X + ...
struct OrthKinds {
    Kind gram, poly, update;
};
static inline OrthKinds orth_kinds(int64_t k, int64_t L, int64_t batch, bool pairs) {
    const int planes = pairs ? 2 : 1;
    return {product_kind({k, k, batch, static_cast<int>(L / kStep), pairs, true, 0, planes}),
            product_kind({k, k, batch, static_cast<int>(k / kStep), pairs, true, planes, planes}),
            product_kind({k, L, batch, static_cast<int>(k / kStep), pairs, false, 2, 2})};
}

// Sums of squares that a product of k x L leaves per matrix, one of every wavefront of every tile, and room for those of any kind
// (not always the smallest tiles' are the most: one tile of eight wavefronts holds all of 64 x 64).
static inline int64_t square_sums(int64_t k, int64_t L, Kind kind) { return orth_tiles(k, L, edge_of(kind), false) * waves_of(kind); }
static inline int64_t square_room(int64_t k, int64_t L) {
    return std::max({square_sums(k, L, Kind::few), square_sums(k, L, Kind::small), square_sums(k, L, Kind::middle), square_sums(k, L, Kind::large)});
}

}  // namespace spo
