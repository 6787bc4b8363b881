// Launches of the block operators (arguments are checked by eden_blocks_api.hip).
#ifndef EDEN_BLOCKS_KERNELS_H
#define EDEN_BLOCKS_KERNELS_H

#include "eden_blocks_device.h"
#include "eden_layers_kernels.h"

namespace eden_layers {

// Lanes that share a row and chunks of eight columns each of them has: LANES * CHUNKS * 8 columns at least (rows of less than eight: one lane).  Two chunks a lane where a row takes
// more than a wave's eights: what a wave does once for a row (sums over its lanes, addresses) then serves twice as many values.
// WIDE: lanes of the longest rows; FROM: lanes from which on a lane has two chunks before a row gets more lanes
template <int WIDE, int FROM> struct RowShape {
    int lanes, chunks;
    explicit RowShape(uint32_t cols) {
        const int eights = (int)((cols + 7) / 8);
        if (cols < 8) {
            lanes = 1, chunks = 1;
            return;
        }
        for (lanes = 8; lanes < eights && lanes < FROM; lanes *= 2) {}
        for (; lanes < WIDE && lanes * 2 < eights; lanes *= 2) {}
        for (chunks = 1; lanes * chunks < eights; chunks *= 2) {}
    }
    // f(LANES, CHUNKS, RAGGED), integral constants
    template <class F> void use(uint32_t cols, F f) const {
        auto with = [&](auto n, auto c) {
            constexpr int LANES = decltype(n)::value, CHUNKS = decltype(c)::value;
            if constexpr ((CHUNKS == 1 ? LANES <= FROM : LANES >= FROM && LANES <= WIDE) && LANES * (CHUNKS / 2) * 8 < EDEN_MOST_COLUMNS) {
                if (lanes != LANES || chunks != CHUNKS) return;
                if (cols % 8) f(n, c, std::true_type());
                else f(n, c, std::false_type());
            }
        };
        auto one = [&](auto n) { with(n, std::integral_constant<int, 1>()); };
        auto two = [&](auto n) { with(n, std::integral_constant<int, 2>()); };
        if (lanes == 1) f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>(), std::true_type());
        one(std::integral_constant<int, 8>()), one(std::integral_constant<int, 16>()), one(std::integral_constant<int, 32>()), one(std::integral_constant<int, 64>());
        one(std::integral_constant<int, 128>()), one(std::integral_constant<int, 256>()), one(std::integral_constant<int, 512>()), one(std::integral_constant<int, 1024>());
        two(std::integral_constant<int, 64>()), two(std::integral_constant<int, 128>()), two(std::integral_constant<int, 256>()), two(std::integral_constant<int, 512>());
        two(std::integral_constant<int, 1024>());
    }
};
using JoinShape = RowShape<1024, 64>;
// A gradient with the sums of the gate and of two norms takes more registers than 1024 lanes have (128 each): up to 8192 columns it has 512 lanes at most; beyond, two of its sums are
// in the LDS (4096 x 16384 bf16, both norms rms, gate, dropout: 461 -> 320 us against 512 lanes with four chunks each and all sums in registers, which spilled; layer norms 890 -> 525).
using GradShape = RowShape<1024, 1024>;
using FullGradShape = RowShape<1024, 512>;

// How the rows of a gradient are shared out: `gates` groups of `group_rows` rows.  Either splits workgroups share a group, or a workgroup has
// `groups_each` whole ones.
struct Share {
    uint32_t gates, group_rows, splits, groups_each, workers;
};
enum Sums : int { kGateSum = 0, kPostWeight, kPostBias, kPreWeight, kPreBias, kAllSums };
struct GradArgs {
    eden_join_grad_args a;
    Share share;
    float *sums[kAllSums];         // where a sum goes or NULL; workers > 1: its parts in the workspace, one a worker (kGateSum with splits 1: the result itself)
    uint64_t ld_sums;              // of the parts
    uint32_t needs_f;
};

hipError_t launch_dropout(uint32_t dtype, const void *x, size_t ldx, void *y, size_t ldy, uint32_t rows, uint32_t cols, const eden_random &random, hipStream_t st);
hipError_t launch_block_join(const eden_join_args &args, hipStream_t st);
// one for each type and kind of norm behind the branch (-1: no branch), so that they are compiled side by side
template <uint32_t DTYPE, int POST> hipError_t launch_block_grad(const GradArgs &args, hipStream_t st);

// out[c] (+)= sum of parts x cols partial sums in their order, for several sums at once
struct SumsOf {
    const float *from;
    float *to;
};
struct SumsArgs {
    SumsOf of[kAllSums];
    uint64_t ld_from, ld_to[kAllSums];
    uint32_t count, cols, parts[kAllSums], rows[kAllSums];         // rows: results, each from its own parts
    uint32_t first[kAllSums + 1];                                  // workgroups before those of each
    uint32_t accumulate;
};
hipError_t launch_sums(const SumsArgs &args, hipStream_t st);

}  // namespace eden_layers

#endif  // EDEN_BLOCKS_KERNELS_H
