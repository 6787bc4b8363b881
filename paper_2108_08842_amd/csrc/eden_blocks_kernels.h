// Launches of the block operators (arguments are checked by eden_blocks_api.hip).
#ifndef EDEN_BLOCKS_KERNELS_H
#define EDEN_BLOCKS_KERNELS_H

#include "eden_blocks_device.h"
#include "eden_layers_kernels.h"

namespace eden_layers {

// Lanes that share a row and chunks of eight columns each of them has: LANES * CHUNKS * 8 columns at least
struct RowShape {
    int lanes, chunks;
};
inline RowShape row_shape(uint32_t cols) {
    const uint32_t eights = (cols + 7) / 8;
    if (eights > 1024) return {1024, 2};
    int lanes = 8;
    while ((uint32_t)lanes < eights) lanes *= 2;
    return {lanes, 1};
}
// f(integral constants LANES, CHUNKS)
template <class F> inline void for_shape(RowShape s, F f) {
    auto with = [&](auto lanes) { f(lanes, std::integral_constant<int, 1>()); };
    if (s.chunks == 2) f(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
    else if (s.lanes == 8) with(std::integral_constant<int, 8>());
    else if (s.lanes == 16) with(std::integral_constant<int, 16>());
    else if (s.lanes == 32) with(std::integral_constant<int, 32>());
    else if (s.lanes == 64) with(std::integral_constant<int, 64>());
    else if (s.lanes == 128) with(std::integral_constant<int, 128>());
    else if (s.lanes == 256) with(std::integral_constant<int, 256>());
    else if (s.lanes == 512) with(std::integral_constant<int, 512>());
    else with(std::integral_constant<int, 1024>());
}

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
// one for each type, so that they are compiled side by side
template <uint32_t DTYPE> hipError_t launch_block_grad(const GradArgs &args, hipStream_t st);
extern template hipError_t launch_block_grad<EDEN_F32>(const GradArgs &, hipStream_t);
extern template hipError_t launch_block_grad<EDEN_F16>(const GradArgs &, hipStream_t);
extern template hipError_t launch_block_grad<EDEN_BF16>(const GradArgs &, hipStream_t);

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
