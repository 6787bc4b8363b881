// Element-wise launches over a matrix: a thread has eight neighbouring columns.
#ifndef EDEN_LAYERS_SPREAD_H
#define EDEN_LAYERS_SPREAD_H

#include "eden_layers_kernels.h"

#include <algorithm>

namespace eden_layers {

constexpr uint32_t kSpreadThreads = 256;

// threads of a row (a power of two, 4 at least: a block's) and workgroups along it
struct Spread {
    uint32_t shift, segments;
    uint64_t groups;
};
inline Spread spread(uint32_t rows, uint32_t cols) {
    const uint32_t units = (uint32_t)blocks_of(cols) * 4;
    uint32_t shift = 2;
    while (shift < 8 && (1u << shift) < units) ++shift;
    const uint32_t segments = (units + (1u << shift) - 1) >> shift, rows_each = kSpreadThreads >> shift;
    return {shift, segments, (uint64_t)((rows + rows_each - 1) / rows_each) * segments};
}
struct Place {
    uint32_t row, col;
};
// `before`: workgroups of the call's launches before this one
__device__ inline Place place(uint32_t shift, uint32_t segments, uint32_t before) {
    const uint32_t number = before + blockIdx.x, group = number / segments, segment = number - group * segments;
    return {group * (kSpreadThreads >> shift) + (threadIdx.x >> shift), ((segment << shift) + (threadIdx.x & ((1u << shift) - 1))) * 8};
}
__device__ inline int valid_of(uint32_t col, uint32_t cols) { return col < cols ? (int)min(8u, cols - col) : 0; }

template <class F> inline void for_type(uint32_t dtype, F f) {
    if (dtype == EDEN_F32) f(std::integral_constant<uint32_t, EDEN_F32>());
    else if (dtype == EDEN_F16) f(std::integral_constant<uint32_t, EDEN_F16>());
    else f(std::integral_constant<uint32_t, EDEN_BF16>());
}
// f(workgroups before a launch, workgroups of it) until all are launched
template <class F> inline hipError_t launches(const Spread &s, F f) {
    hipError_t e = hipSuccess;
    for (uint64_t before = 0; before < s.groups && e == hipSuccess; before += most_groups(kSpreadThreads)) {
        f((uint32_t)before, (uint32_t)std::min(s.groups - before, most_groups(kSpreadThreads)));
        e = hipGetLastError();
    }
    return e;
}

}  // namespace eden_layers

#endif  // EDEN_LAYERS_SPREAD_H
