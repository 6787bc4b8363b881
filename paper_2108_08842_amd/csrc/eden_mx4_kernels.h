// Launches of the 4-bit kernels (arguments are checked by eden_mx4_api.hip).
#ifndef EDEN_MX4_KERNELS_H
#define EDEN_MX4_KERNELS_H

#include "eden_blocks_kernels.h"
#include "eden_mx4_device.h"

namespace eden_layers {

struct Rounding {
    eden_random random;
    uint32_t stochastic;
};
hipError_t launch_mx4_rows(uint32_t dtype, const void *x, size_t ldx, uint32_t rows, uint32_t cols, const Rounding &rounding, uint8_t *packed, hipStream_t st);
// chunks_each: chunks of 256 rows that a workgroup goes through; sums: NULL, or where each such group's sums of its rows go, ld_sums apart
hipError_t launch_mx4_columns(uint32_t dtype, const void *x, size_t ldx, uint32_t rows, uint32_t cols, const Rounding &rounding, uint8_t *packed, float *sums,
                              uint64_t ld_sums, uint32_t accumulate, uint32_t chunks_each, hipStream_t st);
hipError_t launch_mx4_restore(uint32_t dtype, const uint8_t *packed, uint32_t rows, uint32_t cols, void *x, size_t ldx, hipStream_t st);

// Products: a is rows x depth, b is cols x depth, both packed (Product::a, b); lda, ldb and the widths are not used.  side: of the tiles, 128 or 256
hipError_t launch_mx4_tiles(Op op, uint32_t dtype, const Product &p, uint32_t side, hipStream_t st);
constexpr uint32_t kFewMx4 = 64;
// up to kFewMx4 rows; x: NULL, or the matrix (dtype) that the kernel rounds itself: up to EDEN_MX4_ROWS rows, EDEN_MX4_VALUES values
hipError_t launch_mx4_few(uint32_t dtype, const Product &p, const void *x, size_t ldx, hipStream_t st);

}  // namespace eden_layers

#endif  // EDEN_MX4_KERNELS_H
