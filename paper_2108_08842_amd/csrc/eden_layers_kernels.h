// Launches of the layer kernels (arguments are checked by eden_layers_api.hip).
#ifndef EDEN_LAYERS_KERNELS_H
#define EDEN_LAYERS_KERNELS_H

#include "eden_layers_device.h"

namespace eden_layers {

// A product out[r][c] = sum_d A(r, d) B(c, d):
//   kForward     A = x (rows x depth), B = w (cols x depth)
//   kInputGrad   A = dz (rows x depth), B = w (depth x cols)
//   kWeightGrad  A = dy (depth x rows), B = checkpoint of x (depth x cols): codes and exponents
struct Product {
    const void *a, *b;
    size_t lda, ldb;               // ldb of a checkpoint: bytes between rows of codes
    uint32_t a_width, b_width;     // elements of a row of memory that may be read (in a copy more than the operand has: zeros)
    const uint8_t *b_exps;
    uint32_t b_blocks;
    uint32_t rows, cols, depth;
    Finish finish;
    float *row_sums;               // kWeightGrad: bias_grad or NULL
    float *partial;                // splits > 1: splits x rows x partial_ld sums, then splits x rows of row_sums
    uint32_t partial_ld;
    uint32_t splits, split_depth;  // of a split, a multiple of kSplitUnit
    uint32_t before;               // eden_linear of few rows: workgroups of the launches before this one
};

// Workgroups of a launch: it has less than 2^32 threads.
constexpr uint64_t most_groups(uint32_t threads) { return 0xFFFFFFFFull / threads; }
constexpr uint32_t kSplitUnit = 64;   // the depth is split at multiples of this
// (a result without columns still has row sums: one tile)
__host__ __device__ inline uint32_t tiles_of(uint32_t n, uint32_t side) { return n ? (n + side - 1) / side : 1; }

// side: of the tiles, 64 or 128
hipError_t launch_tiles(Op op, uint32_t dtype, const Product &p, uint32_t side, hipStream_t st);
// side: 128 or 256
hipError_t launch_direct(Op op, uint32_t dtype, const Product &p, uint32_t side, hipStream_t st);
// fp32 operands, tiles of 128 x 128
hipError_t launch_direct_fp32(Op op, const Product &p, hipStream_t st);
constexpr uint32_t kFewRows = 16;
hipError_t launch_rows(uint32_t dtype, const Product &p, hipStream_t st);
hipError_t launch_join(Op op, uint32_t dtype, const Product &p, hipStream_t st);

// rows x cols at distance ld -> rows at distance `to_ld`, zeros behind the columns
hipError_t launch_copy_rows(uint32_t dtype, const void *from, size_t ld, uint32_t rows, uint32_t cols, void *to, uint32_t to_ld, hipStream_t st);

hipError_t launch_save(uint32_t dtype, const void *x, size_t ldx, uint32_t rows, uint32_t cols, uint8_t *codes, uint8_t *exps, hipStream_t st);
hipError_t launch_restore(uint32_t dtype, const uint8_t *codes, const uint8_t *exps, uint32_t rows, uint32_t cols, void *x, size_t ldx, hipStream_t st);
hipError_t launch_activation_grad(uint32_t dtype, const void *dy, size_t ldy, const uint8_t *codes, const uint8_t *exps, uint32_t activation,
                                  void *dz, size_t ldz, uint32_t rows, uint32_t cols, hipStream_t st);

}  // namespace eden_layers

#endif  // EDEN_LAYERS_KERNELS_H
