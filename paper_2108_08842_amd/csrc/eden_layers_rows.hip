// eden_linear for up to 64 rows (single tokens, a few tokens at a time): the weights are read once and everything else is small.
//
// Bound by memory: w's bytes.  A workgroup has 16 or 32 columns of the result and all rows; its eight waves go through the depth in turn, 256 bytes of
// each of w's rows at a time, from memory to the matrix cores' registers without the LDS (lane l holds row l % 16 of w and 16 bytes of the
// depth, so a load takes 64 bytes of 16 rows; the next chunk is on its way while one is multiplied).  16 x 16 products; fp32 operands
// are multiplied in fp32.  The waves' sums meet in the LDS, in the order of the waves.
#include "eden_layers_kernels.h"

namespace eden_layers {
namespace {

constexpr int kWaves = 8, kSteps = 4;              // steps (loads of 64 bytes a row) of a chunk

template <uint32_t DTYPE> __device__ inline f32x4 multiply16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (DTYPE == EDEN_F32) {                             // depths 4 (l / 16) + i, i = 0 .. 3, of 16: any order does if both operands have it
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = a[i], y = b[i];
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x), __uint_as_float(y), c, 0, 0, 0);
        }
        return c;
    } else if constexpr (DTYPE == EDEN_F16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
}

// COLS: sixteens of columns; ROWS: sixteens of rows
template <uint32_t DTYPE, int COLS, int ROWS> __global__ __launch_bounds__(kWaves * 64) void k_rows(const Product p) {
    using T = typename Elem<DTYPE>::type;
    constexpr int kPiece = 16 / Elem<DTYPE>::kBytes, kStep = 4 * kPiece, kChunk = kSteps * kStep;
    __shared__ f32x4 sums[kWaves][COLS][ROWS][64];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col0 = blockIdx.x * (16 * COLS);
    const T *w[COLS], *x[ROWS];
    bool has_w[COLS], has_x[ROWS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
        const uint32_t col = col0 + c * 16 + (lane & 15);
        has_w[c] = col < p.cols;
        w[c] = static_cast<const T *>(p.b) + (size_t)(has_w[c] ? col : 0) * p.ldb + (lane >> 4) * kPiece;
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t row = r * 16 + (lane & 15);
        has_x[r] = row < p.rows;
        x[r] = static_cast<const T *>(p.a) + (size_t)(has_x[r] ? row : 0) * p.lda + (lane >> 4) * kPiece;
    }

    f32x4 acc[COLS][ROWS] = {};
    struct Chunk { Vec<T, kPiece> w[kSteps][COLS], x[kSteps][ROWS]; };
    auto load = [&](Chunk &to, uint32_t k) {                       // what is outside the operands is 0
        const bool full = k + kChunk <= p.depth;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const uint32_t at = k + s * kStep, piece = at + (lane >> 4) * kPiece;
            const int valid = full ? kPiece : piece < p.depth ? (int)min((uint32_t)kPiece, p.depth - piece) : 0;
#pragma unroll
            for (int c = 0; c < COLS; ++c) to.w[s][c] = load_some<T, kPiece>(w[c] + at, has_w[c] ? valid : 0);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) to.x[s][r] = load_some<T, kPiece>(x[r] + at, has_x[r] ? valid : 0);
        }
    };
    auto multiply = [&](const Chunk &from) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int c = 0; c < COLS; ++c)
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
                    acc[c][r] = multiply16<DTYPE>(__builtin_bit_cast(u32x4, from.w[s][c]), __builtin_bit_cast(u32x4, from.x[s][r]), acc[c][r]);
    };
    constexpr uint32_t kStride = kWaves * kChunk;
    Chunk even, odd;
    uint32_t k = wave * kChunk;
    if (k < p.depth) {
        load(even, k);
        for (;;) {
            if (k + kStride < p.depth) load(odd, k + kStride);
            multiply(even);
            if (k + kStride >= p.depth) break;
            k += 2 * kStride;
            if (k < p.depth) load(even, k);
            multiply(odd);
            if (k >= p.depth) break;
        }
    }
#pragma unroll
    for (int c = 0; c < COLS; ++c)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) sums[wave][c][r][lane] = acc[c][r];
    __syncthreads();

    // thread -> row and four columns; 4 COLS threads side by side have a row (COLS = 2: a block of a checkpoint)
    constexpr int kQuads = 4 * COLS;
    for (int t = tid; t < 16 * ROWS * kQuads; t += kWaves * 64) {
        const int row = t / kQuads, quad = t % kQuads;
        f32x4 sum = sums[0][quad >> 2][row >> 4][(quad & 3) * 16 + (row & 15)];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) sum += sums[i][quad >> 2][row >> 4][(quad & 3) * 16 + (row & 15)];
        const uint32_t col = col0 + quad * 4;
        const int valid = (uint32_t)row < p.rows && col < p.cols ? (int)min(4u, p.cols - col) : 0;
        float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        if (valid) finish_bias<kForward, DTYPE>(p.finish, col, valid, v);
        if constexpr (COLS == 2)
            if (p.finish.codes_out) {
                uint32_t largest = 0;
                float z[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z[e] = e < valid ? v[e] : 0.0f;
                    largest = max(largest, magnitude_bits(z[e]));
                }
#pragma unroll
                for (int step = 1; step < 8; step *= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, step));
                const uint32_t exponent = block_exponent(largest);
                if ((uint32_t)row < p.rows) {                      // (the workgroup has a column: its block exists)
                    const size_t block = (size_t)row * p.finish.blocks + col0 / kBlock;
                    if (quad == 0) p.finish.exps_out[block] = (uint8_t)exponent;
                    *reinterpret_cast<uint32_t *>(p.finish.codes_out + block * kBlock + quad * 4) = codes4(z, exponent);
                }
            }
        if (valid) finish_store<kForward, DTYPE>(p.finish, row, col, valid, v);
    }
}

template <uint32_t DTYPE, int COLS> void launch(const Product &p, hipStream_t st) {
    const uint32_t grid = (p.cols + 16 * COLS - 1) / (16 * COLS);
    if (p.rows <= 16) k_rows<DTYPE, COLS, 1><<<grid, kWaves * 64, 0, st>>>(p);
    else if (p.rows <= 32) k_rows<DTYPE, COLS, 2><<<grid, kWaves * 64, 0, st>>>(p);
    else k_rows<DTYPE, COLS, 4><<<grid, kWaves * 64, 0, st>>>(p);
}

}  // namespace

hipError_t launch_rows(uint32_t dtype, const Product &p, bool wide, hipStream_t st) {
    if (dtype == EDEN_F32) wide ? launch<EDEN_F32, 2>(p, st) : launch<EDEN_F32, 1>(p, st);
    else if (dtype == EDEN_F16) wide ? launch<EDEN_F16, 2>(p, st) : launch<EDEN_F16, 1>(p, st);
    else wide ? launch<EDEN_BF16, 2>(p, st) : launch<EDEN_BF16, 1>(p, st);
    return hipGetLastError();
}

}  // namespace eden_layers
