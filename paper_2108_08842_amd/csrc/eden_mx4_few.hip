// eden_mx4_linear for up to 16 rows, where it pays 64 (single tokens, some tokens at a time): the weights are read once and everything else is small.  Bound by memory: w's bytes.
//
// A workgroup has 32 columns of the result (16 of a narrow one) and all rows, in sixteens; its eight waves go through the chunks of 256 in turn, from memory to the matrix cores' registers without the LDS: lane l holds
// row l % 16 of either operand and blocks 2 (l / 16), + 1 of the chunk, so a load takes whole lines of 16 rows.  The waves' sums meet in the LDS, in the order of the waves.
// Up to 16384 values are rounded by every workgroup itself, into the LDS: the weights' first loads are on their way meanwhile.
//
// In a captured graph, bf16 next to 16384 x 4096 (35.7 MB): one row 8.7 us = 4.1 TB/s, four 10.7, sixteen (rounded by a launch before) 12.6; next to 1024 x 1024 3.5, four 3.7, sixteen 4.9.  With a launch of their
// own to round x: four rows of 4096 11.6, four of 1024 5.5, sixteen 6.1; eight rows of 4096 rounded by every workgroup 13.4 against 11.9.
// Above sixteen rows, x rounded before, against tiles: 32 rows next to 4096 x 4096 6.3 us and 10.8, 8192 x 4096 7.7 and 14.0, 16384 x 4096 13.1 and 14.9, 4096 x 8192 9.9 and 11.8, 64 rows next to 4096 x 4096 9.5 and 14.2,
// 5000 x 2048 6.6 and 9.5, 1024 x 1024 4.9 and 6.6; 1024 x 4096 is the other way round, 9.1 and 8.2.  Each workgroup reads all of x from the L2: deep sums (32 rows next to 4096 x 16384 16.4 and 13.8) and results of several rounds of
// workgroups (32000 x 2048 14.7 and 11.1) are better off with tiles.
#include "eden_layers_product.h"
#include "eden_layers_spread.h"
#include "eden_mx4_kernels.h"

namespace eden_layers {
namespace {

constexpr int kWaves = 8;
constexpr uint32_t kNarrow = 16 * 256;                             // columns that 256 CUs have in sixteens

struct Piece4 {
    u32x4 code[2];
    uint32_t exps;                                                 // of the two blocks
};
__device__ inline f32x4 multiply4(const Piece4 &a, const Piece4 &b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const i32x8 x = {(int)a.code[i][0], (int)a.code[i][1], (int)a.code[i][2], (int)a.code[i][3], 0, 0, 0, 0};
        const i32x8 y = {(int)b.code[i][0], (int)b.code[i][1], (int)b.code[i][2], (int)b.code[i][3], 0, 0, 0, 0};
        if (i == 0) c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)a.exps, 0, (int)b.exps);
        else c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 1, (int)a.exps, 1, (int)b.exps);
    }
    return c;
}

// OWN: x comes as values; kCols: sixteens of columns; kRows: of rows
template <uint32_t DTYPE, bool OWN, int kCols, int kRows> __global__ __launch_bounds__(kWaves * 64) void k_mx4_few(const Product p, const typename Elem<DTYPE>::type *x, size_t ldx) {
    constexpr int kRun = 4 / kCols;                                // chunks on their way at a time
    static_assert(!OWN || kRows == 1, "values are rounded into the LDS for 16 rows");
    __shared__ f32x4 sums[kWaves][kRows][kCols][64];
    __shared__ __attribute__((aligned(16))) uint8_t mine[OWN ? EDEN_MX4_VALUES / 2 + EDEN_MX4_ROWS * kChunkBytes : 16];
    __shared__ __attribute__((aligned(16))) uint8_t my_exps[OWN ? EDEN_MX4_VALUES / kBlock + EDEN_MX4_ROWS * kChunkBlocks : 16];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t chunks = chunks_of(p.depth), col0 = (p.before + blockIdx.x) * (16 * kCols), quarter = lane >> 4;
    const uint8_t *w = static_cast<const uint8_t *>(p.b), *w_exps = w + mx4_codes_bytes(p.cols, p.depth);
    const uint8_t *a = static_cast<const uint8_t *>(p.a), *a_exps = a + (OWN ? 0 : mx4_codes_bytes(p.rows, p.depth));
    bool has_w[kCols];
    uint32_t col[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        has_w[c] = col0 + c * 16 + (lane & 15) < p.cols;
        col[c] = has_w[c] ? col0 + c * 16 + (lane & 15) : 0;
    }

    struct Run { Piece4 w[kRun][kCols]; };
    auto load = [&](Run &to, uint32_t chunk) {                     // what is outside the operands is 0
#pragma unroll
        for (int r = 0; r < kRun; ++r) {
            const uint32_t at = chunk + r * kWaves;
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                if (at < chunks && has_w[c]) {
                    const uint8_t *from = w + ((size_t)col[c] * chunks + at) * kChunkBytes + quarter * 32;
                    to.w[r][c].code[0] = *reinterpret_cast<const u32x4 *>(from);
                    to.w[r][c].code[1] = *reinterpret_cast<const u32x4 *>(from + 16);
                    to.w[r][c].exps = *reinterpret_cast<const uint16_t *>(w_exps + exps_at(p.cols, col[c], at) + quarter * 2);
                } else {
                    to.w[r][c] = {};
                }
            }
        }
    };
    f32x4 acc[kRows][kCols] = {};
    auto multiply = [&](const Run &from, uint32_t chunk) {
#pragma unroll
        for (int r = 0; r < kRun; ++r) {
            const uint32_t at = chunk + r * kWaves;
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                const uint32_t row = q * 16 + (lane & 15);
                Piece4 v = {};
                if (at < chunks && row < p.rows) {
                    const uint8_t *codes = (OWN ? mine : a) + ((size_t)row * chunks + at) * kChunkBytes + quarter * 32;
                    v.code[0] = *reinterpret_cast<const u32x4 *>(codes);
                    v.code[1] = *reinterpret_cast<const u32x4 *>(codes + 16);
                    v.exps = *reinterpret_cast<const uint16_t *>(OWN ? my_exps + ((size_t)row * chunks + at) * kChunkBlocks + quarter * 2 : a_exps + exps_at(p.rows, row, at) + quarter * 2);
                }
#pragma unroll
                for (int c = 0; c < kCols; ++c) acc[q][c] = multiply4(from.w[r][c], v, acc[q][c]);
            }
        }
    };
    constexpr uint32_t kStride = kWaves * kRun;
    Run even_run, odd_run;
    uint32_t chunk = wave;
    load(even_run, chunk);
    if constexpr (OWN) {
        const uint32_t eights = chunks * (kChunk / 8);             // of a row
        for (uint32_t i = tid; i < p.rows * eights; i += kWaves * 64) {      // (whole waves: a row has a multiple of 32, and four lanes have a block)
            const uint32_t r = i / eights, at = i - r * eights;
            Eight<DTYPE> in;
            in.load(x + r * ldx, at * 8, at * 8 < p.depth ? (int)min(8u, p.depth - at * 8) : 0);
            float v[8];
            uint32_t largest = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = in[e];
                largest = max(largest, magnitude_bits(v[e]));
            }
            const uint32_t t = mx4_exponent(largest_of_quad(largest));
            *reinterpret_cast<uint32_t *>(mine + i * 4) = mx4_codes(v, t);
            if (i % 4 == 0) my_exps[i / 4] = (uint8_t)t;
        }
        __syncthreads();
    }
    while (chunk < chunks) {
        if (chunk + kStride < chunks) load(odd_run, chunk + kStride);
        multiply(even_run, chunk);
        chunk += kStride;
        if (chunk >= chunks) break;
        if (chunk + kStride < chunks) load(even_run, chunk + kStride);
        multiply(odd_run, chunk);
        chunk += kStride;
    }
#pragma unroll
    for (int q = 0; q < kRows; ++q)
#pragma unroll
        for (int c = 0; c < kCols; ++c) sums[wave][q][c][lane] = acc[q][c];
    __syncthreads();

    // thread -> row and four columns; eight threads side by side have a row, a block of a checkpoint
    constexpr int kQuads = 4 * kCols;
    if (tid < 16 * kRows * kQuads) {
        const int r = tid / kQuads, quad = tid % kQuads, place = (quad & 3) * 16 + r % 16;
        f32x4 sum = sums[0][r / 16][quad >> 2][place];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) sum += sums[i][r / 16][quad >> 2][place];
        const uint32_t at = col0 + quad * 4;
        const int valid = (uint32_t)r < p.rows && at < p.cols ? (int)min(4u, p.cols - at) : 0;
        float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        finish_quad<(kCols == 2), DTYPE>(p, r, col0, at, valid, v);
    }
}

}  // namespace

hipError_t launch_mx4_few(uint32_t dtype, const Product &product, const void *x, size_t ldx, hipStream_t st) {
    Product p = product;
    // 16 columns a workgroup where each CU has one of them at most (a checkpoint's block is 32): one row next to 4096 x 16384 9.5 us against 13.5, 4096 x 4096 4.4 and 5.1, 1024 x 8192 4.8 and 6.9.  With more,
    // 5000 x 2048 takes 5.0 against 4.1, 8192 x 4096 6.8 against 5.7: the second workgroup of a CU waits as long as the first.
    const uint32_t wide = p.cols <= kNarrow && p.rows <= 32 && p.finish.codes_out == nullptr ? 16 : 32;
    const uint32_t groups = (p.cols + wide - 1) / wide;
    hipError_t e = hipSuccess;
    for (p.before = 0; p.before < groups && e == hipSuccess; p.before += (uint32_t)most_groups(kWaves * 64)) {
        const uint32_t now = min(groups - p.before, (uint32_t)most_groups(kWaves * 64));
        // (four sixteens of rows next to one of columns take more registers than there are)
        auto typed = [&](auto t, auto cols) {
            constexpr uint32_t DTYPE = decltype(t)::value;
            constexpr int COLS = decltype(cols)::value;
            using T = typename Elem<DTYPE>::type;
            if (x) k_mx4_few<DTYPE, true, COLS, 1><<<now, kWaves * 64, 0, st>>>(p, static_cast<const T *>(x), ldx);
            else if (p.rows <= 16) k_mx4_few<DTYPE, false, COLS, 1><<<now, kWaves * 64, 0, st>>>(p, nullptr, 0);
            else if (p.rows <= 32) k_mx4_few<DTYPE, false, COLS, 2><<<now, kWaves * 64, 0, st>>>(p, nullptr, 0);
            else k_mx4_few<DTYPE, false, 2, 4><<<now, kWaves * 64, 0, st>>>(p, nullptr, 0);
        };
        for_type(dtype, [&](auto t) {
            if (wide == 16) typed(t, std::integral_constant<int, 1>());
            else typed(t, std::integral_constant<int, 2>());
        });
        e = hipGetLastError();
    }
    return e;
}

}  // namespace eden_layers
