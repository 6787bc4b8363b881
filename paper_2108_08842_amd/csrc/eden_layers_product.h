// What the matrix-core kernels of the layer operators share: bf16 terms, places in the LDS, operands of a 32 x 32 x 16 product, the workgroup's
// place in the result, and the end of a 32 x 32 tile.
#ifndef EDEN_LAYERS_PRODUCT_H
#define EDEN_LAYERS_PRODUCT_H

#include "eden_layers_kernels.h"

namespace eden_layers {

// Byte offset of a 16-byte piece.  Rows of the depth: 16 neighbouring rows at one depth lie in different banks.
template <int DEPTH> __device__ inline int piece_of_row(int row, int piece) {
    return row * (DEPTH * 2) + ((DEPTH == 64 ? piece ^ ((row >> 1) & 7) : piece ^ ((row >> 2) & 3)) << 4);
}
// Rows of columns: 32 columns at four neighbouring depths do.
template <int WIDTH> __device__ inline int piece_of_depth(int depth, int piece) {
    return depth * (WIDTH * 2) + ((WIDTH == 64 ? piece ^ (2 * (depth & 2)) : piece ^ (4 * (depth & 3))) << 4);
}

// Next to an operand of one term, where all products are taken: x = term + rest, term = the upper 16 bits (exact; an infinity leaves nothing, a NaN a NaN)
__device__ inline float take_term(float &x) {
    const float term = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
    const float rest = x - term;
    x = __builtin_isinf(x) ? 0.0f : rest;
    return term;
}
__device__ inline uint32_t upper_halves(float lo, float hi) { return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u); }

// Between two fp32 operands, where the products of second and third terms are left out: the next term of a and of b, side by side, and what they leave.  `first`: the
// upper 16 bits (a number that rounds to an infinity keeps its size; of an infinity the other terms are NaN).  The others are the nearest bf16 numbers, so that the
// third ones are at most 2^-16 of the power of two below |a| and of either sign: what is left out of a product is below 2^-22 of it, 2^-25.4 in the mean square (an
// fp32 rounding: 2^-25.2).  All terms cut off: up to 2^-21.03, always towards zero.  The first one to the nearest as well: below 2^-24, but with the numbers next to fp32's largest
// taken care of 4096 x 8192 x 4096 takes 6.4% longer.
__device__ inline uint32_t take_nearest(float &a, float &b, bool first) {
    const uint32_t pair = first ? upper_halves(a, b) : __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
    a -= __uint_as_float(pair << 16);
    b -= __uint_as_float(pair & 0xFFFF0000u);
    return pair;
}

__device__ inline u32x4 code_values(uint32_t c0, uint32_t c1, float unit) {
    float a[4], b[4];
    values4(c0, unit, a);
    values4(c1, unit, b);
    return u32x4{upper_halves(a[0], a[1]), upper_halves(a[2], a[3]), upper_halves(b[0], b[1]), upper_halves(b[2], b[3])};
}

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Operand of a 32 x 32 x 16 product: lane l holds index base + l % 32 and depths 8 (l / 32) .. + 7 of the 16 from `depth` on.
template <bool STRIDED, int DEPTH, int WIDTH> __device__ inline u32x4 fragment(const char *plane, int base, int depth, int lane) {
    if constexpr (!STRIDED) {
        const int row = base + (lane & 31), piece = (depth >> 3) + (lane >> 5);
        return *reinterpret_cast<const u32x4 *>(plane + piece_of_row<DEPTH>(row, piece));
    } else {
        // transposing reads: 16 lanes read four depths of 16 columns and get four depths of one column each
        const int col = base + (lane & 16) + (lane & 3) * 4, d = depth + (lane >> 5) * 8 + ((lane & 15) >> 2);
        const char *p = plane + piece_of_depth<WIDTH>(d, col >> 3) + (col & 7) * 2;
        const char *q = plane + piece_of_depth<WIDTH>(d + 4, col >> 3) + (col & 7) * 2;
        union { s16x4 h[2]; u32x4 w; } r;
        r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
        r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)q);
        return r.w;
    }
}

template <bool HALF> __device__ inline f32x16 multiply(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Workgroup -> tile: workgroups go round the eight XCDs in turn; each XCD gets a run of neighbouring tiles, eight row tiles at a time, so that its L2
// serves their operands.
__device__ inline void place_of(uint32_t id, uint32_t total, uint32_t row_tiles, uint32_t col_tiles, uint32_t &split, uint32_t &row_tile, uint32_t &col_tile) {
    const uint32_t xcd = id & 7u, each = total >> 3, more = total & 7u;
    const uint32_t t = xcd * each + min(xcd, more) + (id >> 3);
    const uint32_t tiles = row_tiles * col_tiles;
    split = t / tiles;
    const uint32_t tile = t - split * tiles, group = tile / (8 * col_tiles), first = group * 8, height = min(8u, row_tiles - first);
    const uint32_t within = tile - group * 8 * col_tiles;
    row_tile = first + within % height;
    col_tile = within / height;
}

// Orders a wave's own accesses to the LDS.
__device__ inline void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The end of 32 x 32 T sums that a wave has left in the LDS: eight columns a lane, so that four lanes have a checkpoint's block and a row's
// results leave in pieces of 16 bytes side by side; up to four rows at a time.
template <int T> constexpr int kRowFloats = 32 * T + 4;            // the four: neighbouring rows begin in different banks
template <int OP, uint32_t DTYPE, int T, bool STREAM = false>
__device__ inline void finish_rows(const Product &p, const float *sums, uint32_t row0, uint32_t col0, int lane, uint32_t split) {
    constexpr int kLanes = 4 * T, kStep = 64 / kLanes;             // lanes of a row; rows side by side
    constexpr int kRows = 32 / kStep < 4 ? 32 / kStep : 4;
    const uint32_t first = lane / kLanes, within = lane % kLanes * 8, col = col0 + within;
    const int valid = col < p.cols ? (int)min(8u, p.cols - col) : 0;
    const bool inside = row0 + 32 <= p.rows && col0 + 32 * T <= p.cols;
    for (uint32_t r = first; r < 32; r += kRows * kStep) {
        const uint32_t row = row0 + r;
        float v[kRows][8];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            *reinterpret_cast<f32x4 *>(v[i]) = *reinterpret_cast<const f32x4 *>(sums + (r + kStep * i) * kRowFloats<T> + within);
            *reinterpret_cast<f32x4 *>(v[i] + 4) = *reinterpret_cast<const f32x4 *>(sums + (r + kStep * i) * kRowFloats<T> + within + 4);
        }
        if (p.splits > 1) {
            float *out = p.partial + ((size_t)split * p.rows + row) * p.partial_ld + col;             // partial_ld is a multiple of 4
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                if (row + kStep * i >= p.rows) break;
                if (valid > 0) *reinterpret_cast<f32x4 *>(out + (size_t)(kStep * i) * p.partial_ld) = *reinterpret_cast<f32x4 *>(v[i]);
                if (valid > 4) *reinterpret_cast<f32x4 *>(out + (size_t)(kStep * i) * p.partial_ld + 4) = *reinterpret_cast<f32x4 *>(v[i] + 4);
            }
        } else if (inside) {
            finish_eight<true, OP, DTYPE, kRows, kStep, STREAM>(p.finish, row, p.rows, col, 8, v);
        } else {
            finish_eight<false, OP, DTYPE, kRows, kStep, STREAM>(p.finish, row, p.rows, col, valid, v);
        }
    }
}

// The end of a wave's T x T tiles of 32 x 32 through `mine`, its own 32 * kRowFloats<T> floats of the LDS (that nobody else uses any more); row tile i is
// number i ^ swap from row0 on.
template <int OP, uint32_t DTYPE, int T, bool STREAM = false>
__device__ inline void finish_wave(const Product &p, const f32x16 (&acc)[T][T], float *mine, uint32_t row0, uint32_t col0, int swap, int lane, uint32_t split) {
    for (int i = 0; i < T; ++i) {
        wave_fence();
        auto put = [&](const f32x16 (&from)[T]) {
#pragma unroll
            for (int j = 0; j < T; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<f32x4 *>(mine + (lane & 31) * kRowFloats<T> + j * 32 + 8 * g + 4 * (lane >> 5)) =
                        f32x4{from[j][4 * g], from[j][4 * g + 1], from[j][4 * g + 2], from[j][4 * g + 3]};
        };
        if (i == 0) put(acc[0]);
        else if (T <= 2 || i == 1) put(acc[T > 1 ? 1 : 0]);
        else if (i == 2) put(acc[T / 2]);
        else put(acc[T - 1]);
        wave_fence();
        finish_rows<OP, DTYPE, T, STREAM>(p, mine, row0 + (i ^ swap) * 32, col0, lane, split);
    }
}

// The end of four neighbouring columns; BLOCK: eight lanes side by side have the 32 columns from col0 on.
template <bool BLOCK, uint32_t DTYPE> __device__ inline void finish_quad(const Product &p, uint32_t row, uint32_t col0, uint32_t col, int valid, float (&v)[4]) {
    if (valid) finish_bias<kForward, DTYPE>(p.finish, col, valid, v);
    if constexpr (BLOCK)
        if (p.finish.codes_out) {
            uint32_t largest = 0;
            float z[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                z[e] = e < valid ? v[e] : 0.0f;
                largest = max(largest, magnitude_bits(z[e]));
            }
            largest = largest_of_quad(largest);
            largest = max(largest, (uint32_t)__shfl_xor((int)largest, 4));
            const uint32_t t = block_exponent(largest);
            if (row < p.rows) {                                    // (the workgroup has a column: its block exists)
                const size_t block = (size_t)row * p.finish.blocks + col0 / kBlock;
                if (col == col0) p.finish.exps_out[block] = (uint8_t)t;
                *reinterpret_cast<uint32_t *>(p.finish.codes_out + block * kBlock + (col - col0)) = codes4(z, t);
            }
        }
    if (valid) finish_store<kForward, DTYPE>(p.finish, row, col, valid, v);
}

// Row sums (sums: the product with ones, any of its rows) of row `row`, for one lane of each.
__device__ inline void finish_row_sum(const Product &p, float sum, uint32_t row, uint32_t split) {
    if (row >= p.rows) return;
    if (p.splits > 1) p.partial[(size_t)p.splits * p.rows * p.partial_ld + (size_t)split * p.rows + row] = sum;
    else p.row_sums[row] = p.finish.accumulate ? p.row_sums[row] + sum : sum;
}

}  // namespace eden_layers

#endif  // EDEN_LAYERS_PRODUCT_H
