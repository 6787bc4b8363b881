// Matrix products of the layer operators for any size, distance, alignment and type.
//
// out[r][c] = sum_d A(r, d) B(c, d) on the matrix cores, 32 x 32 x 16 products of bf16 (fp16 where both operands are fp16) summed in fp32.
// A workgroup of four waves has a tile of 128 x 128, a wave 64 x 64 of it.  Operands go through registers into the LDS, where
// those that the matrix cores cannot take are turned into bf16 terms that add up to them exactly:
//   fp32                three terms of 8 bits; fp16 next to a checkpoint: two.  With three on both sides the products below 2^-24 are left out.
//   8-bit checkpoint    q 2^(t - 127) itself: seven bits.
// The LDS holds an operand as memory does: rows of the depth (x, w, dz), or rows of columns at one depth (dy, checkpoints, w in the
// input gradient), which the transposing reads of the LDS turn by the way.  16-byte pieces of a row are swapped so that neither kind of
// read meets its own bank.  The operand of the columns goes first into the products, so that a lane ends up with one row and runs of four
// columns of the result: the end of the product works on vectors, and a checkpoint's block of 32 columns is 16 values in each of two lanes.
#include "eden_layers_product.h"

namespace eden_layers {
namespace {

constexpr int kThreads = 256;

template <int OP, uint32_t DTYPE> struct Plan {
    static constexpr bool kTwoBytes = DTYPE != EDEN_F32;
    static constexpr int kTermsA = DTYPE == EDEN_F32 ? 3 : (OP == kWeightGrad && DTYPE == EDEN_F16) ? 2 : 1;
    static constexpr int kTermsB = OP == kWeightGrad ? 1 : DTYPE == EDEN_F32 ? 3 : 1;
    static constexpr bool kHalf = DTYPE == EDEN_F16 && OP != kWeightGrad;      // fp16 products
    static constexpr bool kStridedA = OP == kWeightGrad, kStridedB = OP != kForward;
    // one term: 64 deep, two stages (64 KiB, two workgroups per CU); more: 32 deep, one stage (up to 48 KiB)
    static constexpr int kDepth = kTermsA * kTermsB == 1 ? 64 : 32;
    static constexpr int kStages = kTermsA * kTermsB == 1 ? 2 : 1;
    static constexpr int kPlane = (int)kTile * kDepth * 2;                     // bytes of one term of an operand's tile
    static constexpr int kStageBytes = (kTermsA + kTermsB) * kPlane;
    static constexpr int kPieces = (int)kTile * kDepth / 8 / kThreads;         // pieces of 8 elements per thread and operand
};

// Eight elements of an operand on their way from memory to the LDS.
template <uint32_t DTYPE> struct Piece { Vec<typename Elem<DTYPE>::type, 8> v; };
struct CodePiece { u32x4 codes; uint32_t exponent; };              // 16 codes

template <uint32_t DTYPE, int TERMS> __device__ inline void store_piece(char *lds, int plane, const Piece<DTYPE> &p) {
    if constexpr (TERMS == 1) {
        static_assert(sizeof(p) == 16, "");
        __builtin_memcpy(__builtin_assume_aligned(lds, 16), &p, 16);
    } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)p.v.v[i];
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = take_term(x[2 * i]), b = take_term(x[2 * i + 1]);
                w[i] = upper_halves(a, b);
            }
            *reinterpret_cast<u32x4 *>(lds + t * plane) = w;
        }
    }
}

template <int OP, uint32_t DTYPE> __global__ __launch_bounds__(kThreads, 2) void k_tiles(const Product p) {
    using P = Plan<OP, DTYPE>;
    using T = typename Elem<DTYPE>::type;
    constexpr int D = P::kDepth, N = P::kPieces;
    __shared__ __attribute__((aligned(16))) char lds[P::kStages * P::kStageBytes];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wave_row = wave >> 1, wave_col = wave & 1;
    const uint32_t row_tiles = tiles_of(p.rows), col_tiles = tiles_of(p.cols);
    uint32_t split, row_tile, col_tile;
    place_of(blockIdx.x, gridDim.x, row_tiles, col_tiles, split, row_tile, col_tile);
    const uint32_t row0 = row_tile * kTile, col0 = col_tile * kTile;
    const uint32_t begin = split * p.split_depth, end = min(p.depth, begin + p.split_depth);
    const bool inside = row0 + kTile <= p.rows && col0 + kTile <= p.cols;      // of the codes: up to the row's last whole block

    Piece<DTYPE> a[N], b[OP == kWeightGrad ? 1 : N];
    CodePiece codes[OP == kWeightGrad ? N / 2 : 1];

    // pieces of a tile at one depth: piece i of this thread is number i * kThreads + tid, along the rows of memory
    auto load_operand = [&](Piece<DTYPE> (&r)[N], const T *base, size_t ld, bool strided, uint32_t first, uint32_t count, uint32_t k, bool full) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t c = (uint32_t)(i * kThreads + tid), per_row = strided ? kTile / 8 : D / 8;
            const uint32_t outer = c / per_row, inner = c % per_row * 8;
            const uint32_t row = strided ? k + outer : first + outer, col = strided ? first + inner : k + inner;
            const uint32_t rows = strided ? end : count, cols = strided ? count : end;
            const T *at = base + (size_t)row * ld + col;
            if (full) r[i].v = load_some<T, 8>(at, 8);
            else r[i].v = load_some<T, 8>(at, row < rows ? (int)min(8u, cols > col ? cols - col : 0u) : 0);
        }
    };
    auto load = [&](uint32_t k) {
        const bool full = inside && k + D <= end;
        load_operand(a, static_cast<const T *>(p.a), p.lda, P::kStridedA, row0, p.rows, k, full);
        if constexpr (OP != kWeightGrad) {
            load_operand(b, static_cast<const T *>(p.b), p.ldb, P::kStridedB, col0, p.cols, k, full);
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const uint32_t c = (uint32_t)(i * kThreads + tid), row = k + c / 8, col = col0 + c % 8 * 16;
                if (row < end && col < p.b_blocks * kBlock) {
                    codes[i].codes = *reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(p.b) + (size_t)row * p.ldb + col);
                    codes[i].exponent = p.b_exps[(size_t)row * p.b_blocks + col / kBlock];
                } else {
                    codes[i].codes = u32x4{0, 0, 0, 0};
                    codes[i].exponent = 1;
                }
            }
        }
    };
    auto store = [&](char *stage) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * kThreads + tid;
            store_piece<DTYPE, P::kTermsA>(stage + (P::kStridedA ? piece_of_depth<kTile>(c / 16, c % 16) : piece_of_row<D>(c / (D / 8), c % (D / 8))), P::kPlane, a[i]);
        }
        char *second = stage + P::kTermsA * P::kPlane;
        if constexpr (OP != kWeightGrad) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = i * kThreads + tid;
                store_piece<DTYPE, P::kTermsB>(second + (P::kStridedB ? piece_of_depth<kTile>(c / 16, c % 16) : piece_of_row<D>(c / (D / 8), c % (D / 8))), P::kPlane, b[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const int c = i * kThreads + tid;
                const float unit = block_unit(codes[i].exponent);
                *reinterpret_cast<u32x4 *>(second + piece_of_depth<kTile>(c / 8, c % 8 * 2)) = code_values(codes[i].codes[0], codes[i].codes[1], unit);
                *reinterpret_cast<u32x4 *>(second + piece_of_depth<kTile>(c / 8, c % 8 * 2 + 1)) = code_values(codes[i].codes[2], codes[i].codes[3], unit);
            }
        }
    };

    f32x16 acc[2][2] = {};
    f32x16 sums = {};                                              // row sums: the product with ones, 32 rows per wave
    const bool with_sums = OP == kWeightGrad && p.row_sums && col_tile == 0;
    const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};

    auto compute = [&](const char *stage) {
        const char *second = stage + P::kTermsA * P::kPlane;
#pragma unroll
        for (int d = 0; d < D; d += 16) {
            u32x4 fa[P::kTermsA][2], fb[P::kTermsB][2];
#pragma unroll
            for (int t = 0; t < P::kTermsA; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) fa[t][i] = fragment<P::kStridedA, D, kTile>(stage + t * P::kPlane, wave_row * 64 + i * 32, d, lane);
#pragma unroll
            for (int t = 0; t < P::kTermsB; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j) fb[t][j] = fragment<P::kStridedB, D, kTile>(second + t * P::kPlane, wave_col * 64 + j * 32, d, lane);
#pragma unroll
            for (int ta = P::kTermsA - 1; ta >= 0; --ta)           // small products first
#pragma unroll
                for (int tb = P::kTermsB - 1; tb >= 0; --tb) {
                    if (P::kTermsB > 1 && ta + tb > 2) continue;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j) acc[i][j] = multiply<P::kHalf>(fb[tb][j], fa[ta][i], acc[i][j]);
                }
            if constexpr (OP == kWeightGrad)
                if (with_sums) {
#pragma unroll
                    for (int ta = P::kTermsA - 1; ta >= 0; --ta) sums = multiply<false>(ones, wave_col ? fa[ta][1] : fa[ta][0], sums);
                }
        }
    };

    if (begin < end) {
        load(begin);
        store(lds);
        __syncthreads();
        int stage = 0;
        for (uint32_t k = begin; k < end; k += D) {
            const bool more = k + D < end;
            if (more) load(k + D);
            compute(lds + stage * P::kStageBytes);
            if constexpr (P::kStages == 1) __syncthreads();
            else stage ^= 1;
            if (more) store(lds + stage * P::kStageBytes);
            __syncthreads();
        }
    }

    if constexpr (OP == kWeightGrad)
        if (with_sums && lane < 32) finish_row_sum(p, sums[0], row0 + wave_row * 64 + wave_col * 32 + lane, split);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            finish_tile<OP, DTYPE>(p, acc[i][j], row0 + wave_row * 64 + i * 32 + (lane & 31), col0 + wave_col * 64 + j * 32, lane, split);
}

// Sums of the splits, in their order, and the end of the product.  A thread has four columns, eight threads a block of a checkpoint.
template <int OP, uint32_t DTYPE> __global__ __launch_bounds__(256) void k_join(const Product p) {
    const uint32_t quads = (uint32_t)blocks_of(p.cols) * (kBlock / 4);
    const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (at < (uint64_t)p.rows * quads) {
        const uint32_t row = (uint32_t)(at / quads), col = (uint32_t)(at % quads) * 4;
        const int valid = col < p.cols ? (int)min(4u, p.cols - col) : 0;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (valid)
            for (uint32_t s = 0; s < p.splits; ++s) {
                const f32x4 add = *reinterpret_cast<const f32x4 *>(p.partial + ((size_t)s * p.rows + row) * p.partial_ld + col);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += add[e];
            }
        if (valid) finish_bias<OP, DTYPE>(p.finish, col, valid, v);
        if constexpr (OP == kForward)
            if (p.finish.codes_out) {                              // whole blocks are in range together: quads is a multiple of 8
                uint32_t largest = 0;
                float z[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z[e] = e < valid ? v[e] : 0.0f;
                    largest = max(largest, magnitude_bits(z[e]));
                }
#pragma unroll
                for (int step = 1; step < 8; step *= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, step));
                const uint32_t t = block_exponent(largest);
                const size_t block = (size_t)row * p.finish.blocks + col / kBlock;
                if (col % kBlock == 0) p.finish.exps_out[block] = (uint8_t)t;
                *reinterpret_cast<uint32_t *>(p.finish.codes_out + block * kBlock + col % kBlock) = codes4(z, t);
            }
        if (valid) finish_store<OP, DTYPE>(p.finish, row, col, valid, v);
        if constexpr (OP == kWeightGrad)
            if (p.row_sums && col == 0) {
                float sum = 0.0f;
                for (uint32_t s = 0; s < p.splits; ++s) sum += p.partial[(size_t)p.splits * p.rows * p.partial_ld + (size_t)s * p.rows + row];
                p.row_sums[row] = p.finish.accumulate ? p.row_sums[row] + sum : sum;
            }
    }
}

template <class F> hipError_t for_type(Op op, uint32_t dtype, F f) {
    auto typed = [&](auto o) {
        if (dtype == EDEN_F32) f(o, std::integral_constant<uint32_t, EDEN_F32>());
        else if (dtype == EDEN_F16) f(o, std::integral_constant<uint32_t, EDEN_F16>());
        else f(o, std::integral_constant<uint32_t, EDEN_BF16>());
    };
    if (op == kForward) typed(std::integral_constant<int, kForward>());
    else if (op == kInputGrad) typed(std::integral_constant<int, kInputGrad>());
    else typed(std::integral_constant<int, kWeightGrad>());
    return hipGetLastError();
}

}  // namespace

hipError_t launch_tiles(Op op, uint32_t dtype, const Product &p, hipStream_t st) {
    const uint32_t grid = (uint32_t)((uint64_t)tiles_of(p.rows) * tiles_of(p.cols) * p.splits);
    return for_type(op, dtype, [&](auto o, auto t) { k_tiles<decltype(o)::value, decltype(t)::value><<<grid, kThreads, 0, st>>>(p); });
}

hipError_t launch_join(Op op, uint32_t dtype, const Product &p, hipStream_t st) {
    const uint64_t quads = (uint64_t)p.rows * blocks_of(p.cols) * (kBlock / 4);
    return for_type(op, dtype, [&](auto o, auto t) { k_join<decltype(o)::value, decltype(t)::value><<<(uint32_t)((quads + 255) / 256), 256, 0, st>>>(p); });
}

}  // namespace eden_layers
