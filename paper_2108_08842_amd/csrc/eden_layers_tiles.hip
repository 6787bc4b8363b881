// Matrix products of the layer operators for any size, distance, alignment and type.
//
// out[r][c] = sum_d A(r, d) B(c, d) on the matrix cores, 32 x 32 x 16 products of bf16 (fp16 where both operands are fp16) summed in fp32.
// A workgroup of four waves has a tile of 128 x 128, a wave 64 x 64 of it; where such tiles would leave most of the device idle and each step
// of a few workgroups would be waited for, 64 x 64 and 32 x 32.  Operands go through registers into the LDS, where
// those that the matrix cores cannot take are turned into bf16 terms that add up to them exactly:
//   fp32                three terms of 8 bits; fp16 next to a checkpoint: two.  With three on both sides the smallest products are left out, below 2^-22 together.
//   8-bit checkpoint    q 2^(t - 127) itself: seven bits.
// The LDS holds an operand as memory does: rows of the depth (x, w, dz), or rows of columns at one depth (dy, checkpoints, w in the
// input gradient), which the transposing reads of the LDS turn by the way.  16-byte pieces of a row are swapped so that neither kind of
// read meets its own bank.  The operand of the columns goes first into the products, so that a lane ends up with one row and runs of four
// columns of the result: the end of the product works on vectors, and a checkpoint's block of 32 columns is 16 values in each of two lanes.
//
// Takes what the kernels with loads straight into the LDS do not: rows that begin anywhere, small products, fp32 and fp16 next to a checkpoint.  Bound by the way
// through the registers: a step's loads are as far ahead as its registers reach, and with more than one term there is one stage, so that a step has two barriers and takes its operands
// apart between them, when no product runs: weight gradient of 4096 x 4096, 4096 deep, fp16 345 us (400 TFLOP/s, twice that in terms; matrix cores busy 34% of the
// cycles), fp32 460 us (300 TFLOP/s; 40%).  1001 x 1024, 555 deep, fp32: 256 tiles in two parts, 14.5 us and 4.4 for the join, most of it waiting.
#include "eden_layers_product.h"

namespace eden_layers {
namespace {

constexpr int kThreads = 256;

// W: a wave has W x W products of 32 x 32, a workgroup 64 W x 64 W
template <int OP, uint32_t DTYPE, int W> struct Plan {
    static constexpr int kTermsA = DTYPE == EDEN_F32 ? 3 : (OP == kWeightGrad && DTYPE == EDEN_F16) ? 2 : 1;
    static constexpr int kTermsB = OP == kWeightGrad ? 1 : DTYPE == EDEN_F32 ? 3 : 1;
    static constexpr bool kNearest = kTermsB > 1;                              // not all products of terms are taken
    static constexpr bool kHalf = DTYPE == EDEN_F16 && OP != kWeightGrad;      // fp16 products
    static constexpr bool kStridedA = OP == kWeightGrad, kStridedB = OP != kForward;
    static constexpr int kSide = 64 * W;
    // tiles of 128, one term: 64 deep, two stages (64 KiB, two workgroups per CU); more terms: 32 deep, one stage (up to 48 KiB).  Tiles of 64: 64 deep.
    static constexpr int kDepth = W == 1 || kTermsA * kTermsB == 1 ? 64 : 32;
    static constexpr int kStages = kTermsA * kTermsB == 1 ? 2 : 1;
    static constexpr int kPlane = kSide * kDepth * 2;                          // bytes of one term of an operand's tile
    static constexpr int kStageBytes = (kTermsA + kTermsB) * kPlane;
    static constexpr int kEnd = 4 * 32 * kRowFloats<W> * 4;                    // what the end of the sums takes of the LDS
    static constexpr int kShared = kStages * kStageBytes > kEnd ? kStages * kStageBytes : kEnd;
    static constexpr int kPieces = kSide * kDepth / 8 / kThreads;              // pieces of 8 elements per thread and operand
};

// Eight elements of an operand on their way from memory to the LDS.
template <uint32_t DTYPE> struct Piece { Vec<typename Elem<DTYPE>::type, 8> v; };
struct CodePiece { u32x4 codes; uint32_t exponent; };              // 16 codes

// Eight neighbouring elements from `at` on, at the ends of rows and operands: read as one vector that may hold elements of the next row, or the operand's last
// eight where it would reach beyond `end` or none is `wanted`.  Nothing depends on what was read until the piece goes into the LDS, so that a thread's loads are all on their way at
// once (with the selection right behind each load 512 x 1001 x 1003 bf16 took 17 us in place of 14).
template <class T> __device__ inline Vec<T, 8> load_near(const T *at, const T *base, const T *end, bool wanted) {
    if (end - base < 8) return Vec<T, 8>{};
    return load_some<T, 8>(wanted && end - at >= 8 ? at : end - 8, 8);
}
// ... and then: the first `valid` of the elements from `at` on, zeros behind them.
template <class T> __device__ inline void select_near(Vec<T, 8> &v, const T *at, const T *end, int valid) {
    if (valid > 0 && end - at < 8) {
        v = load_some<T, 8>(at, valid < 8 ? valid : 7);            // (there are fewer than eight)
    } else if constexpr (sizeof(T) == 2) {
        u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = valid >= 2 * i + 2 ? w[i] : valid == 2 * i + 1 ? w[i] & 0xFFFFu : 0u;
        v = __builtin_bit_cast(Vec<T, 8>, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.v[i] = i < valid ? v.v[i] : (T)0;
    }
}

template <uint32_t DTYPE, int TERMS, bool NEAREST> __device__ inline void store_piece(char *lds, int plane, const Piece<DTYPE> &p) {
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
                if constexpr (NEAREST) {
                    w[i] = take_nearest(x[2 * i], x[2 * i + 1], t == 0);
                } else {
                    const float a = take_term(x[2 * i]), b = take_term(x[2 * i + 1]);
                    w[i] = upper_halves(a, b);
                }
            }
            *reinterpret_cast<u32x4 *>(lds + t * plane) = w;
        }
    }
}

template <int OP, uint32_t DTYPE, int W> __global__ __launch_bounds__(kThreads, W == 1 ? 3 : 2) void k_tiles(const Product p) {
    using P = Plan<OP, DTYPE, W>;
    using T = typename Elem<DTYPE>::type;
    constexpr int D = P::kDepth, N = P::kPieces;
    constexpr uint32_t kSide = P::kSide, kAcross = kSide / 8;         // pieces of a row of columns
    __shared__ __attribute__((aligned(16))) char lds[P::kShared];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wave_row = wave >> 1, wave_col = wave & 1;
    const uint32_t row_tiles = tiles_of(p.rows, kSide), col_tiles = tiles_of(p.cols, kSide);
    uint32_t split, row_tile, col_tile;
    place_of(blockIdx.x, gridDim.x, row_tiles, col_tiles, split, row_tile, col_tile);
    const uint32_t row0 = row_tile * kSide, col0 = col_tile * kSide;
    const uint32_t begin = split * p.split_depth, end = min(p.depth, begin + p.split_depth);
    const bool inside = row0 + kSide <= p.rows && col0 + kSide <= p.cols;      // of the codes: up to the row's last whole block

    struct Set {
        Piece<DTYPE> a[N], b[OP == kWeightGrad ? 1 : N];
        CodePiece codes[OP == kWeightGrad ? N / 2 : 1];
    };
    // behind the last element of an operand
    const T *end_a = static_cast<const T *>(p.a) + (size_t)((P::kStridedA ? p.depth : p.rows) - 1) * p.lda + (P::kStridedA ? p.rows : p.depth);
    const T *end_b = OP == kWeightGrad ? nullptr : static_cast<const T *>(p.b) + (size_t)((P::kStridedB ? p.depth : p.cols) - 1) * p.ldb + (P::kStridedB ? p.cols : p.depth);

    // pieces of a tile at one depth: piece i of this thread is number i * kThreads + tid, along the rows of memory
    struct Where { uint32_t row, col; };
    auto where = [&](int i, bool strided, uint32_t first, uint32_t k) {
        const uint32_t c = (uint32_t)(i * kThreads + tid), per_row = strided ? kAcross : D / 8, outer = c / per_row, inner = c % per_row * 8;
        return Where{strided ? k + outer : first + outer, strided ? first + inner : k + inner};
    };
    auto load_operand = [&](Piece<DTYPE> (&r)[N], const T *base, const T *base_end, size_t ld, bool strided, uint32_t first, uint32_t count, uint32_t k, bool full) {
        const uint32_t rows = strided ? end : count, cols = strided ? count : end;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Where w = where(i, strided, first, k);
            const T *at = base + (size_t)w.row * ld + w.col;
            if (full) r[i].v = load_some<T, 8>(at, 8);
            else r[i].v = load_near(at, base, base_end, w.row < rows && w.col < cols);
        }
    };
    auto select_operand = [&](Piece<DTYPE> (&r)[N], const T *base, const T *base_end, size_t ld, bool strided, uint32_t first, uint32_t count, uint32_t k) {
        const uint32_t rows = strided ? end : count, cols = strided ? count : end;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Where w = where(i, strided, first, k);
            select_near(r[i].v, base + (size_t)w.row * ld + w.col, base_end, w.row < rows && w.col < cols ? (int)min(8u, cols - w.col) : 0);
        }
    };
    auto load = [&](Set &to, uint32_t k) {
        const bool full = inside && k + D <= end;
        load_operand(to.a, static_cast<const T *>(p.a), end_a, p.lda, P::kStridedA, row0, p.rows, k, full);
        if constexpr (OP != kWeightGrad) {
            load_operand(to.b, static_cast<const T *>(p.b), end_b, p.ldb, P::kStridedB, col0, p.cols, k, full);
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const uint32_t c = (uint32_t)(i * kThreads + tid), row = k + c / (kAcross / 2), col = col0 + c % (kAcross / 2) * 16;
                if (row < end && col < p.b_blocks * kBlock) {
                    to.codes[i].codes = *reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(p.b) + (size_t)row * p.ldb + col);
                    to.codes[i].exponent = p.b_exps[(size_t)row * p.b_blocks + col / kBlock];
                } else {
                    to.codes[i].codes = u32x4{0, 0, 0, 0};
                    to.codes[i].exponent = 1;
                }
            }
        }
    };
    auto store = [&](char *stage, Set &from, uint32_t k) {
        if (!(inside && k + D <= end)) {
            select_operand(from.a, static_cast<const T *>(p.a), end_a, p.lda, P::kStridedA, row0, p.rows, k);
            if constexpr (OP != kWeightGrad) select_operand(from.b, static_cast<const T *>(p.b), end_b, p.ldb, P::kStridedB, col0, p.cols, k);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = i * kThreads + tid;
            store_piece<DTYPE, P::kTermsA, P::kNearest>(stage + (P::kStridedA ? piece_of_depth<P::kSide>(c / kAcross, c % kAcross) : piece_of_row<D>(c / (D / 8), c % (D / 8))), P::kPlane, from.a[i]);
        }
        char *second = stage + P::kTermsA * P::kPlane;
        if constexpr (OP != kWeightGrad) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = i * kThreads + tid;
                store_piece<DTYPE, P::kTermsB, P::kNearest>(second + (P::kStridedB ? piece_of_depth<P::kSide>(c / kAcross, c % kAcross) : piece_of_row<D>(c / (D / 8), c % (D / 8))), P::kPlane, from.b[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const int c = i * kThreads + tid;
                const float unit = block_unit(from.codes[i].exponent);
                *reinterpret_cast<u32x4 *>(second + piece_of_depth<P::kSide>(c / (kAcross / 2), c % (kAcross / 2) * 2)) = code_values(from.codes[i].codes[0], from.codes[i].codes[1], unit);
                *reinterpret_cast<u32x4 *>(second + piece_of_depth<P::kSide>(c / (kAcross / 2), c % (kAcross / 2) * 2 + 1)) = code_values(from.codes[i].codes[2], from.codes[i].codes[3], unit);
            }
        }
    };

    f32x16 acc[W][W] = {};
    f32x16 sums = {};                                              // row sums: the product with ones, 32 rows per wave (W = 1: of the first wave of a row)
    const bool with_sums = OP == kWeightGrad && p.row_sums && col_tile == 0 && wave_col < W;
    const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};

    auto compute = [&](const char *stage) {
        const char *second = stage + P::kTermsA * P::kPlane;
#pragma unroll
        for (int d = 0; d < D; d += 16) {
            u32x4 fa[P::kTermsA][W], fb[P::kTermsB][W];
#pragma unroll
            for (int t = 0; t < P::kTermsA; ++t)
#pragma unroll
                for (int i = 0; i < W; ++i) fa[t][i] = fragment<P::kStridedA, D, P::kSide>(stage + t * P::kPlane, wave_row * (32 * W) + i * 32, d, lane);
#pragma unroll
            for (int t = 0; t < P::kTermsB; ++t)
#pragma unroll
                for (int j = 0; j < W; ++j) fb[t][j] = fragment<P::kStridedB, D, P::kSide>(second + t * P::kPlane, wave_col * (32 * W) + j * 32, d, lane);
#pragma unroll
            for (int ta = P::kTermsA - 1; ta >= 0; --ta)           // small products first
#pragma unroll
                for (int tb = P::kTermsB - 1; tb >= 0; --tb) {
                    if (P::kTermsB > 1 && ta + tb > 2) continue;
#pragma unroll
                    for (int i = 0; i < W; ++i)
#pragma unroll
                        for (int j = 0; j < W; ++j) acc[i][j] = multiply<P::kHalf>(fb[tb][j], fa[ta][i], acc[i][j]);
                }
            if constexpr (OP == kWeightGrad)
                if (with_sums) {
#pragma unroll
                    for (int ta = P::kTermsA - 1; ta >= 0; --ta) sums = multiply<false>(ones, wave_col ? fa[ta][W - 1] : fa[ta][0], sums);
                }
        }
    };

    Set next;
    if (begin < end) {
        load(next, begin);
        store(lds, next, begin);
        __syncthreads();
        int stage = 0;
        for (uint32_t k = begin; k < end; k += D) {
            const bool more = k + D < end;
            if (more) load(next, k + D);
            compute(lds + stage * P::kStageBytes);
            if constexpr (P::kStages == 1) __syncthreads();
            else stage ^= 1;
            if (more) store(lds + stage * P::kStageBytes, next, k + D);
            __syncthreads();
        }
    }

    if constexpr (OP == kWeightGrad)
        if (with_sums && lane < 32) finish_row_sum(p, sums[0], row0 + wave_row * (32 * W) + wave_col * 32 + lane, split);
    // (behind the last barrier nobody reads a stage any more)
    finish_wave<OP, DTYPE, W>(p, acc, reinterpret_cast<float *>(lds) + wave * 32 * kRowFloats<W>, row0 + wave_row * (32 * W), col0 + wave_col * (32 * W), 0, lane, split);
}

// Sums of the splits, in their order, and the end of the product.  A thread has four columns, eight threads a block of a checkpoint.
template <int OP, uint32_t DTYPE> __global__ __launch_bounds__(256) void k_join(const Product p) {
    const uint32_t quads = (uint32_t)blocks_of(p.cols) * (kBlock / 4);
    const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (at < (uint64_t)p.rows * quads) {
        const uint32_t row = (uint32_t)(at / quads), col = (uint32_t)(at % quads) * 4;
        const int valid = col < p.cols ? (int)min(4u, p.cols - col) : 0;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (valid) {
            const float *from = p.partial + (size_t)row * p.partial_ld + col;
            const size_t step = (size_t)p.rows * p.partial_ld;
            uint32_t s = 0;
            for (; s + 8 <= p.splits; s += 8) {                    // eight reads on their way at a time
                f32x4 add[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) add[i] = *reinterpret_cast<const f32x4 *>(from + (s + i) * step);
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += add[i][e];
            }
            for (; s < p.splits; ++s) {
                const f32x4 add = *reinterpret_cast<const f32x4 *>(from + s * step);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += add[e];
            }
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
                largest = largest_of_quad(largest);
                largest = max(largest, (uint32_t)__shfl_xor((int)largest, 4));
                const uint32_t t = block_exponent(largest);
                const size_t block = (size_t)row * p.finish.blocks + col / kBlock;
                if (col % kBlock == 0) p.finish.exps_out[block] = (uint8_t)t;
                *reinterpret_cast<uint32_t *>(p.finish.codes_out + block * kBlock + col % kBlock) = codes4(z, t);
            }
        if (valid) finish_store<OP, DTYPE>(p.finish, row, col, valid, v);
        if constexpr (OP == kWeightGrad)
            if (p.row_sums && col == 0) {
                const float *from = p.partial + (size_t)p.splits * p.rows * p.partial_ld + row;
                float sum = 0.0f;
                uint32_t s = 0;
                for (; s + 8 <= p.splits; s += 8) {
                    float add[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) add[i] = from[(size_t)(s + i) * p.rows];
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += add[i];
                }
                for (; s < p.splits; ++s) sum += from[(size_t)s * p.rows];
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

hipError_t launch_tiles(Op op, uint32_t dtype, const Product &p, uint32_t side, hipStream_t st) {
    const uint32_t grid = tiles_of(p.rows, side) * tiles_of(p.cols, side) * p.splits;
    return for_type(op, dtype, [&](auto o, auto t) {
        if (side == 64) k_tiles<decltype(o)::value, decltype(t)::value, 1><<<grid, kThreads, 0, st>>>(p);
        else k_tiles<decltype(o)::value, decltype(t)::value, 2><<<grid, kThreads, 0, st>>>(p);
    });
}

hipError_t launch_join(Op op, uint32_t dtype, const Product &p, hipStream_t st) {
    const uint64_t quads = (uint64_t)p.rows * blocks_of(p.cols) * (kBlock / 4);
    return for_type(op, dtype, [&](auto o, auto t) { k_join<decltype(o)::value, decltype(t)::value><<<(uint32_t)((quads + 255) / 256), 256, 0, st>>>(p); });
}

}  // namespace eden_layers
