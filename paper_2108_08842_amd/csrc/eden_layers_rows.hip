// eden_linear for up to 16 rows (single tokens, a few tokens at a time): the weights are read once and everything else is small.  Bound by memory: w's bytes.
//
// k_dots, up to 4 rows (fp32: 8): x lies in the LDS, a wave has one, two or four rows of w and reads a kilobyte of one at a time; every lane multiplies
// its 16 bytes with those of x two elements an instruction, the lanes' sums are added at the end.
// k_rows, up to 16 rows: a workgroup has 16 or 32 columns of the result and all rows; its eight waves go through the depth in turn, 256 bytes of
// each of w's rows at a time, from memory to the matrix cores' registers without the LDS (lane l holds row l % 16 of w and 16 bytes of the
// depth, so a load takes 64 bytes of 16 rows; the next chunk is on its way while one is multiplied).  16 x 16 products; fp32 operands
// are multiplied in fp32.  The waves' sums meet in the LDS, in the order of the waves.
//
// One row of bf16 next to 16384 x 4096: 26 us = 5.2 TB/s, what a copy reaches.  7 x 1024 next to 1001 x 1024 in fp32: 6.3 us, a launch, the way of x into the LDS and one
// of w's rows a wave, one after the other.  16 rows next to 4096 x 4096: 11.1 us = 3.0 TB/s (x comes from the L2 once for every 16 columns: as many bytes as w).
// 8 rows of fp32 next to 16384 x 4096: 71 us = 3.8 TB/s (x from the LDS for every piece of w; a library's product of 5 to 16 rows takes 52).
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

// COLS: sixteens of columns
template <uint32_t DTYPE, int COLS> __global__ __launch_bounds__(kWaves * 64) void k_rows(const Product p) {
    using T = typename Elem<DTYPE>::type;
    constexpr int kPiece = 16 / Elem<DTYPE>::kBytes, kStep = 4 * kPiece, kChunk = kSteps * kStep;
    __shared__ f32x4 sums[kWaves][COLS][64];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col0 = (p.before + blockIdx.x) * (16 * COLS);
    const T *w[COLS];
    bool has_w[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
        const uint32_t col = col0 + c * 16 + (lane & 15);
        has_w[c] = col < p.cols;
        w[c] = static_cast<const T *>(p.b) + (size_t)(has_w[c] ? col : 0) * p.ldb + (lane >> 4) * kPiece;
    }
    const bool has_x = (lane & 15u) < p.rows;
    const T *x = static_cast<const T *>(p.a) + (has_x ? (lane & 15) : 0) * p.lda + (lane >> 4) * kPiece;

    f32x4 acc[COLS] = {};
    struct Chunk { Vec<T, kPiece> w[kSteps][COLS], x[kSteps]; };
    auto load = [&](Chunk &to, uint32_t k) {                       // what is outside the operands is 0
        const bool full = k + kChunk <= p.depth;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const uint32_t at = k + s * kStep, piece = at + (lane >> 4) * kPiece;
            const int valid = full ? kPiece : piece < p.depth ? (int)min((uint32_t)kPiece, p.depth - piece) : 0;
#pragma unroll
            for (int c = 0; c < COLS; ++c) to.w[s][c] = load_some<T, kPiece>(w[c] + at, has_w[c] ? valid : 0);
            to.x[s] = load_some<T, kPiece>(x + at, has_x ? valid : 0);
        }
    };
    auto multiply = [&](const Chunk &from) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int c = 0; c < COLS; ++c)
                acc[c] = multiply16<DTYPE>(__builtin_bit_cast(u32x4, from.w[s][c]), __builtin_bit_cast(u32x4, from.x[s]), acc[c]);
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
    for (int c = 0; c < COLS; ++c) sums[wave][c][lane] = acc[c];
    __syncthreads();

    // thread -> row and four columns; 4 COLS threads side by side have a row (COLS = 2: a block of a checkpoint)
    constexpr int kQuads = 4 * COLS;
    if (tid < 16 * kQuads) {
        const int row = tid / kQuads, quad = tid % kQuads;
        f32x4 sum = sums[0][quad >> 2][(quad & 3) * 16 + row];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) sum += sums[i][quad >> 2][(quad & 3) * 16 + row];
        const uint32_t col = col0 + quad * 4;
        const int valid = (uint32_t)row < p.rows && col < p.cols ? (int)min(4u, p.cols - col) : 0;
        float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        finish_quad<COLS == 2, DTYPE>(p, row, col0, col, valid, v);
    }
}

// c + a . b for the eight (fp32: four) elements of two pieces, the fp32 sums in the order of the elements
template <uint32_t DTYPE> __device__ inline float dot_piece(u32x4 a, u32x4 b, float c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = a[i], y = b[i];
        if constexpr (DTYPE == EDEN_F32) c = __builtin_fmaf(__uint_as_float(x), __uint_as_float(y), c);
        else if constexpr (DTYPE == EDEN_F16) c = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, x), __builtin_bit_cast(f16x2, y), c, false);
        else c = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, y), c, false);
    }
    return c;
}

// The sums over the wave's lanes of N values a lane (N a power of two up to 64): value i ends up in the lanes whose upper log2 N bits are i.  Half of the
// values change sides at a time, so that N values take N + 5 exchanges and not 6 N.
template <int N, int DISTANCE = 32> __device__ inline float sum_lanes(const float (&v)[N], int lane) {
    if constexpr (N > 1) {
        const bool upper = lane & DISTANCE;
        float half[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) half[i] = (upper ? v[i + N / 2] : v[i]) + __shfl_xor(upper ? v[i] : v[i + N / 2], DISTANCE);
        return sum_lanes<N / 2, DISTANCE / 2>(half, lane);
    } else {
        float sum = v[0];
#pragma unroll
        for (int d = DISTANCE; d >= 1; d /= 2) sum += __shfl_xor(sum, d);
        return sum;
    }
}

constexpr uint32_t kMostShared = 61440;            // bytes of x in the LDS at a time: two workgroups a CU at least
template <int ROWS> __host__ __device__ constexpr uint32_t part_of() { return kMostShared / 16 / ROWS / 64 * 64; }       // pieces of a row

// EACH: rows of w a wave has; ROWS: rows of x (a power of two, those beyond p.rows are zeros)
template <uint32_t DTYPE, int EACH, int ROWS> __global__ __launch_bounds__(kWaves * 64) void k_dots(const Product p) {
    using T = typename Elem<DTYPE>::type;
    constexpr int kPiece = 16 / Elem<DTYPE>::kBytes, kRun = 8 / EACH, kCols = kWaves * EACH;      // pieces of a row on their way at once
    extern __shared__ u32x4 shared[];                              // x: row r, piece i at r * pieces + i; then the sums
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t pieces = (p.depth + kPiece * 64 - 1) / (kPiece * 64) * 64;                     // a lane has one of every 64
    const uint32_t part = min(pieces, part_of<ROWS>());                                           // of x in the LDS at a time
    const uint32_t col0 = (p.before + blockIdx.x) * kCols, first = col0 + wave * EACH;
    const T *w[EACH];
    bool has[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        has[e] = first + e < p.cols;
        w[e] = static_cast<const T *>(p.b) + (size_t)(has[e] ? first + e : 0) * p.ldb + lane * kPiece;
    }
    struct Run { u32x4 q[kRun][EACH]; };
    auto load = [&](Run &to, uint32_t piece) {                     // what is outside w is 0
        const bool full = (piece + kRun * 64) * kPiece <= p.depth;
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            const uint32_t at = (piece + i * 64) * kPiece, mine = at + lane * kPiece;
            const int valid = full ? kPiece : mine < p.depth ? (int)min((uint32_t)kPiece, p.depth - mine) : 0;
#pragma unroll
            for (int e = 0; e < EACH; ++e) to.q[i][e] = __builtin_bit_cast(u32x4, load_some<T, kPiece>(w[e] + at, has[e] ? valid : 0));
        }
    };
    float sums[EACH * ROWS] = {};
    for (uint32_t from = 0; from < pieces; from += part) {
        const uint32_t end = min(pieces, from + part), held = end - from;
        Run even, odd;
        load(even, from);                                          // w is on its way while x is fetched
        if (from) __syncthreads();
        for (uint32_t i = tid; i < ROWS * held; i += kWaves * 64) {
            const uint32_t row = i / held, piece = i - row * held, k = (from + piece) * kPiece;
            const int valid = row < p.rows && k < p.depth ? (int)min((uint32_t)kPiece, p.depth - k) : 0;
            shared[row * part + piece] = __builtin_bit_cast(u32x4, load_some<T, kPiece>(static_cast<const T *>(p.a) + (valid ? row * p.lda + k : 0), valid));
        }
        __syncthreads();

        auto multiply = [&](const Run &run, uint32_t piece) {
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                if (piece + i * 64 >= end) break;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const u32x4 x = shared[r * part + piece - from + i * 64 + lane];
#pragma unroll
                    for (int e = 0; e < EACH; ++e) sums[e * ROWS + r] = dot_piece<DTYPE>(run.q[i][e], x, sums[e * ROWS + r]);
                }
            }
        };
        for (uint32_t piece = from; piece < end;) {
            if (piece + kRun * 64 < end) load(odd, piece + kRun * 64);
            multiply(even, piece);
            piece += kRun * 64;
            if (piece >= end) break;
            if (piece + kRun * 64 < end) load(even, piece + kRun * 64);
            multiply(odd, piece);
            piece += kRun * 64;
        }
    }
    float *out = reinterpret_cast<float *>(shared + ROWS * part);                                 // [ROWS][kCols]
    const float sum = sum_lanes<EACH * ROWS>(sums, lane);
    constexpr int kSame = 64 / (EACH * ROWS);                                                     // lanes with the same sum
    if (lane % kSame == 0) out[lane / kSame % ROWS * kCols + wave * EACH + lane / kSame / ROWS] = sum;
    __syncthreads();

    constexpr int kQuads = kCols / 4;                              // EACH = 4: a block of a checkpoint
    if (tid < ROWS * kQuads) {
        const int row = tid / kQuads, quad = tid % kQuads;
        const uint32_t col = col0 + quad * 4;
        const int valid = (uint32_t)row < p.rows && col < p.cols ? (int)min(4u, p.cols - col) : 0;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = out[row * kCols + quad * 4 + i];
        finish_quad<kCols == kBlock, DTYPE>(p, row, col0, col, valid, v);
    }
}

// f(the product, workgroups of a launch) until all `groups` are launched
template <class F> hipError_t launches(Product p, uint32_t groups, F f) {
    constexpr uint32_t kMost = (uint32_t)most_groups(kWaves * 64);
    hipError_t e = hipSuccess;
    for (p.before = 0; p.before < groups && e == hipSuccess; p.before += kMost) {
        f(p, groups - p.before < kMost ? groups - p.before : kMost);
        e = hipGetLastError();
    }
    return e;
}
template <uint32_t DTYPE, int COLS> hipError_t launch(const Product &p, hipStream_t st) {
    return launches(p, (p.cols + 16 * COLS - 1) / (16 * COLS), [&](const Product &q, uint32_t groups) { k_rows<DTYPE, COLS><<<groups, kWaves * 64, 0, st>>>(q); });
}
template <uint32_t DTYPE, int EACH> hipError_t launch_dots(const Product &p, hipStream_t st) {
    constexpr uint32_t kRun = 1024 / Elem<DTYPE>::kBytes;          // elements of a wave's load
    const uint32_t all = (p.cols + kWaves * EACH - 1) / (kWaves * EACH), pieces = (p.depth + kRun - 1) / kRun * 64;
    auto with_rows = [&](auto rows) {
        constexpr int ROWS = decltype(rows)::value;
        const uint32_t part = pieces < part_of<ROWS>() ? pieces : part_of<ROWS>();
        return launches(p, all, [&](const Product &q, uint32_t groups) {
            k_dots<DTYPE, EACH, ROWS><<<groups, kWaves * 64, ROWS * (part * 16 + kWaves * EACH * sizeof(float)), st>>>(q);
        });
    };
    constexpr bool kFull = DTYPE == EDEN_F32;
    if constexpr (EACH != 2) {                                     // (two rows of w are for more rows of x)
        if (p.rows == 1) return with_rows(std::integral_constant<int, 1>());
    }
    if constexpr (EACH != 2 || !kFull) {
        if (p.rows <= 2) return with_rows(std::integral_constant<int, 2>());
    }
    if constexpr (kFull) {
        if (p.rows > 4) return with_rows(std::integral_constant<int, 8>());
    }
    return with_rows(std::integral_constant<int, 4>());
}
template <uint32_t DTYPE> hipError_t launch_type(const Product &p, hipStream_t st) {
    // k_dots in us, w of 16384 x 4096: 4 rows of bf16 28.5 (k_rows 34), 5 rows 40 (35); fp32, 8 rows 67 (72) and at 1024 x 1024 5.9 (6.3).
    // Rows of w a wave: a checkpoint's block takes four.  Rows of up to 2 KiB are two loads, so that four of them keep a wave's eight loads on their way
    // (bf16, 1024 x 1024: 3.8 us against 4.7 with one).  Else two read x half as often where they leave no CU idle (8192 x 4096 bf16, 4 rows:
    // 16.8 against 18.7 with one, but 4096 x 4096 11.8 against 10.6), one is best while x is small (fp32, 16384 x 4096, 2 rows: 47 against 54 with two).
    const bool keeps = p.finish.codes_out != nullptr;
    constexpr bool kFull = DTYPE == EDEN_F32;
    if (p.rows <= (kFull ? 8 : 4)) {
        if (keeps || (!kFull && p.depth <= 1024)) return launch_dots<DTYPE, 4>(p, st);
        if (p.cols >= 512 * 16 && p.rows > (kFull ? 2 : 1)) return launch_dots<DTYPE, 2>(p, st);
        return launch_dots<DTYPE, 1>(p, st);
    }
    return keeps ? launch<DTYPE, 2>(p, st) : launch<DTYPE, 1>(p, st);
}

}  // namespace

hipError_t launch_rows(uint32_t dtype, const Product &p, hipStream_t st) {
    if (dtype == EDEN_F32) return launch_type<EDEN_F32>(p, st);
    if (dtype == EDEN_F16) return launch_type<EDEN_F16>(p, st);
    return launch_type<EDEN_BF16>(p, st);
}

}  // namespace eden_layers
