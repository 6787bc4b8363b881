// 4 bits from and to values.
//
// Bound by memory, the stochastic rounding by the vector unit (the hash's 64-bit products).  Rows: a thread has eight neighbouring columns, four threads a block; a
// workgroup eight rows of a chunk, so that the exponents, which lie together for all rows of a chunk, leave in words.
// Transpose: a workgroup has 256 rows of 128 columns, a wave 32 rows of them and a lane two columns, so a block lies in one lane's registers; codes and exponents
// go through the LDS and leave in whole lines.
#include "eden_layers_spread.h"
#include "eden_mx4_kernels.h"

namespace eden_layers {
namespace {

constexpr int kThreads = 256, kRowsEach = kThreads / (kChunk / 8);

template <uint32_t DTYPE, bool STOCHASTIC>
__global__ __launch_bounds__(kThreads) void k_mx4_rows(const typename Elem<DTYPE>::type *x, size_t ldx, uint32_t rows, uint32_t cols, uint32_t chunks, eden_random random, uint8_t *packed, uint32_t before) {
    const uint32_t number = before + blockIdx.x, group = number / chunks, chunk = number - group * chunks;
    const uint32_t row = group * kRowsEach + threadIdx.x / 32, within = threadIdx.x % 32, col = chunk * kChunk + within * 8;
    const bool has = row < rows;                                   // (all lanes take part in the exchanges)
    Eight<DTYPE> in;
    in.load(x + (has ? row : 0) * ldx, col, has ? valid_of(col, cols) : 0);
    float v[8];
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = in[i];
        largest = max(largest, magnitude_bits(v[i]));
    }
    const uint32_t t = mx4_exponent(largest_of_quad(largest));
    uint32_t codes;
    if constexpr (STOCHASTIC) codes = mx4_codes(v, t, bits_of(key_of(random, eden::kStreamRounding), row * words_of(cols) + col / 4));
    else codes = mx4_codes(v, t);
    // the exponents of four blocks, one in each lane's byte, come together
    uint32_t four = t << (8 * ((within >> 2) & 3));
    four |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)four, 0x141, 0xF, 0xF, false);
    four |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)four, 0x140, 0xF, 0xF, false);
    if (!has) return;
    *reinterpret_cast<uint32_t *>(packed + (size_t)(row * (uint64_t)chunks + chunk) * kChunkBytes + within * 4) = codes;
    if (within % 16 == 0) *reinterpret_cast<uint32_t *>(packed + (size_t)rows * chunks * kChunkBytes + exps_at(rows, row, chunk) + within / 4) = four;
}

constexpr int kWide = 128, kWaves = 8;                             // columns of a workgroup

template <uint32_t DTYPE, bool STOCHASTIC>
__global__ __launch_bounds__(kWaves * 64) void k_mx4_columns(const typename Elem<DTYPE>::type *x, size_t ldx, uint32_t rows, uint32_t cols, uint32_t chunks, eden_random random, uint8_t *packed,
                                                             float *sums, uint64_t ld_sums, uint32_t accumulate, uint32_t chunks_each) {
    using T = typename Elem<DTYPE>::type;
    __shared__ u32x4 codes[kWide * 8];                             // column c, block b at 8 c + (b ^ (c / 2 mod 8))
    __shared__ uint8_t exps[kWide * 8];
    __shared__ float shared[kWaves][kWide];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col0 = blockIdx.x * kWide, col = col0 + 2 * lane;
    const int valid = col < cols ? (int)min(2u, cols - col) : 0;
    const uint64_t key = STOCHASTIC ? key_of(random, eden::kStreamRounding) : 0, words = words_of(rows);
    uint8_t *all_exps = packed + (size_t)cols * chunks * kChunkBytes;
    float sum[2] = {0.0f, 0.0f};
    const uint32_t first = blockIdx.y * chunks_each, end = min(chunks, first + chunks_each);
    for (uint32_t chunk = first; chunk < end; ++chunk) {
        const uint32_t row0 = chunk * kChunk + wave * kBlock;
        Vec<T, 2> in[kBlock];
#pragma unroll
        for (int r = 0; r < kBlock; ++r) in[r] = load_some<T, 2>(x + (row0 + r < rows ? row0 + r : 0) * ldx + col, row0 + r < rows ? valid : 0);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t largest = 0;
#pragma unroll
            for (int r = 0; r < kBlock; ++r) {
                const float v = (float)in[r].v[c];
                largest = max(largest, magnitude_bits(v));
                sum[c] += v;
            }
            const uint32_t t = mx4_exponent(largest);
            u32x4 four;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = (float)in[8 * q + i].v[c];
                if constexpr (STOCHASTIC) four[q] = mx4_codes(v, t, bits_of(key, (col + c) * words + (row0 + 8 * q) / 4));
                else four[q] = mx4_codes(v, t);
            }
            codes[(2 * lane + c) * 8 + (wave ^ (lane & 7))] = four;
            exps[(2 * lane + c) * 8 + wave] = (uint8_t)t;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < kWide * 8; i += kWaves * 64) {
            const uint32_t c = i >> 3, b = i & 7;
            if (col0 + c < cols) *reinterpret_cast<u32x4 *>(packed + ((size_t)(col0 + c) * chunks + chunk) * kChunkBytes + b * 16) = codes[c * 8 + (b ^ ((c >> 1) & 7))];
        }
        if (threadIdx.x < kWide && col0 + threadIdx.x < cols)
            *reinterpret_cast<u32x2 *>(all_exps + exps_at(cols, col0 + threadIdx.x, chunk)) = *reinterpret_cast<const u32x2 *>(exps + threadIdx.x * 8);
        __syncthreads();
    }
    if (sums == nullptr) return;
    shared[wave][2 * lane] = sum[0], shared[wave][2 * lane + 1] = sum[1];
    __syncthreads();
    if (threadIdx.x < kWide && col0 + threadIdx.x < cols) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += shared[w][threadIdx.x];
        float *to = sums + blockIdx.y * ld_sums + col0 + threadIdx.x;
        *to = accumulate ? *to + s : s;
    }
}

template <uint32_t DTYPE>
__global__ __launch_bounds__(kThreads) void k_mx4_restore(const uint8_t *packed, uint32_t rows, uint32_t cols, uint32_t chunks, typename Elem<DTYPE>::type *x, size_t ldx, uint32_t before) {
    const uint32_t number = before + blockIdx.x, group = number / chunks, chunk = number - group * chunks;
    const uint32_t row = group * kRowsEach + threadIdx.x / 32, within = threadIdx.x % 32, col = chunk * kChunk + within * 8;
    if (row >= rows || col >= cols) return;
    const uint32_t codes = *reinterpret_cast<const uint32_t *>(packed + (size_t)(row * (uint64_t)chunks + chunk) * kChunkBytes + within * 4);
    const uint8_t t = packed[(size_t)rows * chunks * kChunkBytes + exps_at(rows, row, chunk) + within / 4];
    float v[8];
    mx4_values(codes, mx4_unit(t), v);
    store_eight<DTYPE>(x + row * ldx, col, v, valid_of(col, cols));
}

// f(workgroups before a launch, workgroups of it) until all are launched
template <class F> hipError_t by_chunks(uint32_t rows, uint32_t chunks, F f) {
    Spread s = {};
    s.groups = (uint64_t)((rows + kRowsEach - 1) / kRowsEach) * chunks;
    return launches(s, f);
}

}  // namespace

hipError_t launch_mx4_rows(uint32_t dtype, const void *x, size_t ldx, uint32_t rows, uint32_t cols, const Rounding &rounding, uint8_t *packed, hipStream_t st) {
    const uint32_t chunks = chunks_of(cols);
    return by_chunks(rows, chunks, [&](uint32_t before, uint32_t groups) {
        for_type(dtype, [&](auto t) {
            using T = typename Elem<decltype(t)::value>::type;
            if (rounding.stochastic) k_mx4_rows<decltype(t)::value, true><<<groups, kThreads, 0, st>>>(static_cast<const T *>(x), ldx, rows, cols, chunks, rounding.random, packed, before);
            else k_mx4_rows<decltype(t)::value, false><<<groups, kThreads, 0, st>>>(static_cast<const T *>(x), ldx, rows, cols, chunks, rounding.random, packed, before);
        });
    });
}

hipError_t launch_mx4_columns(uint32_t dtype, const void *x, size_t ldx, uint32_t rows, uint32_t cols, const Rounding &rounding, uint8_t *packed, float *sums, uint64_t ld_sums, uint32_t accumulate,
                              uint32_t chunks_each, hipStream_t st) {
    const uint32_t chunks = chunks_of(rows);
    const dim3 grid((cols + kWide - 1) / kWide, (chunks + chunks_each - 1) / chunks_each);
    for_type(dtype, [&](auto t) {
        using T = typename Elem<decltype(t)::value>::type;
        if (rounding.stochastic)
            k_mx4_columns<decltype(t)::value, true><<<grid, kWaves * 64, 0, st>>>(static_cast<const T *>(x), ldx, rows, cols, chunks, rounding.random, packed, sums, ld_sums, accumulate, chunks_each);
        else
            k_mx4_columns<decltype(t)::value, false><<<grid, kWaves * 64, 0, st>>>(static_cast<const T *>(x), ldx, rows, cols, chunks, rounding.random, packed, sums, ld_sums, accumulate, chunks_each);
    });
    return hipGetLastError();
}

hipError_t launch_mx4_restore(uint32_t dtype, const uint8_t *packed, uint32_t rows, uint32_t cols, void *x, size_t ldx, hipStream_t st) {
    const uint32_t chunks = chunks_of(cols);
    return by_chunks(rows, chunks, [&](uint32_t before, uint32_t groups) {
        for_type(dtype, [&](auto t) {
            using T = typename Elem<decltype(t)::value>::type;
            k_mx4_restore<decltype(t)::value><<<groups, kThreads, 0, st>>>(packed, rows, cols, chunks, static_cast<T *>(x), ldx, before);
        });
    });
}

}  // namespace eden_layers
