// 4 bits from and to values.
//
// Bound by memory, the stochastic rounding by the vector unit: two 64-bit products of the hash for every four values, each several 32-bit ones at a quarter of the rate.  Rows: a thread has eight neighbouring
// columns, four threads a block, 32 threads a chunk, whose exponents leave in words.
// Transpose: a workgroup has 256 rows of 128 columns, a wave 32 rows of them and a lane eight columns of eight rows: loads of 16 bytes, four lanes to a block, whose codes are a word
// each; codes and exponents go through the LDS and leave in whole lines.
//
// 8192 x 16384 bf16 (268 MB of values, 71 of 4 bits): rows to the nearest 58 us = 5.8 TB/s, stochastically 101 to 107; the transpose to the nearest 68 to 71 = 4.9 TB/s, stochastically 103 to 105 with vector
// instructions in four fifths of the cycles, with sums of columns 109 in two launches; restored 45 in a loop (part of it from the last cache), 60 with other work between.
// Restoring stores past the caches: 109 -> 47 us.  The transpose by loads of 16 bytes: 166 -> 68 (of single columns by neighbouring lanes before).
#include "eden_layers_spread.h"
#include "eden_mx4_kernels.h"

namespace eden_layers {
namespace {

constexpr int kThreads = 256;

// A workgroup has 2^shift neighbouring chunks of each of its 8 / 2^shift rows; workgroups go round the eight XCDs in turn, and each of them gets a run of neighbouring ones (the exponents of
// neighbouring rows share lines).
struct ChunkPlace {
    uint32_t row, chunk, within;
    // each: such rows one after the other
    __device__ ChunkPlace(uint32_t shift, uint32_t before, uint32_t groups, uint32_t each = 1) {
        const uint32_t xcd = blockIdx.x & 7u, run = gridDim.x >> 3, more = gridDim.x & 7u, number = before + xcd * run + min(xcd, more) + (blockIdx.x >> 3);
        const uint32_t group = number / groups, unit = threadIdx.x / 32;
        row = group * each * (8u >> shift) + (unit >> shift);
        chunk = ((number - group * groups) << shift) + (unit & ((1u << shift) - 1));
        within = threadIdx.x % 32;
    }
};

template <uint32_t DTYPE, bool STOCHASTIC>
__global__ __launch_bounds__(kThreads) void k_mx4_rows(const typename Elem<DTYPE>::type *x, size_t ldx, uint32_t rows, uint32_t cols, uint32_t chunks, eden_random random, uint8_t *packed, uint32_t before, uint32_t shift,
                                                       uint32_t groups, uint32_t each) {
    const ChunkPlace place(shift, before, groups, each);
    const uint32_t chunk = place.chunk, within = place.within, col = chunk * kChunk + within * 8, step = 8u >> shift;
    const int valid = chunk < chunks ? valid_of(col, cols) : 0;
    uint64_t state = 0;
    const uint64_t words = words_of(cols);
    if constexpr (STOCHASTIC) state = state_of(key_of(random, eden::kStreamRounding), place.row * words + col / 4);
    for (uint32_t row = place.row, i = 0; i < each; ++i, row += step, state += eden::kPhi * words * step) {
        const bool has = row < rows && chunk < chunks;             // (all lanes take part in the exchanges)
        Eight<DTYPE> in;
        in.load(x + (has ? row : 0) * ldx, col, has ? valid : 0);
        float v[8];
        uint32_t largest = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = in[e];
            largest = max(largest, magnitude_bits(v[e]));
        }
        const uint32_t t = mx4_exponent(largest_of_quad(largest));
        uint32_t codes;
        if constexpr (STOCHASTIC) codes = mx4_codes(v, t, bits_of(state));
        else codes = mx4_codes(v, t);
        // the exponents of four blocks, one in each lane's byte, come together
        uint32_t four = t << (8 * ((within >> 2) & 3));
        four |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)four, 0x141, 0xF, 0xF, false);
        four |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)four, 0x140, 0xF, 0xF, false);
        if (!has) continue;
        *reinterpret_cast<uint32_t *>(packed + (size_t)(row * (uint64_t)chunks + chunk) * kChunkBytes + within * 4) = codes;
        if (within % 16 == 0) *reinterpret_cast<uint32_t *>(packed + (size_t)rows * chunks * kChunkBytes + exps_at(rows, row, chunk) + within / 4) = four;
    }
}

constexpr int kWide = 128, kWaves = 8;                             // columns of a workgroup

// The largest over the four lanes that share columns (16 apart)
__device__ inline uint32_t largest_of_four(uint32_t v) {
    v = max(v, (uint32_t)__shfl_xor((int)v, 16));
    return max(v, (uint32_t)__shfl_xor((int)v, 32));
}

// Four waves of a SIMD are two workgroups to a CU: 128 registers are enough, and the compiler takes more if it may (8192 x 16384 stochastically 145 us against 108, to the nearest the same).
template <uint32_t DTYPE, bool STOCHASTIC>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(4))) void k_mx4_columns(const typename Elem<DTYPE>::type *x, size_t ldx, uint32_t rows, uint32_t cols, uint32_t chunks, eden_random random, uint8_t *packed,
                                                             float *sums, uint64_t ld_sums, uint32_t accumulate, uint32_t chunks_each, uint32_t wide) {
    __shared__ uint32_t codes[kWide * 32];                         // column c, block b, word g at 32 c + 4 (b ^ (c / 8 mod 8)) + g
    __shared__ __attribute__((aligned(8))) uint8_t exps[kWide * 8];
    __shared__ float shared[kWaves][kWide];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane >> 4;
    // workgroups go round the eight XCDs in turn; each of them gets a run of neighbouring columns
    const uint32_t xcd = blockIdx.x & 7u, each = gridDim.x >> 3, more = gridDim.x & 7u, number = xcd * each + min(xcd, more) + (blockIdx.x >> 3);
    const uint32_t part = number / wide, col0 = (number - part * wide) * kWide, col = col0 + 8 * (lane & 15);
    const int valid = valid_of(col, cols);
    const uint64_t key = STOCHASTIC ? key_of(random, eden::kStreamRounding) : 0, words = words_of(rows);
    uint8_t *all_exps = packed + (size_t)cols * chunks * kChunkBytes;
    float sum[8] = {};
    const uint32_t first = part * chunks_each, end = min(chunks, first + chunks_each);
    for (uint32_t chunk = first; chunk < end; ++chunk) {
        const uint32_t row0 = chunk * kChunk + wave * kBlock + group * 8;          // of this lane's eight rows
        const uint64_t step = eden::kPhi * words;
        uint64_t state = STOCHASTIC ? state_of(key, col * words + row0 / 4) : 0;
        Eight<DTYPE> in[8];
        if (col0 + kWide <= cols && (chunk + 1) * kChunk <= rows) {
#pragma unroll
            for (int r = 0; r < 8; ++r) in[r].load(x + (row0 + r) * ldx, (uint32_t)(col * sizeof(x[0])));
        } else {
#pragma unroll
            for (int r = 0; r < 8; ++r) in[r].load(x + (row0 + r < rows ? row0 + r : 0) * ldx, col, row0 + r < rows ? valid : 0);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            uint32_t largest = 0;
            float v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                v[r] = in[r][c];
                largest = max(largest, magnitude_bits(v[r]));
                sum[c] += v[r];
            }
            const uint32_t t = mx4_exponent(largest_of_four(largest)), at = 8 * (lane & 15) + c;
            uint32_t word;
            if constexpr (STOCHASTIC) word = mx4_codes(v, t, bits_of(state)), state += step;
            else word = mx4_codes(v, t);
            codes[at * 32 + (wave ^ (lane & 7)) * 4 + group] = word;
            if (group == 0) exps[at * 8 + wave] = (uint8_t)t;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < kWide * 8; i += kWaves * 64) {
            const uint32_t c = i >> 3, b = i & 7;
            if (col0 + c < cols)
                *reinterpret_cast<u32x4 *>(packed + ((size_t)(col0 + c) * chunks + chunk) * kChunkBytes + b * 16) = *reinterpret_cast<const u32x4 *>(codes + c * 32 + (b ^ ((c >> 3) & 7)) * 4);
        }
        if (threadIdx.x < kWide && col0 + threadIdx.x < cols)
            *reinterpret_cast<u32x2 *>(all_exps + exps_at(cols, col0 + threadIdx.x, chunk)) = *reinterpret_cast<const u32x2 *>(exps + threadIdx.x * 8);
        __syncthreads();
    }
    if (sums == nullptr) return;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        sum[c] += __shfl_xor(sum[c], 16);
        sum[c] += __shfl_xor(sum[c], 32);
        if (group == 0) shared[wave][8 * (lane & 15) + c] = sum[c];
    }
    __syncthreads();
    if (threadIdx.x < kWide && col0 + threadIdx.x < cols) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += shared[w][threadIdx.x];
        float *to = sums + part * ld_sums + col0 + threadIdx.x;
        *to = accumulate ? *to + s : s;
    }
}

template <uint32_t DTYPE>
__global__ __launch_bounds__(kThreads) void k_mx4_restore(const uint8_t *packed, uint32_t rows, uint32_t cols, uint32_t chunks, typename Elem<DTYPE>::type *x, size_t ldx, uint32_t before, uint32_t shift, uint32_t groups) {
    const ChunkPlace place(shift, before, groups);
    const uint32_t row = place.row, chunk = place.chunk, within = place.within, col = chunk * kChunk + within * 8;
    if (row >= rows || col >= cols) return;
    const uint32_t codes = *reinterpret_cast<const uint32_t *>(packed + (size_t)(row * (uint64_t)chunks + chunk) * kChunkBytes + within * 4);
    const uint8_t t = packed[(size_t)rows * chunks * kChunkBytes + exps_at(rows, row, chunk) + within / 4];
    float v[8];
    mx4_values(codes, mx4_unit(t), v);
    store_eight<DTYPE, true>(x + row * ldx, col, v, valid_of(col, cols));
}

// f(workgroups before a launch, workgroups of it, shift, workgroups along a row) until all are launched
template <class F> hipError_t by_chunks(uint32_t rows, uint32_t chunks, uint32_t each, F f) {
    const uint32_t shift = chunks >= 4 ? 2 : chunks >= 2 ? 1 : 0, along = (chunks + (1u << shift) - 1) >> shift, rows_each = each * (8u >> shift);
    Spread s = {};
    s.groups = (uint64_t)((rows + rows_each - 1) / rows_each) * along;
    return launches(s, [&](uint32_t before, uint32_t groups) { f(before, groups, shift, along); });
}

}  // namespace

hipError_t launch_mx4_rows(uint32_t dtype, const void *x, size_t ldx, uint32_t rows, uint32_t cols, const Rounding &rounding, uint8_t *packed, hipStream_t st) {
    // Four rows a thread where there is more than the device holds at once: the key of the random numbers and the first row's word are made once for them (8192 x 16384 stochastically 140 us against 120,
    // 8192 x 4096 31 against 28, to the nearest 15.6 against 14.3, with the codes made in more instructions than now; 1024 x 4096 is below and takes 6.7 either way)
    const uint32_t chunks = chunks_of(cols), each = (uint64_t)rows * chunks >= (1u << 16) ? 4 : 1;
    return by_chunks(rows, chunks, each, [&](uint32_t before, uint32_t groups, uint32_t shift, uint32_t along) {
        for_type(dtype, [&](auto t) {
            using T = typename Elem<decltype(t)::value>::type;
            if (rounding.stochastic) k_mx4_rows<decltype(t)::value, true><<<groups, kThreads, 0, st>>>(static_cast<const T *>(x), ldx, rows, cols, chunks, rounding.random, packed, before, shift, along, each);
            else k_mx4_rows<decltype(t)::value, false><<<groups, kThreads, 0, st>>>(static_cast<const T *>(x), ldx, rows, cols, chunks, rounding.random, packed, before, shift, along, each);
        });
    });
}

hipError_t launch_mx4_columns(uint32_t dtype, const void *x, size_t ldx, uint32_t rows, uint32_t cols, const Rounding &rounding, uint8_t *packed, float *sums, uint64_t ld_sums, uint32_t accumulate,
                              uint32_t chunks_each, hipStream_t st) {
    const uint32_t chunks = chunks_of(rows);
    const uint32_t wide = (cols + kWide - 1) / kWide;
    const uint32_t grid = wide * ((chunks + chunks_each - 1) / chunks_each);
    for_type(dtype, [&](auto t) {
        using T = typename Elem<decltype(t)::value>::type;
        if (rounding.stochastic)
            k_mx4_columns<decltype(t)::value, true><<<grid, kWaves * 64, 0, st>>>(static_cast<const T *>(x), ldx, rows, cols, chunks, rounding.random, packed, sums, ld_sums, accumulate, chunks_each, wide);
        else
            k_mx4_columns<decltype(t)::value, false><<<grid, kWaves * 64, 0, st>>>(static_cast<const T *>(x), ldx, rows, cols, chunks, rounding.random, packed, sums, ld_sums, accumulate, chunks_each, wide);
    });
    return hipGetLastError();
}

hipError_t launch_mx4_restore(uint32_t dtype, const uint8_t *packed, uint32_t rows, uint32_t cols, void *x, size_t ldx, hipStream_t st) {
    const uint32_t chunks = chunks_of(cols);
    return by_chunks(rows, chunks, 1, [&](uint32_t before, uint32_t groups, uint32_t shift, uint32_t along) {
        for_type(dtype, [&](auto t) {
            using T = typename Elem<decltype(t)::value>::type;
            k_mx4_restore<decltype(t)::value><<<groups, kThreads, 0, st>>>(packed, rows, cols, chunks, static_cast<T *>(x), ldx, before, shift, along);
        });
    });
}

}  // namespace eden_layers
