// Device-side building blocks of the operators around a residual block: random bits, sums over a row's lanes, norms.
#ifndef EDEN_BLOCKS_DEVICE_H
#define EDEN_BLOCKS_DEVICE_H

#include "eden_blocks.h"
#include "eden_hash.h"
#include "eden_layers_device.h"

namespace eden_layers {

// ---- random bits

__device__ inline uint64_t key_of(const eden_random &random, uint32_t stream) {
    return eden::stream_key(random.seed + (random.seed_at ? *random.seed_at : 0), stream, random.id);
}
// Words of a row: four columns each.
__host__ __device__ inline uint64_t words_of(uint64_t cols) { return (cols + 3) / 4; }
// The 16 bits of eight neighbouring columns, two to a register, the first in the low half; `word`: of the first four
struct Bits8 {
    uint32_t pair[4];
    __device__ uint32_t of(int i) const { return i & 1 ? pair[i >> 1] >> 16 : pair[i >> 1] & 0xFFFFu; }
};
__device__ inline Bits8 bits_of(uint64_t key, uint64_t word) {
    const uint64_t a = eden::hash_word(key, word), b = eden::hash_word(key, word + 1);
    return {{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)}};
}
// What kept values are multiplied by
__host__ __device__ inline float kept_scale(uint32_t threshold) { return 65536.0f / (float)(65536u - threshold); }

// ---- sums over the LANES lanes (a power of two) that share a row; all of them get the sum

template <int CONTROL> __device__ inline float of_lane(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CONTROL, 0xF, 0xF, false)); }
template <int LANES> __device__ inline float sum_in_wave(float v) {
    if constexpr (LANES > 1) v += of_lane<0xB1>(v);                // lane ^ 1
    if constexpr (LANES > 2) v += of_lane<0x4E>(v);                // lane ^ 2
    if constexpr (LANES > 4) v += of_lane<0x141>(v);               // 7 - lane of eight: the other four
    if constexpr (LANES > 8) v += of_lane<0x140>(v);               // 15 - lane of sixteen: the other eight
    if constexpr (LANES > 16) v += __shfl_xor(v, 16);
    if constexpr (LANES > 32) v += __shfl_xor(v, 32);
    return v;
}
// N sums at once.  A row of several waves goes through the LDS: `shared` has 2 N floats a wave, used in turn (`turn` is 0 or 1), so that one
// barrier a call is enough.
template <int LANES, int N> __device__ inline void sum_in_row(float (&v)[N], float *shared, int &turn) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = sum_in_wave<(LANES < 64 ? LANES : 64)>(v[n]);
    if constexpr (LANES > 64) {
        constexpr int kWaves = LANES / 64;
        float *place = shared + turn * (2 * kWaves);
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) place[n * kWaves + (threadIdx.x >> 6)] = v[n];
        }
        __syncthreads();
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = sum_in_wave<kWaves>(place[n * kWaves + (lane & (kWaves - 1))]);
    }
}
template <int LANES> constexpr int kSumFloats = LANES > 64 ? 4 * (LANES / 64) : 1;       // N up to 2

// ---- eight values of a row, as they lie in memory

template <uint32_t DTYPE> struct Eight {
    using T = typename Elem<DTYPE>::type;
    Vec<T, 8> raw;
    __device__ void load(const void *row, uint32_t col, int valid) { raw = load_some<T, 8>(static_cast<const T *>(row) + col, valid); }
    __device__ float operator[](int i) const { return (float)raw.v[i]; }
};
template <uint32_t DTYPE> __device__ inline void store_eight(void *row, uint32_t col, const float (&v)[8], int valid) {
    using T = typename Elem<DTYPE>::type;
    Vec<T, 8> to;
#pragma unroll
    for (int i = 0; i < 8; ++i) to.v[i] = (T)v[i];
    store_some<T, 8>(static_cast<T *>(row) + col, to, valid);
}

template <uint32_t DTYPE> __device__ inline const void *row_of(const void *p, uint64_t row, uint64_t ld) { return static_cast<const typename Elem<DTYPE>::type *>(p) + row * ld; }
template <uint32_t DTYPE> __device__ inline void *row_of(void *p, uint64_t row, uint64_t ld) { return static_cast<typename Elem<DTYPE>::type *>(p) + row * ld; }

}  // namespace eden_layers

#endif  // EDEN_BLOCKS_DEVICE_H
