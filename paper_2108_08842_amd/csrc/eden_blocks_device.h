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
// (the hash's 64-bit products are most of it: `state` is what a word is mixed from, key + phi (word + 1), and the next word's is phi more)
__device__ inline uint64_t state_of(uint64_t key, uint64_t word) { return key + eden::kPhi * (word + 1); }
__device__ inline Bits8 bits_of(uint64_t state) {
    const uint64_t a = eden::mix64(state), b = eden::mix64(state + eden::kPhi);
    return {{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)}};
}
__device__ inline Bits8 bits_of(uint64_t key, uint64_t word) { return bits_of(state_of(key, word)); }
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
// N sums at once.  A row of several waves goes through the LDS: `shared` has kSumFloats floats, used in turn (`turn` is 0 or 1), so that one
// barrier a call is enough.
template <int LANES, int N> __device__ inline void sum_in_row(float (&v)[N], float *shared, int &turn) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = sum_in_wave<(LANES < 64 ? LANES : 64)>(v[n]);
    if constexpr (LANES > 64) {
        constexpr int kWaves = LANES / 64;
        float *place = shared + turn * (3 * kWaves);
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
template <int LANES> constexpr int kSumFloats = LANES > 64 ? 6 * (LANES / 64) : 1;       // N up to 3

// What a norm multiplies a row by: 1 / sqrt(sum / cols + eps), each = 1 / cols, `sum` that of the squares.  The mean of the squares may be in fp32's range where their sum, or one of them, is
// not (rows of 16384 values of 2^57): then it is taken once more of values 2^-72 times as large, behind a branch that a whole wave takes or does not.  squares(by): the lane's part of the sum for
// values times `by`.
constexpr float kMostFinite = 3.402823466e+38f;
template <int LANES, class F> __device__ inline float rho_of(float sum, float each, float eps, float *shared, int turn, F squares) {
    float rho = rsqrtf(sum * each + eps);
    const bool past = sum > kMostFinite;
    if (__builtin_expect(__builtin_amdgcn_readfirstlane((int)(LANES >= 64 ? past : __any(past))), 0)) {
        float again[1] = {squares(0x1p-72f)};
        sum_in_row<LANES>(again, shared, turn);
        if constexpr (LANES > 64) __syncthreads();                 // (the caller's next sum has the same turn)
        if (past) rho = 0x1p-72f * rsqrtf(again[0] * each + 0x1p-144f * eps);
    }
    return rho;
}

// ---- eight values of a row, as they lie in memory

// 16 bytes of memory at any multiple of two (what the part asks for at most), in its own address space: a flat address would wait for the LDS as well
typedef u32x4 piece_anywhere __attribute__((aligned(2)));
typedef const __attribute__((address_space(1))) piece_anywhere *piece_in_memory;
typedef __attribute__((address_space(1))) piece_anywhere *piece_to_memory;

template <uint32_t DTYPE> struct Eight {
    using T = typename Elem<DTYPE>::type;
    static constexpr int kWords = sizeof(T) * 2, kOfWord = 4 / sizeof(T);
    Vec<T, 8> raw;
    __device__ void load(const void *row, uint32_t col, int valid) { raw = load_some<T, 8>(static_cast<const T *>(row) + col, valid); }
    // (32-bit byte offsets from a row that is the same for all lanes: the address stays in scalar registers)
    __device__ void load(const void *row, uint32_t bytes) {
        u32x4 words[kWords / 4];
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) words[i] = *(piece_in_memory)(reinterpret_cast<uintptr_t>(row) + bytes + 16 * i);
        __builtin_memcpy(&raw, words, sizeof(raw));
    }
    __device__ float operator[](int i) const { return (float)raw.v[i]; }
    __device__ void fill(float v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) raw.v[i] = (T)v;
    }
    // Without its first `count` values, zeros behind the others
    __device__ void shift(uint32_t count) {
        uint32_t w[kWords + 1];
        __builtin_memcpy(w, &raw, sizeof(raw));
        w[kWords] = 0;
        if constexpr (kOfWord == 2) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = count & 1 ? __builtin_amdgcn_alignbit(w[i + 1], w[i], 16) : w[i];
        }
#pragma unroll
        for (int by = 1; by <= kWords; by *= 2)
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = count & (by * kOfWord) ? (i + by < kWords ? w[i + by] : 0u) : w[i];
        __builtin_memcpy(&raw, w, sizeof(raw));
    }
    // Without this the compiler keeps the fp32 values that one use has made of these for the next use, at twice the registers
    __device__ void stay_packed() {
        uint32_t w[kWords];
        __builtin_memcpy(w, &raw, sizeof(raw));
#pragma unroll
        for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
        __builtin_memcpy(&raw, w, sizeof(raw));
    }
    __device__ void keep(bool it) {
        uint32_t w[kWords];
        __builtin_memcpy(w, &raw, sizeof(raw));
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = it ? w[i] : 0u;
        __builtin_memcpy(&raw, w, sizeof(raw));
    }
};
template <uint32_t DTYPE, bool STREAM = false> __device__ inline void store_eight(void *row, uint32_t col, const float (&v)[8], int valid) {
    using T = typename Elem<DTYPE>::type;
    Vec<T, 8> to;
#pragma unroll
    for (int i = 0; i < 8; ++i) to.v[i] = (T)v[i];
    if constexpr (STREAM) stream_some<T, 8>(static_cast<T *>(row) + col, to, valid);
    else store_some<T, 8>(static_cast<T *>(row) + col, to, valid);
}

// A lane's columns in a row that LANES lanes share, eight at a time.  Loads take no branch.  RAGGED (rows that are no multiple of eight): a lane whose eight columns end behind the
// row's end reads the row's last eight, and settle() puts them in their place.  A lane that has none reads others and settle() makes them zeros.  (LANES 1: rows of
// less than eight columns.)
template <uint32_t DTYPE, int LANES, int CHUNKS, bool RAGGED> struct RowPlace {
    using T = typename Elem<DTYPE>::type;
    uint32_t col[CHUNKS], at[CHUNKS];                              // at: bytes
    int valid[CHUNKS];
    bool partial;                                                  // the same for all lanes

    __device__ RowPlace(uint32_t cols, uint32_t lane) : partial(cols < LANES * CHUNKS * 8) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            col[c] = (c * LANES + lane) * 8;
            valid[c] = col[c] < cols ? (int)min(8u, cols - col[c]) : 0;
            at[c] = (LANES == 1 ? 0 : valid[c] == 8 ? col[c] : cols - 8) * (uint32_t)sizeof(T);
        }
    }
    __device__ bool inside(int c, int i) const { return RAGGED ? i < valid[c] : valid[c] != 0; }
    __device__ void load(Eight<DTYPE> &to, const void *row, int c) const {
        if constexpr (LANES == 1) to.load(row, 0, valid[0]);
        else to.load(row, at[c]);
    }
    // has: whether there is such a row (LANES below 64: several share a wave)
    __device__ void settle(Eight<DTYPE> &v, int c, bool has) const {
        if constexpr (LANES == 1) {
            v.keep(has);
        } else if constexpr (RAGGED) {
            v.shift(has ? 8 - valid[c] : 8);
        } else {
            if (partial) v.keep(valid[c] != 0);
            if constexpr (LANES < 64) v.keep(has);
        }
    }
    template <bool STREAM> __device__ void store(void *row, int c, const float (&v)[8]) const {
        if constexpr (RAGGED) {
            if (valid[c]) store_eight<DTYPE, STREAM>(row, col[c], v, valid[c]);
        } else if (valid[c]) {
            Vec<T, 8> to;
#pragma unroll
            for (int i = 0; i < 8; ++i) to.v[i] = (T)v[i];
            u32x4 words[sizeof(T) / 2];
            __builtin_memcpy(words, &to, sizeof(to));
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
                const piece_to_memory to_piece = (piece_to_memory)(reinterpret_cast<uintptr_t>(row) + col[c] * (uint32_t)sizeof(T) + 16 * i);
                if constexpr (STREAM && sizeof(T) == 2) __builtin_nontemporal_store(words[i], to_piece);
                else *to_piece = words[i];
            }
        }
    }
};
// The number of the row among those side by side in a workgroup; the same for all lanes of a wave where a row has a wave or more
template <int LANES> __device__ inline uint32_t row_in_group() {
    if constexpr (LANES > 64) return 0;
    if constexpr (LANES == 64) return (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64));
    return threadIdx.x / LANES;
}

// Address of a row.  The compiler does not see where it comes from: it would add a lane's columns to the matrix's address instead, outside of the loop over the rows, and keep two registers
// for every operand.  (A row of a wave or more: the same address in all lanes.)
template <int LANES, class P> __device__ inline P *fixed_address(P *p) {
    if constexpr (LANES >= 64) asm("" : "+s"(p));
    else asm("" : "+v"(p));
    return p;
}
template <uint32_t DTYPE, int LANES> __device__ inline const void *row_of(const void *p, uint64_t row, uint64_t ld) {
    return fixed_address<LANES>(static_cast<const typename Elem<DTYPE>::type *>(p) + row * ld);
}
template <uint32_t DTYPE, int LANES> __device__ inline void *row_of(void *p, uint64_t row, uint64_t ld) { return fixed_address<LANES>(static_cast<typename Elem<DTYPE>::type *>(p) + row * ld); }

}  // namespace eden_layers

#endif  // EDEN_BLOCKS_DEVICE_H
