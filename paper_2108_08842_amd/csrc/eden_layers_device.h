// Device-side building blocks of the layer kernels (gfx950, wave64): operand types, the 8-bit checkpoint, activations, and the
// end of a product (bias, activation, residual, slope, checkpoint).
#ifndef EDEN_LAYERS_DEVICE_H
#define EDEN_LAYERS_DEVICE_H

#include <hip/hip_runtime.h>

#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "eden_layers.h"

namespace eden_layers {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;

constexpr int kBlock = 32;                  // columns of a checkpoint block

__host__ __device__ inline size_t blocks_of(size_t cols) { return (cols + kBlock - 1) / kBlock; }

// ---- elements

template <uint32_t DTYPE> struct Elem;
template <> struct Elem<EDEN_F32> {
    using type = float;
    static constexpr int kBytes = 4;
};
template <> struct Elem<EDEN_F16> {
    using type = _Float16;
    static constexpr int kBytes = 2;
};
template <> struct Elem<EDEN_BF16> {
    using type = __bf16;
    static constexpr int kBytes = 2;
};

// N consecutive elements from any address of their own alignment (the part reads and writes unaligned vectors); elements from
// `valid` on are 0 / not written.
template <class T, int N> struct Vec { T v[N]; };

template <class T, int N> __device__ inline Vec<T, N> load_some(const T *p, int valid) {
    Vec<T, N> r;
    if (valid >= N) {
        __builtin_memcpy(&r, p, sizeof(r));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = i < valid ? p[i] : (T)0.0f;
    }
    return r;
}
template <class T, int N> __device__ inline void store_some(T *p, const Vec<T, N> &r, int valid) {
    if (valid >= N) {
        __builtin_memcpy(p, &r, sizeof(r));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < valid) p[i] = r.v[i];
    }
}

// The same past the caches where it is 16 bytes.  Measured on results that the caches could not hold; a short result goes the same way, and what its next reader pays for that has not been measured.  Neighbouring lanes have to have neighbouring pieces: 32 bytes a lane in two such stores write every line twice.
template <class T, int N> __device__ inline void stream_some(T *p, const Vec<T, N> &r, int valid) {
    if constexpr (sizeof(r) == 16) {
        if (valid >= N) {
            typedef u32x4 anywhere __attribute__((aligned(2)));
            u32x4 words;
            __builtin_memcpy(&words, &r, sizeof(r));
            __builtin_nontemporal_store(words, reinterpret_cast<anywhere *>(p));
            return;
        }
    }
    store_some<T, N>(p, r, valid);
}

// ---- 8-bit checkpoint

// Exponent byte of a block from the bits of its largest |x| (as whole numbers: NaN above infinity above all else).
__device__ inline uint32_t block_exponent(uint32_t largest_bits) {
    const uint32_t e = largest_bits >> 23;
    return e == 255u ? 255u : (uint32_t)max((int)e - 6, 1);
}
// 2^(127 - t), what the values of a block are multiplied by: exact.  A block that is not finite (t = 255) gets 0 and codes of its own.
__device__ inline float block_inverse(uint32_t t) { return t == 255u ? 0.0f : __uint_as_float((254u - t) << 23); }
// 2^(t - 127).  For t = 255 infinity: the codes of such a block are 0, and 0 times infinity is NaN.
__device__ inline float block_unit(uint32_t t) { return __uint_as_float(t << 23); }

// x * inverse is below 128 in size (NaN where the block is not finite: the caller clears those); 1.5 * 2^23 more has its nearest even whole number, a two's
// complement, in the lower byte
__device__ inline uint32_t code_bits(float x, float inverse) { return __float_as_uint(__builtin_amdgcn_fmed3f(x * inverse, -127.0f, 127.0f) + 12582912.0f); }
__device__ inline uint32_t codes4(const float (&x)[4], uint32_t t) {
    const float inverse = block_inverse(t);
    const uint32_t lo = __builtin_amdgcn_perm(code_bits(x[1], inverse), code_bits(x[0], inverse), 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(code_bits(x[3], inverse), code_bits(x[2], inverse), 0x04000C0Cu);
    return t == 255u ? 0u : lo | hi;
}
// Four codes' values.  Exact: seven bits times a power of two.
__device__ inline void values4(uint32_t codes, float unit, float (&x)[4]) {
    x[0] = (float)(int8_t)(codes & 0xFFu) * unit;
    x[1] = (float)(int8_t)((codes >> 8) & 0xFFu) * unit;
    x[2] = (float)(int8_t)((codes >> 16) & 0xFFu) * unit;
    x[3] = (float)(int8_t)(codes >> 24) * unit;
}
// The largest of a value over the two, four lanes around this one (neighbours of a quad by a register move, not through the LDS)
__device__ inline uint32_t largest_of_quad(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0xB1, 0xF, 0xF, false));        // lane ^ 1
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x4E, 0xF, 0xF, false));     // lane ^ 2
}
__device__ inline uint32_t magnitude_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// ---- activations

constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kSqrt2OverPi = 0.79788456080286536f;
constexpr float kTanhCubic = 0.044715f;

// exp and 1 / x: FULL (fp32 results) to an ulp or two; else (results with at most 11 bits) in one instruction each, off by |x| 2^-24 and 2^-23
template <bool FULL> __device__ inline float exp_of(float x) { return FULL ? expf(x) : __expf(x); }
template <bool FULL> __device__ inline float over(float a, float b) { return FULL ? a / b : a * __builtin_amdgcn_rcpf(b); }

// Phi(-|z|) = erfc(|z| / sqrt 2) / 2 for results of at most 11 bits, without a branch: erfc(x) = exp(-x^2) t P(t), t = 1 / (1 + x/2), P of degree 8 fitted to
// exp(x^2) erfc(x) / t in the largest relative error on 0 .. 14: 4.4e-8.  What is left is exp's.  (Degree 6, 2.7e-6, shows where a residual nearly cancels the
// result, and where the slope's two terms cancel, at -0.75; it takes 8 us less in 920 of the largest forward case, 0.2 of 10.5 at 512 x 512 x 512.)  bell: exp(-z^2 / 2).
__device__ inline float normal_tail(float z, float bell) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.5f * kSqrtHalf, fabsf(z), 1.0f));
    float p = -0.029692838f;
    p = __builtin_fmaf(p, t, 0.143060327f);
    p = __builtin_fmaf(p, t, -0.245200247f);
    p = __builtin_fmaf(p, t, 0.140863791f);
    p = __builtin_fmaf(p, t, -0.0145726437f);
    p = __builtin_fmaf(p, t, 0.101875715f);
    p = __builtin_fmaf(p, t, 0.121417664f);
    p = __builtin_fmaf(p, t, 0.141206041f);
    p = __builtin_fmaf(p, t, 0.141042173f);
    return p * t * bell;
}

template <uint32_t ACT, bool FULL> __device__ inline float activate_as(float z) {
    if constexpr (ACT == EDEN_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    else if constexpr (ACT == EDEN_ACT_GELU) {
        if constexpr (FULL) return 0.5f * z * (1.0f + erff(z * kSqrtHalf));
        const float tail = normal_tail(z, __expf(-0.5f * z * z));
        return z * (z > 0.0f ? 1.0f - tail : tail);
    }
    else if constexpr (ACT == EDEN_ACT_GELU_TANH)                  // (1 + tanh u) / 2 = 1 / (1 + exp(-2u))
        return over<FULL>(z, 1.0f + exp_of<FULL>(-2.0f * kSqrt2OverPi * (z + kTanhCubic * z * z * z)));
    else if constexpr (ACT == EDEN_ACT_SILU) return over<FULL>(z, 1.0f + exp_of<FULL>(-z));
    else return z;
}
// Derivative at a checkpoint's value: finite, or NaN for NaN.
template <uint32_t ACT, bool FULL> __device__ inline float slope_as(float z) {
    if constexpr (ACT == EDEN_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    else if constexpr (ACT == EDEN_ACT_GELU) {
        const float bell = exp_of<FULL>(-0.5f * z * z);
        if constexpr (FULL) return 0.5f * (1.0f + erff(z * kSqrtHalf)) + z * kInvSqrt2Pi * bell;
        const float tail = normal_tail(z, bell);
        return (z > 0.0f ? 1.0f - tail : tail) + z * kInvSqrt2Pi * bell;
    }
    else if constexpr (ACT == EDEN_ACT_GELU_TANH) {
        const float c = fminf(fmaxf(z, -12.0f), 12.0f);            // the slope is 0 or 1 in fp32 from there on, and z^3 stays finite
        const float p = over<FULL>(1.0f, 1.0f + exp_of<FULL>(-2.0f * kSqrt2OverPi * (c + kTanhCubic * c * c * c)));
        const float s = p + c * p * (1.0f - p) * (2.0f * kSqrt2OverPi) * (1.0f + 3.0f * kTanhCubic * c * c);
        return z != z ? z : s;
    } else if constexpr (ACT == EDEN_ACT_SILU) {
        const float p = over<FULL>(1.0f, 1.0f + exp_of<FULL>(-z));
        return p * (1.0f + z * (1.0f - p));
    } else return 1.0f;
}

// f(std::integral_constant<uint32_t, ACT>()) for the activation `act`: one branch for all values of a thread
template <class F> __device__ inline void for_activation(uint32_t act, F f) {
    switch (act) {
    case EDEN_ACT_RELU: f(std::integral_constant<uint32_t, EDEN_ACT_RELU>()); break;
    case EDEN_ACT_GELU: f(std::integral_constant<uint32_t, EDEN_ACT_GELU>()); break;
    case EDEN_ACT_GELU_TANH: f(std::integral_constant<uint32_t, EDEN_ACT_GELU_TANH>()); break;
    case EDEN_ACT_SILU: f(std::integral_constant<uint32_t, EDEN_ACT_SILU>()); break;
    default: break;
    }
}
template <bool FULL, int R, int C> __device__ inline void activate_all(float (&v)[R][C], uint32_t act) {
    for_activation(act, [&](auto a) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) v[r][c] = activate_as<decltype(a)::value, FULL>(v[r][c]);
    });
}
template <bool FULL, int R, int C> __device__ inline void multiply_slopes(float (&v)[R][C], const float (&z)[R][C], uint32_t act) {
    for_activation(act, [&](auto a) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) v[r][c] *= slope_as<decltype(a)::value, FULL>(z[r][c]);
    });
}
template <bool FULL> __device__ inline float slope(float z, uint32_t act) {
    float v[1][1] = {{1.0f}};
    const float at[1][1] = {{z}};
    multiply_slopes<FULL>(v, at, act);
    return v[0][0];
}

// ---- the end of a product: from fp32 sums to what the call returns

struct Finish {
    const void *bias;              // per column, dtype (eden_linear)
    const void *residual;          // dtype
    void *out;                     // dtype, or fp32 (eden_linear_weight_grad)
    size_t ld_residual, ld_out;
    uint8_t *codes_out, *exps_out; // checkpoint of z to be written (eden_linear)
    const uint8_t *codes_in, *exps_in;  // checkpoint of z^ to be read (eden_linear_input_grad)
    uint32_t blocks;               // of a row of either checkpoint
    uint32_t activation;
    uint32_t accumulate;           // eden_linear_weight_grad: add to what is there
};

enum Op : int { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };

// z of four consecutive columns, before the checkpoint is taken
template <int OP, uint32_t DTYPE> __device__ inline void finish_bias(const Finish &f, uint32_t col, int valid, float (&v)[4]) {
    using T = typename Elem<DTYPE>::type;
    if constexpr (OP == kForward) {
        if (f.bias) {
            const auto b = load_some<T, 4>(static_cast<const T *>(f.bias) + col, valid);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += (float)b.v[i];
        }
    }
}
// ... and what follows.  `valid`: columns of the four that the result has (the caller sees to it that there is one).
template <int OP, uint32_t DTYPE>
__device__ inline void finish_store(const Finish &f, uint32_t row, uint32_t col, int valid, const float (&sums)[4]) {
    float v[1][4] = {{sums[0], sums[1], sums[2], sums[3]}};
    if constexpr (OP == kWeightGrad) {
        float *out = static_cast<float *>(f.out) + (size_t)row * f.ld_out + col;
        Vec<float, 4> r;
        if (f.accumulate) {
            r = load_some<float, 4>(out, valid);
#pragma unroll
            for (int i = 0; i < 4; ++i) r.v[i] += v[0][i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) r.v[i] = v[0][i];
        }
        store_some<float, 4>(out, r, valid);
    } else {
        using T = typename Elem<DTYPE>::type;
        if constexpr (OP == kForward) {
            activate_all<DTYPE == EDEN_F32>(v, f.activation);
        } else if (f.codes_in) {
            const uint32_t block = col / kBlock;
            float z[1][4];
            uint32_t codes;
            __builtin_memcpy(&codes, f.codes_in + ((size_t)row * f.blocks + block) * kBlock + col % kBlock, 4);
            values4(codes, block_unit(f.exps_in[(size_t)row * f.blocks + block]), z[0]);
            multiply_slopes<DTYPE == EDEN_F32>(v, z, f.activation);
        }
        if (f.residual) {
            const auto a = load_some<T, 4>(static_cast<const T *>(f.residual) + (size_t)row * f.ld_residual + col, valid);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[0][i] += (float)a.v[i];
        }
        Vec<T, 4> r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.v[i] = (T)v[0][i];
        store_some<T, 4>(static_cast<T *>(f.out) + (size_t)row * f.ld_out + col, r, valid);
    }
}

// The whole end of eight neighbouring columns from `col` on of ROWS rows STEP apart; four lanes side by side have a checkpoint's block.  The rows go
// through it side by side, so that their reads and exponentials overlap, and the activation is chosen once for all of them (once for each value: 301 x 2056
// bf16, 64 deep, 9.1 us in place of 5.9).
// STREAM: the result goes past the caches.  Unless INSIDE, the result has `valid` of the columns (none or less: the lane only takes part in its block's largest value) and `rows` rows.
template <bool INSIDE, int OP, uint32_t DTYPE, int ROWS, int STEP, bool STREAM = false>
__device__ inline void finish_eight(const Finish &f, uint32_t row, uint32_t rows, uint32_t col, int valid, float (&v)[ROWS][8]) {
    auto has = [&](int r) { return INSIDE || (valid > 0 && row + r * STEP < rows); };
    const int n = INSIDE ? 8 : valid;
    if constexpr (OP == kWeightGrad) {
        float *out = static_cast<float *>(f.out) + (size_t)row * f.ld_out + col;
        if (f.accumulate) {
            Vec<float, 8> held[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (has(r)) held[r] = load_some<float, 8>(out + (size_t)(r * STEP) * f.ld_out, n);
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (has(r))
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[r][i] += held[r].v[i];
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            if (has(r)) {
                Vec<float, 8> to;
#pragma unroll
                for (int i = 0; i < 8; ++i) to.v[i] = v[r][i];
                store_some<float, 8>(out + (size_t)(r * STEP) * f.ld_out, to, n);
            }
    } else {
        using T = typename Elem<DTYPE>::type;
        constexpr bool FULL = DTYPE == EDEN_F32;
        const size_t block = (size_t)row * f.blocks + col / kBlock;
        Vec<T, 8> added[ROWS];
        if (f.residual) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (has(r)) added[r] = load_some<T, 8>(static_cast<const T *>(f.residual) + (size_t)(row + r * STEP) * f.ld_residual + col, n);
        }
        if constexpr (OP == kForward) {
            if (f.bias && (INSIDE || valid > 0)) {
                const auto b = load_some<T, 8>(static_cast<const T *>(f.bias) + col, n);
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[r][i] += (float)b.v[i];
            }
            if (f.codes_out) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    float lo[4], hi[4];
                    uint32_t largest = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        lo[i] = i < n ? v[r][i] : 0.0f, hi[i] = 4 + i < n ? v[r][4 + i] : 0.0f;
                        largest = max(largest, max(magnitude_bits(lo[i]), magnitude_bits(hi[i])));
                    }
                    largest = largest_of_quad(largest);
                    const uint32_t t = block_exponent(largest);
                    const size_t at = block + (size_t)(r * STEP) * f.blocks;
                    if (INSIDE || (row + r * STEP < rows && col < f.blocks * kBlock)) {
                        *reinterpret_cast<u32x2 *>(f.codes_out + at * kBlock + col % kBlock) = u32x2{codes4(lo, t), codes4(hi, t)};
                        if (col % kBlock == 0) f.exps_out[at] = (uint8_t)t;
                    }
                }
            }
            activate_all<FULL>(v, f.activation);
        } else if (f.codes_in) {
            float z[ROWS][8];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const size_t at = block + (size_t)(r * STEP) * f.blocks;
                const u32x2 c = has(r) ? *reinterpret_cast<const u32x2 *>(f.codes_in + at * kBlock + col % kBlock) : u32x2{0, 0};
                const float unit = block_unit(has(r) ? f.exps_in[at] : (uint8_t)0);
                float lo[4], hi[4];
                values4(c[0], unit, lo);
                values4(c[1], unit, hi);
#pragma unroll
                for (int i = 0; i < 4; ++i) z[r][i] = lo[i], z[r][4 + i] = hi[i];
            }
            multiply_slopes<FULL>(v, z, f.activation);
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            if (has(r)) {
                Vec<T, 8> to;
#pragma unroll
                for (int i = 0; i < 8; ++i) to.v[i] = (T)(f.residual ? v[r][i] + (float)added[r].v[i] : v[r][i]);
                T *place = static_cast<T *>(f.out) + (size_t)(row + r * STEP) * f.ld_out + col;
                if constexpr (STREAM) stream_some<T, 8>(place, to, n);
                else store_some<T, 8>(place, to, n);
            }
    }
}

}  // namespace eden_layers

#endif  // EDEN_LAYERS_DEVICE_H
