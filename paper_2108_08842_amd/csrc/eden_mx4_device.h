// Device-side building blocks of the 4-bit operands: codes, exponents, layout.
#ifndef EDEN_MX4_DEVICE_H
#define EDEN_MX4_DEVICE_H

#include "eden_blocks_device.h"
#include "eden_mx4.h"

namespace eden_layers {

typedef __attribute__((ext_vector_type(8))) int i32x8;

constexpr uint32_t kChunk = 256;                                   // columns of a row's 128 bytes of codes and 8 exponents
constexpr uint32_t kChunkBytes = kChunk / 2, kChunkBlocks = kChunk / kBlock;

__host__ __device__ inline uint32_t chunks_of(uint64_t cols) { return (uint32_t)((cols + kChunk - 1) / kChunk); }
__host__ __device__ inline uint64_t even(uint64_t rows) { return rows + (rows & 1); }
__host__ __device__ inline size_t mx4_codes_bytes(uint64_t rows, uint64_t cols) { return rows * chunks_of(cols) * kChunkBytes; }
__host__ __device__ inline size_t mx4_bytes(uint64_t rows, uint64_t cols) { return mx4_codes_bytes(rows, cols) + chunks_of(cols) * even(rows) * kChunkBlocks; }
// Bytes from the first exponent to those of a row's chunk
__host__ __device__ inline size_t exps_at(uint64_t rows, uint64_t row, uint32_t chunk) { return (chunk * even(rows) + row) * kChunkBlocks; }

// Exponent byte from the bits of the largest |x|: x = f 2^(e - 127), 1 <= f < 2, is at most 6 2^(t - 127) = 1.5 2^(t + 2 - 127) from t = e - 2 on if f <= 1.5, else from e - 1 on
// (subnormal numbers: t = 0).
__device__ inline uint32_t mx4_exponent(uint32_t largest_bits) {
    const int e = (int)((largest_bits + 0x3FFFFFu) >> 23);        // e + 1 if f > 1.5
    return largest_bits >= 0x7F800000u ? 255u : (uint32_t)max(e - 2, 0);
}
// 2^(127 - t), exact.  Of a block that is not finite 0: its codes are 0 whatever the values are (the caller clears NaN).
__device__ inline float mx4_inverse(uint32_t t) { return t == 255u ? 0.0f : __uint_as_float((254u - t) << 23); }
// 2^(t - 127); NaN for 255
__device__ inline float mx4_unit(uint32_t t) { return t == 0u ? __uint_as_float(0x00400000u) : t == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(t << 23); }

// Eight values' codes, to the nearest: the conversion instruction rounds ties to the even code.
__device__ inline uint32_t mx4_codes(const float (&x)[8], uint32_t t) {
    const float inverse = mx4_inverse(t);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0] * inverse, x[1] * inverse, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * inverse, x[3] * inverse, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4] * inverse, x[5] * inverse, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6] * inverse, x[7] * inverse, 1.0f, 3);
    return t == 255u ? 0u : w;
}
// factor times a half of w more than v
template <bool UPPER> __device__ inline uint32_t add_half_times(uint32_t w, uint32_t factor, uint32_t v) {
    uint32_t r;
    if constexpr (UPPER) asm("v_mad_u32_u16 %0, %1, %2, %3 op_sel:[1,0,0,0]" : "=v"(r) : "v"(w), "s"(factor), "v"(v));
    else asm("v_mad_u32_u16 %0, %1, %2, %3" : "=v"(r) : "v"(w), "s"(factor), "v"(v));
    return r;
}
// The largest whole number up to -v
__device__ inline uint32_t floor_of_negative(float v) {
    uint32_t r;
    asm("v_cvt_flr_i32_f32_e64 %0, -%1" : "=v"(r) : "v"(v));
    return r;
}
// Eight values' codes, stochastically.  v = |x| 2^(127 - t) lies between codes 2 e + floor(f) and the next, f = v 2^(1 - e), e = max(exponent of v, 0).  Its share is
// f - floor(f), and d + 1/2 < 65536 share iff ceil(2^28 f) + 4096 (65535 - d) + 2047 reaches the next multiple of 2^28: whole numbers, so nothing is rounded on the way.  With e at 2^29
// the code is bits 28 to 30 of one sum T; what is added up is -T - 1, whose bits are the inverted ones: -ceil is one instruction, and 156 - (e + 127), the distance that v is moved by, adds -e at 2^29 and
// otherwise nothing below bit 31, where x's sign goes.  The four topmost bits move into the word from below, the last value's first.
__device__ inline uint32_t mx4_codes(const float (&x)[8], uint32_t t, const Bits8 &bits) {
    const float inverse = mx4_inverse(t);
    uint32_t w = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
        const float v = fabsf(x[i]) * inverse;
        const uint32_t by = 156u - (__float_as_uint(fmaxf(v, 1.0f)) >> 23);
        const uint32_t sum = (by << 29) + floor_of_negative(__builtin_amdgcn_ldexpf(v, (int)by)), d = bits.pair[i >> 1];
        const uint32_t all = (i & 1 ? add_half_times<true>(d, 4096u, sum) : add_half_times<false>(d, 4096u, sum)) + (2048u - (3u << 28));
        w = __builtin_amdgcn_alignbit(w, (all & 0x7FFFFFFFu) | (__float_as_uint(x[i]) & 0x80000000u), 28);
    }
    return t == 255u ? 0u : w ^ 0x77777777u;
}
__device__ inline void mx4_values(uint32_t codes, float unit, float (&x)[8]) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3);
    x[0] = a[0] * unit, x[1] = a[1] * unit, x[2] = b[0] * unit, x[3] = b[1] * unit;
    x[4] = c[0] * unit, x[5] = c[1] * unit, x[6] = d[0] * unit, x[7] = d[1] * unit;
}

}  // namespace eden_layers

#endif  // EDEN_MX4_DEVICE_H
