// Element-wise kernels of the layer operators: 8-bit checkpoint from and to values, the gradient through an activation.
//
// Bound by memory: each value is read and written once.  A thread has eight neighbouring columns (16 bytes of a two-byte type),
// four threads have a checkpoint's block and find its largest value by two lane exchanges.  A workgroup has 2^s threads for each of its 256 / 2^s
// rows, s so that a short row leaves few of them idle.
//
// 8192 x 8192 bf16: save 38 us = 5.3 TB/s, restore 37 us = 5.4 TB/s.  Gradient through gelu_tanh, 8192 x 16384 bf16: 143 us = 4.7 TB/s, with vector instructions in
// 84% of the cycles.  17 x 1000: 2.6 us a launch, whatever it does.
#include "eden_layers_kernels.h"

#include <algorithm>

namespace eden_layers {
namespace {

constexpr uint32_t kThreads = 256;

// threads of a row (a power of two, 4 at least: a block's) and workgroups along it
struct Spread {
    uint32_t shift, segments;
    uint64_t groups;
};
Spread spread(uint32_t rows, uint32_t cols) {
    const uint32_t units = (uint32_t)blocks_of(cols) * 4;
    uint32_t shift = 2;
    while (shift < 8 && (1u << shift) < units) ++shift;
    const uint32_t segments = (units + (1u << shift) - 1) >> shift, rows_each = kThreads >> shift;
    return {shift, segments, (uint64_t)((rows + rows_each - 1) / rows_each) * segments};
}
struct Place {
    uint32_t row, col;
};
// `before`: workgroups of the call's launches before this one
__device__ inline Place place(uint32_t shift, uint32_t segments, uint32_t before) {
    const uint32_t number = before + blockIdx.x, group = number / segments, segment = number - group * segments;
    return {group * (kThreads >> shift) + (threadIdx.x >> shift), ((segment << shift) + (threadIdx.x & ((1u << shift) - 1))) * 8};
}
__device__ inline int valid_of(uint32_t col, uint32_t cols) { return col < cols ? (int)min(8u, cols - col) : 0; }

template <uint32_t DTYPE>
__global__ __launch_bounds__(kThreads) void k_save(const typename Elem<DTYPE>::type *x, size_t ldx, uint32_t rows, uint32_t cols, uint32_t blocks,
                                                   uint8_t *codes, uint8_t *exps, uint32_t shift, uint32_t segments, uint32_t before) {
    using T = typename Elem<DTYPE>::type;
    const Place at = place(shift, segments, before);
    if (at.row >= rows || at.col >= blocks * kBlock) return;       // four threads of a block leave or stay together
    const auto v = load_some<T, 8>(x + (size_t)at.row * ldx + at.col, valid_of(at.col, cols));
    float lo[4], hi[4];
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo[i] = (float)v.v[i];
        hi[i] = (float)v.v[4 + i];
        largest = max(largest, max(magnitude_bits(lo[i]), magnitude_bits(hi[i])));
    }
    largest = largest_of_quad(largest);
    const uint32_t t = block_exponent(largest);
    const size_t block = (size_t)at.row * blocks + at.col / kBlock;
    *reinterpret_cast<u32x2 *>(codes + block * kBlock + at.col % kBlock) = u32x2{codes4(lo, t), codes4(hi, t)};
    if (at.col % kBlock == 0) exps[block] = (uint8_t)t;
}

__device__ inline void read_values(const uint8_t *codes, const uint8_t *exps, uint32_t blocks, Place at, float (&lo)[4], float (&hi)[4]) {
    const size_t block = (size_t)at.row * blocks + at.col / kBlock;
    const u32x2 c = *reinterpret_cast<const u32x2 *>(codes + block * kBlock + at.col % kBlock);
    const float unit = block_unit(exps[block]);
    values4(c[0], unit, lo);
    values4(c[1], unit, hi);
}

template <uint32_t DTYPE>
__global__ __launch_bounds__(kThreads) void k_restore(const uint8_t *codes, const uint8_t *exps, uint32_t rows, uint32_t cols, uint32_t blocks,
                                                      typename Elem<DTYPE>::type *x, size_t ldx, uint32_t shift, uint32_t segments, uint32_t before) {
    using T = typename Elem<DTYPE>::type;
    const Place at = place(shift, segments, before);
    if (at.row >= rows || at.col >= cols) return;
    float lo[4], hi[4];
    read_values(codes, exps, blocks, at, lo, hi);
    Vec<T, 8> v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v.v[i] = (T)lo[i];
        v.v[4 + i] = (T)hi[i];
    }
    store_some<T, 8>(x + (size_t)at.row * ldx + at.col, v, valid_of(at.col, cols));
}

template <uint32_t DTYPE>
__global__ __launch_bounds__(kThreads) void k_activation_grad(const typename Elem<DTYPE>::type *dy, size_t ldy, const uint8_t *codes, const uint8_t *exps,
                                                              uint32_t activation, typename Elem<DTYPE>::type *dz, size_t ldz, uint32_t rows,
                                                              uint32_t cols, uint32_t blocks, uint32_t shift, uint32_t segments, uint32_t before) {
    using T = typename Elem<DTYPE>::type;
    constexpr bool FULL = DTYPE == EDEN_F32;
    const Place at = place(shift, segments, before);
    if (at.row >= rows || at.col >= cols) return;
    const int valid = valid_of(at.col, cols);
    auto v = load_some<T, 8>(dy + (size_t)at.row * ldy + at.col, valid);
    float lo[4], hi[4];
    read_values(codes, exps, blocks, at, lo, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v.v[i] = (T)((float)v.v[i] * slope<FULL>(lo[i], activation));
        v.v[4 + i] = (T)((float)v.v[4 + i] * slope<FULL>(hi[i], activation));
    }
    store_some<T, 8>(dz + (size_t)at.row * ldz + at.col, v, valid);
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_copy_rows(const T *from, size_t ld, uint32_t rows, uint32_t cols, T *to, uint32_t to_ld, uint32_t shift, uint32_t segments, uint32_t before) {
    const Place at = place(shift, segments, before);
    if (at.row >= rows || at.col >= to_ld) return;
    Vec<T, 8> v;
    const int valid = valid_of(at.col, cols);
    const T *p = from + (size_t)at.row * ld + at.col;
    if (valid == 8) {
        __builtin_memcpy(&v, p, sizeof(v));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.v[i] = i < valid ? p[i] : (T)0;
    }
    __builtin_memcpy(__builtin_assume_aligned(to + (size_t)at.row * to_ld + at.col, 16), &v, sizeof(v));
}

template <class F> void for_type(uint32_t dtype, F f) {
    if (dtype == EDEN_F32) f(std::integral_constant<uint32_t, EDEN_F32>());
    else if (dtype == EDEN_F16) f(std::integral_constant<uint32_t, EDEN_F16>());
    else f(std::integral_constant<uint32_t, EDEN_BF16>());
}
// f(workgroups before a launch, workgroups of it) until all are launched
template <class F> hipError_t launches(const Spread &s, F f) {
    hipError_t e = hipSuccess;
    for (uint64_t before = 0; before < s.groups && e == hipSuccess; before += most_groups(kThreads)) {
        f((uint32_t)before, (uint32_t)std::min(s.groups - before, most_groups(kThreads)));
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

hipError_t launch_save(uint32_t dtype, const void *x, size_t ldx, uint32_t rows, uint32_t cols, uint8_t *codes, uint8_t *exps, hipStream_t st) {
    const Spread s = spread(rows, cols);
    return launches(s, [&](uint32_t before, uint32_t groups) {
        for_type(dtype, [&](auto t) {
            using T = typename Elem<decltype(t)::value>::type;
            k_save<decltype(t)::value><<<groups, kThreads, 0, st>>>(static_cast<const T *>(x), ldx, rows, cols, (uint32_t)blocks_of(cols), codes, exps, s.shift, s.segments, before);
        });
    });
}

hipError_t launch_copy_rows(uint32_t dtype, const void *from, size_t ld, uint32_t rows, uint32_t cols, void *to, uint32_t to_ld, hipStream_t st) {
    const Spread s = spread(rows, to_ld);
    return launches(s, [&](uint32_t before, uint32_t groups) {
        auto copy = [&](auto element) {
            using T = decltype(element);
            k_copy_rows<<<groups, kThreads, 0, st>>>(static_cast<const T *>(from), ld, rows, cols, static_cast<T *>(to), to_ld, s.shift, s.segments, before);
        };
        if (dtype == EDEN_F32) copy(uint32_t());
        else copy(uint16_t());
    });
}

hipError_t launch_restore(uint32_t dtype, const uint8_t *codes, const uint8_t *exps, uint32_t rows, uint32_t cols, void *x, size_t ldx, hipStream_t st) {
    const Spread s = spread(rows, cols);
    return launches(s, [&](uint32_t before, uint32_t groups) {
        for_type(dtype, [&](auto t) {
            using T = typename Elem<decltype(t)::value>::type;
            k_restore<decltype(t)::value><<<groups, kThreads, 0, st>>>(codes, exps, rows, cols, (uint32_t)blocks_of(cols), static_cast<T *>(x), ldx, s.shift, s.segments, before);
        });
    });
}

hipError_t launch_activation_grad(uint32_t dtype, const void *dy, size_t ldy, const uint8_t *codes, const uint8_t *exps, uint32_t activation,
                                  void *dz, size_t ldz, uint32_t rows, uint32_t cols, hipStream_t st) {
    const Spread s = spread(rows, cols);
    return launches(s, [&](uint32_t before, uint32_t groups) {
        for_type(dtype, [&](auto t) {
            using T = typename Elem<decltype(t)::value>::type;
            k_activation_grad<decltype(t)::value><<<groups, kThreads, 0, st>>>(static_cast<const T *>(dy), ldy, codes, exps, activation, static_cast<T *>(dz), ldz, rows, cols,
                                                                              (uint32_t)blocks_of(cols), s.shift, s.segments, before);
        });
    });
}

}  // namespace eden_layers
