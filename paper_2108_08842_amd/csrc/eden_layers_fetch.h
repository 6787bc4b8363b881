// Loads from memory straight into the LDS, and what goes with them.
#ifndef EDEN_LAYERS_FETCH_H
#define EDEN_LAYERS_FETCH_H

#include "eden_layers_product.h"

#include <utility>

namespace eden_layers {

constexpr uint32_t kMostBytes = 0x7FFFFF00u;       // reach of a descriptor; offsets from kNowhere on lie beyond it (and below 2^32)
constexpr uint32_t kNowhere = 0x7FFFFFF0u;

using rsrc_t = __amdgpu_buffer_rsrc_t;
typedef __attribute__((address_space(3))) char lds_char;

// A barrier behind which every wave finds what all waves' loads, but for a wave's last LATER, have written into the LDS, and behind which no wave has LDS
// reads or writes on their way.  (__syncthreads() would wait for all loads, or for none.)
template <int LATER> __device__ inline void meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LATER) : "memory");
}

template <int... I, class F> __device__ inline void each_of(std::integer_sequence<int, I...>, F f) { (f(std::integral_constant<int, I>()), ...); }
// `count` things to do among `of` products, evenly: the one that comes behind product j, or -1
constexpr int due(int j, int count, int of) {
    for (int i = 0; i < count; ++i)
        if ((2 * i + 1) * of / (2 * count) == j) return i;
    return -1;
}
template <int N, class F> __device__ inline void each(F f) { each_of(std::make_integer_sequence<int, N>(), f); }

// A descriptor in scalar registers
__device__ inline u32x4 descriptor(const char *base, uint64_t reach) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    const uint32_t bytes = reach < kMostBytes ? (uint32_t)reach : kMostBytes;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32) & 0xFFFF),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}

// 16 bytes a lane from `offset` of a descriptor's buffer (zeros beyond its end) to the wave's kilobyte of the LDS at `to`.  Written out: the compiler would have
// every LDS read wait for the loads into any other part of the LDS.  It has no result in registers; meet() waits for it.
__device__ inline void load_to_lds(uint32_t to, uint32_t offset, u32x4 buffer) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"((uint32_t)__builtin_amdgcn_readfirstlane((int)to)), "v"(offset), "s"(buffer)
                 : "memory", "m0");
}

}  // namespace eden_layers

#endif  // EDEN_LAYERS_FETCH_H
