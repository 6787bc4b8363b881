// The counter hash that all random numbers come from.
#ifndef EDEN_HASH_H
#define EDEN_HASH_H

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace eden {

// ---- shared randomness (Sec. 2.1): counter hash = splitmix64 stream started at a per-(seed,stream,client) key
constexpr uint64_t kPhi = 0x9E3779B97F4A7C15ull;
enum : uint32_t { kStreamSign = 0, kStreamSubsample = 1, kStreamLoss = 2, kStreamMix = 3, kStreamSparse = 4,
                  kStreamDropout = 5, kStreamRounding = 6 };   // of the block operators and of rounding to 4 bits

__host__ __device__ inline uint64_t mix64(uint64_t z) {
    z ^= z >> 30; z *= 0xBF58476D1CE4E5B9ull;
    z ^= z >> 27; z *= 0x94D049BB133111EBull;
    z ^= z >> 31;
    return z;
}
__host__ __device__ inline uint64_t stream_key(uint64_t seed, uint32_t stream, uint32_t client) {
    const uint64_t tag = ((uint64_t)stream << 32) | (uint64_t)client;
    return mix64(mix64(seed + kPhi) + kPhi * tag + kPhi);
}
__host__ __device__ inline uint64_t hash_word(uint64_t key, uint64_t j) { return mix64(key + kPhi * (j + 1)); }

}  // namespace eden

#endif  // EDEN_HASH_H
