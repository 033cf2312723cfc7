// SplitMix64 (Steele, Lea, Flood: Fast splittable pseudorandom number generators, 2014): its finishing function and increment, for
// counter-based numbers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sr {

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ULL;

__device__ __forceinline__ uint64_t smx_finalize(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ULL;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBULL;
    return z ^ (z >> 31);
}

// The key of stream number `which` of a seed
__device__ __forceinline__ uint64_t smx_key(uint64_t seed, uint64_t which) {
    return smx_finalize(smx_finalize(seed + kGolden) ^ (which * 0xD1342543DE82EF95ULL + 1ULL));
}

}  // namespace sr
