// SplitMix64 (Steele, Lea, Flood 2014): output number c + 1 of the generator seeded with `seed` is a function of the counter c alone,
// because the state after i steps is seed + i*gamma.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kavg {

constexpr uint64_t SPLITMIX_GAMMA = 0x9E3779B97F4A7C15ull;

__device__ __forceinline__ uint64_t splitmix64_mix(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

}  // namespace kavg
