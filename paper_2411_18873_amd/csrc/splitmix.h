// The counter-based generator of the library: output number j of a SplitMix64 stream is the finaliser of (state + j * kGamma),
// so any thread draws any word by itself.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace eck {

constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;

__host__ __device__ __forceinline__ uint64_t splitmix_finalise(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// state that stream (seed, round) starts from
inline uint64_t stream_state(uint64_t seed, uint32_t round) { return splitmix_finalise(seed + kGamma * ((uint64_t)round + 1)); }

} // namespace eck
