// SplitMix64 (Steele, Lea & Flood, OOPSLA 2014) as a keyed hash: its output function,
// and keys folded from components.
#pragma once

#include <cstdint>

#ifdef __HIPCC__
#include <hip/hip_runtime.h>
#define RIP_HOST_DEVICE __host__ __device__
#else
#define RIP_HOST_DEVICE
#endif

namespace rip {

constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ULL;

RIP_HOST_DEVICE inline uint64_t mix(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ULL;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBULL;
  return z ^ (z >> 31);
}

RIP_HOST_DEVICE inline uint64_t fold(uint64_t k, uint64_t c) { return mix(k + kGamma * (c + 1)); }

}  // namespace rip
