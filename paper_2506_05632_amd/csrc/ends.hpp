// What the kernels at the vocabulary's two ends (scores.hip, embed.hip, clip.hip) share.
#pragma once

#include <cmath>

#include "common.hpp"

namespace llc {

constexpr long long kMaxIndex = 2147483643LL;  // 2^31 - 5: the largest V, N, D, T

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// Rounded to the nearest, ties to even; a NaN stays one.
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float v) {
  const uint32_t b = __float_as_uint(v);
  if (!(v == v)) return (uint16_t)((b >> 16) | 0x40u);
  return (uint16_t)((b + 0x7FFFu + ((b >> 16) & 1u)) >> 16);
}

inline bool known_type(int dtype) { return dtype == LLC_F32 || dtype == LLC_BF16; }
inline size_t type_size(int dtype) { return dtype == LLC_F32 ? 4 : 2; }
inline bool fits(const void *p, size_t bytes) { return ((uintptr_t)p % bytes) == 0; }

// Records the caller's events around what `launch` enqueues.
template <typename F> int between_events(void *begin, void *end, hipStream_t st, F launch) {
  if (begin != nullptr && hipEventRecord((hipEvent_t)begin, st) != hipSuccess) return LLC_E_LAUNCH;
  if (launch() != hipSuccess) return LLC_E_LAUNCH;
  if (end != nullptr && hipEventRecord((hipEvent_t)end, st) != hipSuccess) return LLC_E_LAUNCH;
  return LLC_OK;
}

}  // namespace llc
