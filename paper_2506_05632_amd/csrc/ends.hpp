// What the kernels at the vocabulary's two ends (scores.hip, embed.hip, clip.hip) share.
#pragma once

#include <cmath>

#include "common.hpp"

namespace llc {

constexpr long long kMaxIndex = 2147483643LL;  // 2^31 - 5: the largest V, N, D, T

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// Rounded to the nearest, ties to even, by the hardware's conversion of a pair; a NaN stays one.
typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
typedef float float_pair __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t narrow_pair(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(float_pair{a, b}, bf16_pair));
}
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float v) { return (uint16_t)narrow_pair(v, 0.0f); }

// N consecutive entries (4 or 8) wherever they start, at full width: the alignment stated is the entry's own.
typedef uint32_t word2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t word4_any __attribute__((ext_vector_type(4), aligned(2)));
template <int N> __device__ __forceinline__ void load_some(const float *p, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4_any t = *reinterpret_cast<const float4_any *>(p + i);
    v[i] = t.x; v[i + 1] = t.y; v[i + 2] = t.z; v[i + 3] = t.w;
  }
}
__device__ __forceinline__ void split_pair(uint32_t w, float &a, float &b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xFFFF0000u);
}
template <int N> __device__ __forceinline__ void load_some(const uint16_t *p, float (&v)[N]) {
  static_assert(N == 4 || N == 8, "a load of 8 or 16 bytes");
  if constexpr (N == 4) {
    const word2_any t = *reinterpret_cast<const word2_any *>(p);
    split_pair(t.x, v[0], v[1]); split_pair(t.y, v[2], v[3]);
  } else {
    const word4_any t = *reinterpret_cast<const word4_any *>(p);
    split_pair(t.x, v[0], v[1]); split_pair(t.y, v[2], v[3]); split_pair(t.z, v[4], v[5]); split_pair(t.w, v[6], v[7]);
  }
}
template <int N> __device__ __forceinline__ void store_some(float *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<float4_any *>(p + i) = float4_any{v[i], v[i + 1], v[i + 2], v[i + 3]};
}
template <int N> __device__ __forceinline__ void store_some(uint16_t *p, const float (&v)[N]) {
  if constexpr (N == 4)
    *reinterpret_cast<word2_any *>(p) = word2_any{narrow_pair(v[0], v[1]), narrow_pair(v[2], v[3])};
  else
    *reinterpret_cast<word4_any *>(p) = word4_any{narrow_pair(v[0], v[1]), narrow_pair(v[2], v[3]), narrow_pair(v[4], v[5]), narrow_pair(v[6], v[7])};
}
// What is written here and not read again soon goes past the caches, which then keep what is read.  (The embedding's gradient, 128 256 x
// 4096 bf16 of 16 384 tokens: 277 us with stores that the caches keep, 215 so; a call that writes zeros alone 196, 160.)
template <int N> __device__ __forceinline__ void stream_some(float *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4)
    __builtin_nontemporal_store(float4_any{v[i], v[i + 1], v[i + 2], v[i + 3]}, reinterpret_cast<float4_any *>(p + i));
}
template <int N> __device__ __forceinline__ void stream_some(uint16_t *p, const float (&v)[N]) {
  if constexpr (N == 4)
    __builtin_nontemporal_store(word2_any{narrow_pair(v[0], v[1]), narrow_pair(v[2], v[3])}, reinterpret_cast<word2_any *>(p));
  else
    __builtin_nontemporal_store(word4_any{narrow_pair(v[0], v[1]), narrow_pair(v[2], v[3]), narrow_pair(v[4], v[5]), narrow_pair(v[6], v[7])},
                                reinterpret_cast<word4_any *>(p));
}
// The same where only the first `n` of them belong to the caller.
template <int N, typename E> __device__ __forceinline__ void load_first(const E *p, long long n, float (&v)[N]) {
  if (n >= N) { load_some<N>(p, v); return; }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i < n ? widen(p[i]) : 0.0f;
}
template <int N, typename E> __device__ __forceinline__ void store_first(E *p, long long n, const float (&v)[N]) {
  if (n >= N) { store_some<N>(p, v); return; }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < n) p[i] = narrow<E>(v[i]);
}
template <int N, typename E> __device__ __forceinline__ void stream_first(E *p, long long n, const float (&v)[N]) {
  if (n >= N) { stream_some<N>(p, v); return; }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < n) p[i] = narrow<E>(v[i]);
}
template <typename E> constexpr int kWide = 16 / sizeof(E);  // entries of 16 bytes

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
