// Products of a few rows with a layer held in 4 bits: out[r,n] = sum over groups g of scale[n,g] * sum over d in g of (q[n,d] - zero[n,g]) x[r,d].
//
// The codes are read once and bound the call (a layer of 128 256 x 4096 is 263 MB; 8 rows in bf16 take 61 us); matrix instructions take the products, 16 columns of the output by 16
// rows of x at a time, so that a row of x costs nothing until there are sixteen.
//
// A code becomes a bf16 number by two integer operations for a pair: its four bits are the upper mantissa bits of a number between 16 and
// 31, so that the product's operand is 16 + q, exactly.  What that adds, and the zero, are taken off beforehand: a group's sum starts at
// -(16 + zero) times the sum of x over the group.  Products of bf16 numbers are exact in fp32; the sum of a group of standard normal x
// stays below some 300, so its roundings are 2^-16 at most and 6e-7 of a result, as large as those of the sum over the groups.
// x of 32 bits is split into three bf16 parts that hold all its bits; the second and third have a sum of their own.
#pragma once

#include "quantized.hpp"

namespace llc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight codes as 16 + q: the pairs (0,4), (1,5), (2,6), (3,7).  x lies in LDS in the same order.
__device__ __forceinline__ bf16x8 widen_codes(uint32_t w) {
  constexpr uint32_t kMask = 0x00780078u, kSixteen = 0x41804180u;
  const u32x4 v = {((w << 3) & kMask) | kSixteen, ((w >> 1) & kMask) | kSixteen, ((w >> 5) & kMask) | kSixteen, ((w >> 9) & kMask) | kSixteen};
  return __builtin_bit_cast(bf16x8, v);
}

// The sum over the lanes of a group's pieces (4, 8 or 16 neighbours), in each of them.
template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int LANES> __device__ __forceinline__ float sum_lanes(float v) {
  v = dpp_add<0xB1>(v);                               // quad_perm 1 0 3 2
  v = dpp_add<0x4E>(v);                               // quad_perm 2 3 0 1
  if constexpr (LANES >= 8) v = dpp_add<0x141>(v);    // row_half_mirror
  if constexpr (LANES >= 16) v = dpp_add<0x140>(v);   // row_mirror
  return v;
}

// A lane's part of a slab: row `lane & 15` of the tile, 32 of the 128 columns, as words of eight codes that the steps of the product take in
// turn.  The four quarters of a wavefront hold the same group's columns in every step.
template <int G, typename S> struct Slab {
  static constexpr int kGroups = 128 / G;
  uint32_t words[4];
  float scale[kGroups];
  float shift[kGroups];  // -(16 + zero)
};
// The same with its scales and zeros as they lie in memory, until they are needed.
template <int G, typename S> struct RawSlab {
  static constexpr int kGroups = 128 / G, kScaleWords = (kGroups * sizeof(S) + 3) / 4;
  uint32_t words[4];
  uint32_t scale[kScaleWords];
  uint32_t zero;
};
// Four slabs that follow each other, their scales and zeros as they lie in memory.
template <int G, typename S> struct Batch {
  static constexpr int kSlabs = 4, kGroups = kSlabs * 128 / G, kScaleWords = kGroups * sizeof(S) / 4, kZeroWords = kGroups / 4;
  uint32_t words[kSlabs][4];
  uint32_t scale[kScaleWords];
  uint32_t zero[kZeroWords];
};

// A quarter has 16 bytes of a row, one after the other.  Groups of 128 take them as they lie; with smaller groups a step's words are those of one quarter's 16 bytes, so that the step
// is within a group: four words of four quarters, turned.  (A load for each word instead, 128 256 x 4096 in groups of 32, 8 rows: 155 us.)
template <int G> __device__ __forceinline__ void turn_words(uint32_t (&w)[4]) {
  if constexpr (G < 128) {
    // (what the upper half of one has goes where the lower half of the other is, and the other way round; then by rows of 16 lanes)
    const auto halves = [](uint32_t &a, uint32_t &b) {
      const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
      a = r[0]; b = r[1];
    };
    const auto rows = [](uint32_t &a, uint32_t &b) {
      const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
      a = r[0]; b = r[1];
    };
    halves(w[0], w[2]);
    halves(w[1], w[3]);
    rows(w[0], w[1]);
    rows(w[2], w[3]);
  }
}

// N words from anywhere.
template <int N> __device__ __forceinline__ void load_words(uint32_t (&w)[N], const void *from) {
  const uint8_t *at = reinterpret_cast<const uint8_t *>(from);
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const word1_byte *>(at);
  } else if constexpr (N == 2) {
    const word2_byte v = *reinterpret_cast<const word2_byte *>(at);
    w[0] = v.x; w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const word4_byte v = *reinterpret_cast<const word4_byte *>(at + 4 * i);
      w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
  }
}
template <typename S, int WORDS> __device__ __forceinline__ float scale_of(const uint32_t (&words)[WORDS], int at) {
  if constexpr (sizeof(S) == 4) return __uint_as_float(words[at]);
  return __uint_as_float(at % 2 == 0 ? words[at / 2] << 16 : words[at / 2] & 0xFFFF0000u);
}
template <bool Z, int G, typename S> __device__ __forceinline__ Slab<G, S> slab_of(const RawSlab<G, S> &r) {
  Slab<G, S> s;
#pragma unroll
  for (int j = 0; j < 4; ++j) s.words[j] = r.words[j];
  turn_words<G>(s.words);
#pragma unroll
  for (int g = 0; g < 128 / G; ++g) {
    s.scale[g] = scale_of<S>(r.scale, g);
    s.shift[g] = Z ? -16.0f - (float)((r.zero >> (8 * g)) & 255u) : -24.0f;
  }
  return s;
}
template <bool Z, int G, typename S>
__device__ __forceinline__ RawSlab<G, S> load_slab(const uint8_t *codes, const S *scales, const uint8_t *zeros, int slab, int quarter) {
  constexpr int kGroups = 128 / G;
  RawSlab<G, S> s;
  load_words(s.words, codes + (long long)slab * 64 + 16 * quarter);
  const S *scale = scales + (long long)slab * kGroups;
  if constexpr (kGroups * sizeof(S) == 2) s.scale[0] = *scale;
  else load_words(s.scale, scale);
  if constexpr (Z) {
    const uint8_t *zero = zeros + (long long)slab * kGroups;
    if constexpr (kGroups == 4) s.zero = *reinterpret_cast<const word1_byte *>(zero);
    else if constexpr (kGroups == 2) s.zero = *reinterpret_cast<const half_byte *>(zero);
    else s.zero = *zero;
  }
  return s;
}
// The last slab of a row that is not a whole one: nothing behind the row's end is read, and what is multiplied there is no matter, since x is 0.
template <bool Z, int G, typename S>
__device__ __forceinline__ RawSlab<G, S> load_last_slab(const MatvecParams &p, const uint8_t *codes, const S *scales, const uint8_t *zeros, int slab, int quarter) {
  RawSlab<G, S> s;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long at = (long long)slab * 64 + 16 * quarter + 4 * i, last = (p.D + 1) / 2 - 4;
    if (last < 0) {  // (uniform: a row of up to six entries)
      s.words[i] = load_codes(codes, 2 * at, p.D);
    } else {  // (under no condition, so that the four are under way together)
      const uint32_t word = *reinterpret_cast<const word1_byte *>(codes + (at < last ? at : last));
      s.words[i] = at <= last ? word : at - last < 4 ? word >> (8 * (int)(at - last)) : 0;
    }
  }
#pragma unroll
  for (int i = 0; i < RawSlab<G, S>::kScaleWords; ++i) s.scale[i] = 0;
  s.zero = 0;
#pragma unroll
  for (int g = 0; g < 128 / G; ++g) {
    int of = slab * (128 / G) + g;
    of = of < p.groups ? of : p.groups - 1;  // (columns behind the row's end: x is 0 there)
    if constexpr (sizeof(S) == 4) s.scale[g] = __float_as_uint(scales[of]);
    else s.scale[g / 2] |= (uint32_t)scales[of] << (16 * (g % 2));
    if constexpr (Z) s.zero |= (uint32_t)zeros[of] << (8 * g);
  }
  return s;
}
template <bool Z, int G, typename S> __device__ __forceinline__ void load_batch(Batch<G, S> &b, const uint8_t *codes, const S *scales, const uint8_t *zeros, int slab, int quarter) {
#pragma unroll
  for (int i = 0; i < Batch<G, S>::kSlabs; ++i) load_words(b.words[i], codes + (long long)(slab + i) * 64 + 16 * quarter);
  load_words(b.scale, scales + (long long)slab * (128 / G));
  if constexpr (Z) load_words(b.zero, zeros + (long long)slab * (128 / G));
}
template <bool Z, int G, typename S> __device__ __forceinline__ Slab<G, S> slab_of(const Batch<G, S> &b, int i) {
  Slab<G, S> s;
#pragma unroll
  for (int j = 0; j < 4; ++j) s.words[j] = b.words[i][j];
  turn_words<G>(s.words);
#pragma unroll
  for (int g = 0; g < 128 / G; ++g) {
    const int at = i * (128 / G) + g;
    s.scale[g] = scale_of<S>(b.scale, at);
    s.shift[g] = Z ? -16.0f - (float)((b.zero[at / 4] >> (8 * (at % 4))) & 255u) : -24.0f;
  }
  return s;
}

// Adds a slab's products to the sums of WIDE tiles of columns, which share what is read of x.  s_x, s_sum: the slab's, and its groups' sums.
template <int TILES, int PARTS, int G, typename S, int WIDE>
__device__ __forceinline__ void add_slab(f32x4 (&total)[WIDE][TILES], const Slab<G, S> (&s)[WIDE], const uint4 *s_x, const float *s_sum, const int (&at_x)[TILES],
                                         int pitch, int quarter) {
  int from = 0;
  constexpr int kSteps = G / 32;  // of a group
  f32x4 sum[WIDE][TILES], low[WIDE][TILES];
#pragma unroll
  for (int step = 0; step < 4; ++step) {
    const int g = step / kSteps;
    if (step % kSteps == 0) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const f32x4 sx = *reinterpret_cast<const f32x4 *>(s_sum + g * (TILES * 16) + 16 * t + 4 * quarter);
#pragma unroll
        for (int w = 0; w < WIDE; ++w) {
#pragma unroll
          for (int j = 0; j < 4; ++j) sum[w][t][j] = s[w].shift[g] * sx[j];
          low[w][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
      }
    }
    bf16x8 codes[WIDE];
#pragma unroll
    for (int w = 0; w < WIDE; ++w) codes[w] = widen_codes(s[w].words[step]);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      asm volatile("" : "+s"(from));  // (an addition a read: all the places at once, as they follow from the slab's, would take more registers than there are)
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const bf16x8 a = __builtin_bit_cast(bf16x8, s_x[from + at_x[t]]);
#pragma unroll
        for (int w = 0; w < WIDE; ++w) {
          if (part == 0) sum[w][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, codes[w], sum[w][t], 0, 0, 0);
          else low[w][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, codes[w], low[w][t], 0, 0, 0);
        }
      }
      from += 4 * pitch;
    }
    if (step % kSteps == kSteps - 1) {
#pragma unroll
      for (int w = 0; w < WIDE; ++w)
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) total[w][t][j] = fmaf(s[w].scale[g], PARTS > 1 ? sum[w][t][j] + low[w][t][j] : sum[w][t][j], total[w][t][j]);
    }
    if (TILES * PARTS > 2 || step == 3) __builtin_amdgcn_sched_barrier(0);  // (what later steps read of x, read ahead, would take more registers than there are)
  }
}

// The same with places of x that are known when this is compiled: what the next products take of x is asked for before these.
template <int TILES, int PARTS, int G, typename S, int WIDE>
__device__ __forceinline__ void add_streamed_slab(f32x4 (&total)[WIDE][TILES], const Slab<G, S> (&s)[WIDE], const uint4 *s_x, const float *s_sum, int lane) {
  constexpr int kOf = G / 32 * PARTS, kAll = 4 * PARTS;  // products of a group, of the slab
  const uint4 *at = s_x + (lane >> 4) * 16 * TILES + (lane & 15);
  const float *at_sum = s_sum + 4 * (lane >> 4);
  f32x4 sum[WIDE][TILES], low[WIDE][TILES], sx[TILES];
  bf16x8 a[2][TILES], codes[WIDE];
  const auto ask = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) a[i & 1][t] = __builtin_bit_cast(bf16x8, at[i * 64 * TILES + 16 * t]);
  };
  const auto ask_sums = [&](int g) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) sx[t] = *reinterpret_cast<const f32x4 *>(at_sum + g * (TILES * 16) + 16 * t);
  };
  ask_sums(0);
  ask(0);
#pragma unroll
  for (int i = 0; i < kAll; ++i) {
    const int g = i / kOf;
    if (i % kOf == 0) {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int w = 0; w < WIDE; ++w) {
#pragma unroll
          for (int j = 0; j < 4; ++j) sum[w][t][j] = s[w].shift[g] * sx[t][j];
          low[w][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
    if (i + 1 < kAll) {
      ask(i + 1);
      if ((i + 1) % kOf == 0) ask_sums(g + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (i % PARTS == 0) {
#pragma unroll
      for (int w = 0; w < WIDE; ++w) codes[w] = widen_codes(s[w].words[i / PARTS]);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int w = 0; w < WIDE; ++w) {
        if (i % PARTS == 0) sum[w][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i & 1][t], codes[w], sum[w][t], 0, 0, 0);
        else low[w][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i & 1][t], codes[w], low[w][t], 0, 0, 0);
      }
    if (i % kOf == kOf - 1) {
#pragma unroll
      for (int w = 0; w < WIDE; ++w)
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) total[w][t][j] = fmaf(s[w].scale[g], PARTS > 1 ? sum[w][t][j] + low[w][t][j] : sum[w][t][j], total[w][t][j]);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// x to LDS as the operands lie: [slab][step][part][quarter][row], 16 bytes each, rows an odd number of them apart so that pieces of one row lie in unlike banks; and the groups' sums [group][16 rows of a tile].  A piece is eight columns of a row.
template <typename X> struct Piece;
template <> struct Piece<float> { float4_any a, b; };
template <> struct Piece<uint16_t> { word4_any a; };
template <typename X> __device__ __forceinline__ Piece<X> load_x(const MatvecParams &p, long long r, int at) {
  const X *row = reinterpret_cast<const X *>(p.x) + r * p.x_stride;
  const int D = (int)p.D;
  Piece<X> v;
  if (at + 8 <= D) {
    v.a = *reinterpret_cast<const decltype(v.a) *>(row + at);
    if constexpr (sizeof(X) == 4) v.b = *reinterpret_cast<const decltype(v.b) *>(row + at + 4);
  } else {  // nothing behind the row's end
    X e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = row[at + j < D ? at + j : D - 1];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = at + j < D ? e[j] : (X)0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(X) == 4) {
        v.a[j] = e[j]; v.b[j] = e[j + 4];
      } else {
        v.a[j] = (uint32_t)e[2 * j] | (uint32_t)e[2 * j + 1] << 16;
      }
    }
  }
  return v;
}
template <int PARTS, int G, typename X>
__device__ __forceinline__ void store_x(const Piece<X> &from, unsigned r, unsigned piece, int pitch, int tiles, uint4 *s_x, float *s_sum) {
  float v[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(X) == 4) {
      v[j] = from.a[j]; v[j + 4] = from.b[j];
    } else {
      split_pair(from.a[j], v[2 * j], v[2 * j + 1]);
    }
  }
  float sum = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  sum = sum_lanes<G / 8>(sum);
  const unsigned slab = piece >> 4, q = piece & 15;
  const unsigned step = G == 128 ? q & 3 : q >> 2, quarter = G == 128 ? q >> 2 : q & 3;
  if ((q & (G / 8 - 1)) == 0) s_sum[(slab * (128 / G) + q / (G / 8)) * (tiles * 16) + r] = sum;
  uint4 *to = s_x + ((slab * 4 + step) * PARTS * 4 + quarter) * pitch + r;
#pragma unroll
  for (int part = 0; part < PARTS; ++part) {
    const uint4 w = make_uint4(narrow_pair(v[0], v[4]), narrow_pair(v[1], v[5]), narrow_pair(v[2], v[6]), narrow_pair(v[3], v[7]));
    to[part * 4 * pitch] = w;
    if (part + 1 < PARTS) {  // what is left is exact
      const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float a, b;
        split_pair(in[j], a, b);
        v[j] -= a;
        v[j + 4] -= b;
      }
    }
  }
}

// The sums of wavefronts that share tiles of columns are joined, and the tiles written.
template <int TILES, int WIDE>
__device__ __forceinline__ void finish_tiles(const MatvecParams &p, f32x4 (&total)[WIDE][TILES], float *s_join, int share, int part_of, int wave, int lane, long long r0, int rows,
                                             const long long (&n0)[WIDE]) {
  const int column = lane & 15, quarter = lane >> 4;
  if (share > 1) {
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WIDE; ++w)
#pragma unroll
      for (int t = 0; t < TILES; ++t) *reinterpret_cast<f32x4 *>(s_join + (((wave * WIDE + w) * TILES + t) * 64 + lane) * 4) = total[w][t];
    __syncthreads();
    if (part_of == 0) {
      for (int other = 1; other < share; ++other)
#pragma unroll
        for (int w = 0; w < WIDE; ++w)
#pragma unroll
          for (int t = 0; t < TILES; ++t) {
            const f32x4 add = *reinterpret_cast<const f32x4 *>(s_join + ((((wave + other) * WIDE + w) * TILES + t) * 64 + lane) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) total[w][t][j] += add[j];
          }
    }
  }
  if (part_of != 0) return;
#pragma unroll
  for (int w = 0; w < WIDE; ++w) {
    const long long n = n0[w] + column;
    if (n0[w] < 0 || n >= p.N) continue;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 16 * t + 4 * quarter + j;
        if (r < rows) {
          const long long to = (r0 + r) * p.out_stride + n;
          if (p.out_type == LLC_F32) reinterpret_cast<float *>(p.out)[to] = total[w][t][j];
          else reinterpret_cast<uint16_t *>(p.out)[to] = narrow<uint16_t>(total[w][t][j]);
        }
      }
  }
}

// A row of the layer.
template <typename S> struct Row {
  const uint8_t *codes;
  const S *scales;
  const uint8_t *zeros;
};
template <typename S> __device__ __forceinline__ Row<S> row_of(const MatvecParams &p, long long n) {
  const long long at = n < p.N ? n : p.N - 1;
  const uint8_t *codes = p.codes + at * p.codes_stride;
  return {codes, reinterpret_cast<const S *>(p.scales) + at * p.scales_stride, p.zeros + at * p.zeros_stride};
}

// x in LDS as a whole, put there once; a workgroup takes several blocks of tiles with it.  Wavefronts that share a tile take a run of its slabs each, four at a
// time, of which the next four are asked for before these are multiplied.
template <int PARTS, int G, typename S, bool Z, typename X> __global__ void __launch_bounds__(kMatvecThreads, 4) matvec_quantized_kernel(const MatvecParams p) {
  constexpr int TILES = 1, WIDE = 1, kSlabs = Batch<G, S>::kSlabs;
  extern __shared__ __align__(16) char s_dyn[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int share = 1 << p.share_log, part_of = wave & (share - 1), tile_of = wave >> p.share_log, tiles_each = (blockDim.x >> 6) >> p.share_log;
  const int column = lane & 15, quarter = lane >> 4;
  const long long r0 = (long long)blockIdx.y * kMatvecRows;
  const int rows = (int)(p.R - r0 < 16 * TILES ? p.R - r0 : 16 * TILES), pitch = pitch_of(rows);
  uint4 *s_x = reinterpret_cast<uint4 *>(s_dyn);
  float *s_sum = reinterpret_cast<float *>(s_dyn + (size_t)p.slabs * 256 * PARTS * pitch);
  float *s_join = s_sum + p.slabs * (128 / G) * (TILES * 16);
  const int whole = (int)(p.D / 128), each = (p.slabs + share - 1) >> p.share_log;
  const int begin = part_of * each < whole ? part_of * each : whole, end = begin + each < whole ? begin + each : whole;
  const bool last_too = whole < p.slabs && part_of == whole / each;
  int at_x[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) at_x[t] = quarter * pitch + (16 * t + column < rows ? 16 * t + column : rows - 1);
  for (unsigned block = blockIdx.x; block < p.tile_blocks; block += gridDim.x) {
    const long long n0[WIDE] = {((long long)block * tiles_each + tile_of) * 16};
    const Row<S> row = row_of<S>(p, n0[0] + column);
    f32x4 total[WIDE][TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) total[0][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // (each wavefront's batches: all loads of the loop under no condition, as below)
    Batch<G, S> batch[2];
    const int batches = (end - begin) / kSlabs;
    const auto fetch = [&](Batch<G, S> &to, int i) __attribute__((always_inline)) { load_batch<Z>(to, row.codes, row.scales, row.zeros, begin + (i < batches ? i : batches - 1) * kSlabs, quarter); };
    const auto add = [&](const Batch<G, S> &from, int i) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kSlabs; ++j) {
        const int slab = begin + i * kSlabs + j;
        const Slab<G, S> s[WIDE] = {slab_of<Z>(from, j)};
        add_slab<TILES, PARTS, G, S, WIDE>(total, s, s_x + slab * 16 * PARTS * pitch, s_sum + slab * (128 / G) * 16, at_x, pitch, quarter);
      }
    };
    if (batches > 0) fetch(batch[0], 0);
    if (block == blockIdx.x) {
      const unsigned pieces = (unsigned)p.slabs * 16;
      for (unsigned r = 0; r < (unsigned)rows; ++r)
        for (unsigned piece = threadIdx.x; piece < pieces; piece += blockDim.x) {
          const Piece<X> v = load_x<X>(p, r0 + r, (int)piece * 8);
          store_x<PARTS, G, X>(v, r, piece, pitch, TILES, s_x, s_sum);
        }
      __syncthreads();
    }
    int i = 0;
#pragma unroll 1
    for (; i + 2 <= batches; i += 2) {
      fetch(batch[1], i + 1);
      add(batch[0], i);
      fetch(batch[0], i + 2);
      add(batch[1], i + 1);
    }
    if (i < batches) add(batch[0], i);
#pragma unroll 1
    for (int slab = begin + batches * kSlabs; slab < end + (last_too ? 1 : 0); ++slab) {  // fewer than four, and the row's end
      const Slab<G, S> s[WIDE] = {slab_of<Z>(slab < whole ? load_slab<Z, G, S>(row.codes, row.scales, row.zeros, slab, quarter)
                                                       : load_last_slab<Z, G, S>(p, row.codes, row.scales, row.zeros, slab, quarter))};
      add_slab<TILES, PARTS, G, S, WIDE>(total, s, s_x + slab * 16 * PARTS * pitch, s_sum + slab * (128 / G) * 16, at_x, pitch, quarter);
    }
    int lane_here = lane;
    asm volatile("" : "+v"(lane_here));  // (or every address of the output would be kept in registers from block to block)
    finish_tiles<TILES, WIDE>(p, total, s_join, share, part_of, wave, lane_here, r0, rows, n0);
  }
}

// More rows, or more columns than LDS has room for: x is laid out as LDS will have it by a launch of its own, slab by slab, each with its groups' sums behind it.  A
// wavefront takes a row of a slab.
template <int PARTS, int G, typename X> __global__ void __launch_bounds__(256) matvec_lay_out_kernel(const MatvecParams p) {
  const int lane = threadIdx.x & 63;
  const long long r = blockIdx.y * 4LL + (threadIdx.x >> 6) % 4, block = r / kMatvecRows, r0 = block * kMatvecRows;
  if (r >= p.R) return;
  const unsigned piece = blockIdx.x * 64 + lane, slab = piece >> 4;
  if ((int)slab >= p.slabs) return;  // (16 lanes at a time)
  const int pitch = 16 * p.tiles;
  char *image = p.image + block * p.image_stride + (long long)slab * slab_bytes(PARTS, p.tiles, G);
  const Piece<X> v = (long long)piece * 8 < p.D ? load_x<X>(p, r, (int)piece * 8) : Piece<X>{};
  store_x<PARTS, G, X>(v, (unsigned)(r - r0), piece & 15, pitch, p.tiles, reinterpret_cast<uint4 *>(image), reinterpret_cast<float *>(image + 256 * PARTS * pitch));
}

// x by parts of a few slabs, in two places of LDS in turn: the next part of x, then the codes of the one after it, are asked for before this one is multiplied (in this
// order: loads return in the order they were asked for in).  A wavefront has two
// tiles of columns, so that what it reads of x serves both; every workgroup takes its tiles through all of x once.  Wavefronts that share tiles take a slab of
// a part each.  Every load is made under no condition, those behind an end from the last place there is: how many are under way is known then, and each is waited for by
// itself.  (64 rows of 4096 with 128 256 columns: 122 us in bf16, 213 in fp32; 61 of 2050 in fp32 with 50 257: 78.  With a condition around what a part does not need, 64 rows of 4096 with 128 256 columns took 194 us in bf16.)
template <int TILES, int PARTS, int G, typename S, bool Z, bool SHARED>
__global__ void __launch_bounds__(kMatvecThreads, 2) matvec_streamed_kernel(const MatvecParams p) {
  constexpr int WIDE = 2, kSlabs = streamed_slabs(TILES, PARTS), kShare = SHARED ? kSlabs : 1, kTurns = kSlabs / kShare;
  constexpr int kSize = (int)slab_bytes(PARTS, TILES, G), kPlace = kSize * kSlabs, kUnits = kPlace / 16, kEach = (kUnits + kMatvecThreads - 1) / kMatvecThreads;
  extern __shared__ __align__(16) char s_dyn[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part_of = wave % kShare, tile_of = wave / kShare, column = lane & 15, quarter = lane >> 4;
  constexpr int kTilesEach = (kMatvecThreads >> 6) / kShare;
  const long long r0 = (long long)blockIdx.y * kMatvecRows;
  const int rows = (int)(p.R - r0 < kMatvecRows ? p.R - r0 : kMatvecRows);
  const u32x4 *image = reinterpret_cast<const u32x4 *>(p.image + blockIdx.y * p.image_stride);
  const int whole = (int)(p.D / 128), chunks = (p.slabs + kSlabs - 1) / kSlabs;
  const unsigned image_units = (unsigned)p.slabs * (kSize / 16);  // (over 2^31 of the longest rows)
  long long n0[WIDE];
  Row<S> row[WIDE];
  f32x4 total[WIDE][TILES];
#pragma unroll
  for (int w = 0; w < WIDE; ++w) {
    const int tile = tile_of + w * kTilesEach;
    const long long at = (long long)blockIdx.x * p.block_tiles + tile;
    n0[w] = tile < p.block_tiles && at * 16 < p.N ? at * 16 : -1;
    row[w] = row_of<S>(p, (n0[w] < 0 ? 0 : n0[w]) + column);
    if (whole == 0) row[w] = {reinterpret_cast<const uint8_t *>(image), reinterpret_cast<const S *>(image), reinterpret_cast<const uint8_t *>(image)};  // (read, not used)
#pragma unroll
    for (int t = 0; t < TILES; ++t) total[w][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const int last_whole = whole > 0 ? whole - 1 : 0;
  u32x4 next[kEach];
  RawSlab<G, S> coming[2][kTurns][WIDE];
  const auto ask_x = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int in = i * kMatvecThreads + (int)threadIdx.x;
      const unsigned at = (unsigned)chunk * kUnits + (in < kUnits ? in : kUnits - 1);
      next[i] = image[at < image_units ? at : image_units - 1];
    }
  };
  const auto ask_codes = [&](RawSlab<G, S> (&to)[kTurns][WIDE], int chunk) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int slab = chunk * kSlabs + i * kShare + part_of;
#pragma unroll
      for (int w = 0; w < WIDE; ++w) to[i][w] = load_slab<Z, G, S>(row[w].codes, row[w].scales, row[w].zeros, slab < last_whole ? slab : last_whole, quarter);
    }
  };
  const auto step = [&](char *at_place, RawSlab<G, S> (&codes)[kTurns][WIDE], int chunk) __attribute__((always_inline)) {
    // (the place is free: all have been through the last barrier after they were done with it)
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int in = i * kMatvecThreads + (int)threadIdx.x;
      reinterpret_cast<u32x4 *>(at_place)[in < kUnits ? in : kUnits - 1] = next[i];  // (the last one by several lanes, the same)
    }
    Slab<G, S> now[kTurns][WIDE];
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
#pragma unroll
      for (int w = 0; w < WIDE; ++w) now[i][w] = slab_of<Z>(codes[i][w]);
    __builtin_amdgcn_sched_barrier(0);
    ask_x(chunk + 1 < chunks ? chunk + 1 : chunk);
    __builtin_amdgcn_sched_barrier(0);
    ask_codes(codes, chunk + 2 < chunks ? chunk + 2 : chunk);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int in = i * kShare + part_of, slab = chunk * kSlabs + in;
      if (slab < whole) {  // (uniform)
        const char *at = at_place + in * kSize;
        add_streamed_slab<TILES, PARTS, G, S, WIDE>(total, now[i], reinterpret_cast<const uint4 *>(at), reinterpret_cast<const float *>(at + 256 * PARTS * 16 * TILES), lane);
      }
    }
  };
  ask_codes(coming[0], 0);
  ask_x(0);
  __builtin_amdgcn_sched_barrier(0);
  ask_codes(coming[1], chunks > 1 ? 1 : 0);
#pragma unroll 1
  for (int chunk = 0; chunk < chunks; chunk += 2) {
    step(s_dyn, coming[0], chunk);
    if (chunk + 1 >= chunks) break;
    step(s_dyn + kPlace, coming[1], chunk + 1);
  }
  if (whole < p.slabs && (whole % kSlabs) % kShare == part_of) {  // the row's end, whose part of x is still there
    const char *at = s_dyn + (((chunks - 1) & 1) != 0 ? kPlace : 0) + (whole % kSlabs) * kSize;
    Slab<G, S> now[WIDE];
#pragma unroll
    for (int w = 0; w < WIDE; ++w) {
      const Row<S> r = row_of<S>(p, (n0[w] < 0 ? 0 : n0[w]) + column);
      now[w] = slab_of<Z>(load_last_slab<Z, G, S>(p, r.codes, r.scales, r.zeros, whole, quarter));
    }
    add_streamed_slab<TILES, PARTS, G, S, WIDE>(total, now, reinterpret_cast<const uint4 *>(at), reinterpret_cast<const float *>(at + 256 * PARTS * 16 * TILES), lane);
  }
  finish_tiles<TILES, WIDE>(p, total, reinterpret_cast<float *>(s_dyn + 2 * kPlace), kShare, part_of, wave, lane, r0, rows, n0);
}

template <int PARTS, int G, typename X> hipError_t lay_out(const MatvecParams &p, hipStream_t st) {
  const dim3 grid((unsigned)((p.slabs * 16 + 63) / 64), (unsigned)((p.R + 3) / 4));
  matvec_lay_out_kernel<PARTS, G, X><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}
template <int TILES, int PARTS, int G, typename S, bool Z, typename X> hipError_t launch_tiles(const MatvecParams &p, dim3 grid, size_t lds, hipStream_t st) {
  if (p.streamed == 0) {  // (up to 16 rows)
    matvec_quantized_kernel<PARTS, G, S, Z, X><<<grid, kMatvecThreads, lds, st>>>(p);
  } else {
    const hipError_t e = lay_out<PARTS, G, X>(p, st);
    if (e != hipSuccess) return e;
    if (p.share_log == 0) matvec_streamed_kernel<TILES, PARTS, G, S, Z, false><<<grid, kMatvecThreads, lds, st>>>(p);
    else if constexpr (streamed_slabs(TILES, PARTS) > 1) matvec_streamed_kernel<TILES, PARTS, G, S, Z, true><<<grid, kMatvecThreads, lds, st>>>(p);
  }
  return hipGetLastError();
}
template <int PARTS, int G, typename S, bool Z, typename X> hipError_t by_zeros(const MatvecParams &p, int tiles, dim3 grid, size_t lds, hipStream_t st) {
  switch (tiles) {
    case 1: return launch_tiles<1, PARTS, G, S, Z, X>(p, grid, lds, st);
    case 2: return launch_tiles<2, PARTS, G, S, Z, X>(p, grid, lds, st);
    case 3: return launch_tiles<3, PARTS, G, S, Z, X>(p, grid, lds, st);
    default: return launch_tiles<4, PARTS, G, S, Z, X>(p, grid, lds, st);
  }
}
template <int PARTS, int G, typename S, typename X> hipError_t by_tiles(const MatvecParams &p, int tiles, dim3 grid, size_t lds, hipStream_t st) {
  return p.zeros != nullptr ? by_zeros<PARTS, G, S, true, X>(p, tiles, grid, lds, st) : by_zeros<PARTS, G, S, false, X>(p, tiles, grid, lds, st);
}
template <int PARTS, typename X> hipError_t launch_matvec(const MatvecParams &p, int tiles, int group, int scales_type, dim3 grid, size_t lds, hipStream_t st) {
  const bool wide = scales_type == LLC_F32;
  if (group == 128) return wide ? by_tiles<PARTS, 128, float, X>(p, tiles, grid, lds, st) : by_tiles<PARTS, 128, uint16_t, X>(p, tiles, grid, lds, st);
  if (group == 64) return wide ? by_tiles<PARTS, 64, float, X>(p, tiles, grid, lds, st) : by_tiles<PARTS, 64, uint16_t, X>(p, tiles, grid, lds, st);
  return wide ? by_tiles<PARTS, 32, float, X>(p, tiles, grid, lds, st) : by_tiles<PARTS, 32, uint16_t, X>(p, tiles, grid, lds, st);
}

}  // namespace
}  // namespace llc
