// Products of a few rows with a layer held in 4 bits: out[r,n] = sum over groups g of scale[n,g] * sum over d in g of (q[n,d] - zero[n,g]) x[r,d].
//
// The codes are read once and bound the call (a layer of 128 256 x 4096 is 263 MB); matrix instructions take the products, 16 columns of the output by 16
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

// Column of a slab where the quarter's word of a step starts.
template <int G> __device__ __forceinline__ int column_of(int step, int quarter) {
  if constexpr (G == 128) return 32 * quarter + 8 * step;
  if constexpr (G == 64) return 64 * (step >> 1) + 16 * quarter + 8 * (step & 1);
  return 32 * step + 8 * quarter;
}

template <int G, typename S>
__device__ __forceinline__ void load_scales(Slab<G, S> &s, const MatvecParams &p, const S *scales, const uint8_t *zeros, int slab) {
#pragma unroll
  for (int g = 0; g < 128 / G; ++g) {
    int of = slab * (128 / G) + g;
    of = of < p.groups ? of : p.groups - 1;  // (columns behind the row's end: x is 0 there)
    s.scale[g] = widen(scales[of]);
    s.shift[g] = zeros != nullptr ? -16.0f - (float)zeros[of] : -24.0f;
  }
}
template <int G, typename S>
__device__ __forceinline__ Slab<G, S> load_slab(const MatvecParams &p, const uint8_t *codes, const S *scales, const uint8_t *zeros, int slab, int quarter) {
  Slab<G, S> s;
  const uint8_t *from = codes + (long long)slab * 64;
  if constexpr (G == 128) {
    const word4_byte w = *reinterpret_cast<const word4_byte *>(from + 16 * quarter);
    s.words[0] = w.x; s.words[1] = w.y; s.words[2] = w.z; s.words[3] = w.w;
  } else if constexpr (G == 64) {
    const word2_byte a = *reinterpret_cast<const word2_byte *>(from + 8 * quarter);
    const word2_byte b = *reinterpret_cast<const word2_byte *>(from + 32 + 8 * quarter);
    s.words[0] = a.x; s.words[1] = a.y; s.words[2] = b.x; s.words[3] = b.y;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) s.words[i] = *reinterpret_cast<const word1_byte *>(from + 16 * i + 4 * quarter);
  }
  load_scales(s, p, scales, zeros, slab);
  return s;
}
// The last slab of a row that is not a whole one.
template <int G, typename S>
__device__ __forceinline__ Slab<G, S> load_last_slab(const MatvecParams &p, const uint8_t *codes, const S *scales, const uint8_t *zeros, int slab, int quarter) {
  Slab<G, S> s;
#pragma unroll
  for (int i = 0; i < 4; ++i) s.words[i] = load_codes(codes, (long long)slab * 128 + column_of<G>(i, quarter), p.D);
  load_scales(s, p, scales, zeros, slab);
  return s;
}

// Adds a slab's products to a tile's sums; `here`: its place in the chunk.
template <int TILES, int PARTS, int G, typename S>
__device__ __forceinline__ void add_slab(f32x4 (&total)[TILES], const Slab<G, S> &s, const uint4 *s_x, const float *s_sum, const int (&at_x)[TILES], int rows, int here,
                                         int quarter) {
  constexpr int kSteps = G / 32;  // of a group
  f32x4 sum[TILES], low[TILES];
#pragma unroll
  for (int step = 0; step < 4; ++step) {
    const int g = step / kSteps;
    if (step % kSteps == 0) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const f32x4 sx = *reinterpret_cast<const f32x4 *>(s_sum + (here * (128 / G) + g) * (TILES * 16) + 16 * t + 4 * quarter);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[t][j] = s.shift[g] * sx[j];
        low[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    const bf16x8 w = widen_codes(s.words[step]);
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        const bf16x8 a = __builtin_bit_cast(bf16x8, s_x[((here * 4 + step) * PARTS + part) * 4 * rows + at_x[t]]);
        if (part == 0) sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w, sum[t], 0, 0, 0);
        else low[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w, low[t], 0, 0, 0);
      }
    }
    if (step % kSteps == kSteps - 1) {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) total[t][j] = fmaf(s.scale[g], PARTS > 1 ? sum[t][j] + low[t][j] : sum[t][j], total[t][j]);
    }
  }
}

// x of a chunk of columns to LDS, as the operands lie: [slab][step][part][quarter][row], 16 bytes each; and the groups' sums [group][16 rows of a tile].
template <int TILES, int PARTS, int G, typename X>
__device__ __forceinline__ void stage_x(const MatvecParams &p, long long r0, int rows, int chunk, int slabs, uint4 *s_x, float *s_sum) {
  const unsigned pieces = (unsigned)slabs * 16, all = pieces * (unsigned)rows;
  for (unsigned i = threadIdx.x; i < all; i += blockDim.x) {
    const unsigned r = i / pieces, piece = i - r * pieces;
    const long long at = ((long long)chunk * p.chunk_slabs * 16 + piece) * 8;
    const X *row = reinterpret_cast<const X *>(p.x) + (r0 + r) * p.x_stride;
    float v[8];
    if (at < p.D) {
      load_first<8>(row + at, p.D - at, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.0f;
    }
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += v[j];
    sum = sum_lanes<G / 8>(sum);
    const unsigned slab = piece >> 4, q = piece & 15;
    const unsigned step = G == 128 ? q & 3 : G == 64 ? (q >> 3) * 2 + (q & 1) : q >> 2;
    const unsigned quarter = G == 128 ? q >> 2 : G == 64 ? (q >> 1) & 3 : q & 3;
    if ((q & (G / 8 - 1)) == 0) s_sum[(slab * (128 / G) + q / (G / 8)) * (TILES * 16) + r] = sum;
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      const uint4 w = make_uint4(narrow_pair(v[0], v[4]), narrow_pair(v[1], v[5]), narrow_pair(v[2], v[6]), narrow_pair(v[3], v[7]));
      s_x[(((slab * 4 + step) * PARTS + part) * 4 + quarter) * rows + r] = w;
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
}

template <int TILES, int PARTS, int G, typename S, typename X>
__global__ void __launch_bounds__(kMatvecThreads) matvec_quantized_kernel(const MatvecParams p) {
  constexpr int kAhead = 4;  // slabs that are fetched ahead
  extern __shared__ __align__(16) char s_dyn[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int share = 1 << p.share_log, part_of = wave & (share - 1), tile_of = wave >> p.share_log, tiles_each = waves >> p.share_log;
  const int column = lane & 15, quarter = lane >> 4;
  const long long r0 = (long long)blockIdx.y * kMatvecRows;
  const int rows = (int)(p.R - r0 < 16 * TILES ? p.R - r0 : 16 * TILES);
  uint4 *s_x = reinterpret_cast<uint4 *>(s_dyn);
  float *s_sum = reinterpret_cast<float *>(s_dyn + (size_t)p.chunk_slabs * 256 * PARTS * rows);
  float *s_join = s_sum + p.chunk_slabs * (128 / G) * (TILES * 16);
  const int chunks = (p.slabs + p.chunk_slabs - 1) / p.chunk_slabs, turns = p.chunk_slabs >> p.share_log;
  const int whole = (int)(p.D / 128);  // whole slabs
  int at_x[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) at_x[t] = quarter * rows + (16 * t + column < rows ? 16 * t + column : rows - 1);
  for (unsigned block = blockIdx.x; block < p.tile_blocks; block += gridDim.x) {
    const long long n0 = ((long long)block * tiles_each + tile_of) * 16, n = n0 + column < p.N ? n0 + column : p.N - 1;
    const uint8_t *codes = p.codes + n * p.codes_stride;
    const S *scales = reinterpret_cast<const S *>(p.scales) + n * p.scales_stride;
    const uint8_t *zeros = p.zeros != nullptr ? p.zeros + n * p.zeros_stride : nullptr;
    f32x4 total[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) total[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    Slab<G, S> ring[kAhead];
    // (a slab behind the last whole one is that one again, and is not added)
    const auto fetch = [&](int turn) {
      const int slab = turn * share + part_of;
      return load_slab<G, S>(p, codes, scales, zeros, slab < whole ? slab : whole - 1, quarter);
    };
    for (int chunk = 0; chunk < chunks; ++chunk) {
      if (whole > 0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ring[i] = fetch(chunk * turns + i);
      }
      const int left = p.slabs - chunk * p.chunk_slabs;
      if (chunks > 1 || block == blockIdx.x) {
        __syncthreads();
        stage_x<TILES, PARTS, G, X>(p, r0, rows, chunk, left < p.chunk_slabs ? left : p.chunk_slabs, s_x, s_sum);
        __syncthreads();
      }
      const int whole_here = whole - chunk * p.chunk_slabs;
      for (int turn0 = 0; turn0 < turns; turn0 += kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int turn = turn0 + i, here = turn * share + part_of;
          if (turn < turns && here < whole_here) {  // (uniform)
            add_slab<TILES, PARTS, G, S>(total, ring[i], s_x, s_sum, at_x, rows, here, quarter);
            ring[i] = fetch(chunk * turns + turn + kAhead);
          }
        }
      }
      if (whole < p.slabs && left <= p.chunk_slabs && (whole_here & (share - 1)) == part_of)  // (uniform)
        add_slab<TILES, PARTS, G, S>(total, load_last_slab<G, S>(p, codes, scales, zeros, whole, quarter), s_x, s_sum, at_x, rows, whole_here, quarter);
    }
    if (share > 1) {
      __syncthreads();
#pragma unroll
      for (int t = 0; t < TILES; ++t) *reinterpret_cast<f32x4 *>(s_join + ((wave * TILES + t) * 64 + lane) * 4) = total[t];
      __syncthreads();
      if (part_of == 0) {
        for (int other = 1; other < share; ++other)
#pragma unroll
          for (int t = 0; t < TILES; ++t) {
            const f32x4 add = *reinterpret_cast<const f32x4 *>(s_join + (((wave + other) * TILES + t) * 64 + lane) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) total[t][j] += add[j];
          }
      }
    }
    if (part_of == 0 && n0 + column < p.N) {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 16 * t + 4 * quarter + j;
          if (r < rows) {
            const long long to = (r0 + r) * p.out_stride + n0 + column;
            if (p.out_type == LLC_F32) reinterpret_cast<float *>(p.out)[to] = total[t][j];
            else reinterpret_cast<uint16_t *>(p.out)[to] = narrow<uint16_t>(total[t][j]);
          }
        }
    }
  }
}

template <int PARTS, int G, typename S, typename X>
hipError_t by_tiles(const MatvecParams &p, int tiles, dim3 grid, int threads, size_t lds, hipStream_t st) {
  switch (tiles) {
    case 1: matvec_quantized_kernel<1, PARTS, G, S, X><<<grid, threads, lds, st>>>(p); break;
    case 2: matvec_quantized_kernel<2, PARTS, G, S, X><<<grid, threads, lds, st>>>(p); break;
    case 3: matvec_quantized_kernel<3, PARTS, G, S, X><<<grid, threads, lds, st>>>(p); break;
    default: matvec_quantized_kernel<4, PARTS, G, S, X><<<grid, threads, lds, st>>>(p); break;
  }
  return hipGetLastError();
}
template <int PARTS, typename X>
hipError_t launch_matvec(const MatvecParams &p, int tiles, int group, int scales_type, dim3 grid, int threads, size_t lds, hipStream_t st) {
  const bool wide = scales_type == LLC_F32;
  if (group == 128) return wide ? by_tiles<PARTS, 128, float, X>(p, tiles, grid, threads, lds, st) : by_tiles<PARTS, 128, uint16_t, X>(p, tiles, grid, threads, lds, st);
  if (group == 64) return wide ? by_tiles<PARTS, 64, float, X>(p, tiles, grid, threads, lds, st) : by_tiles<PARTS, 64, uint16_t, X>(p, tiles, grid, threads, lds, st);
  return wide ? by_tiles<PARTS, 32, float, X>(p, tiles, grid, threads, lds, st) : by_tiles<PARTS, 32, uint16_t, X>(p, tiles, grid, threads, lds, st);
}

}  // namespace
}  // namespace llc
