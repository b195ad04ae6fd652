// What the kernels of layers held in 4 bits (quantized.hip, matvec_quantized_*.hip) share.
#pragma once

#include "ends.hpp"

namespace llc {

inline bool known_group(int group) { return group == 32 || group == 64 || group == 128; }
inline long long groups_of(long long D, int group) { return (D + group - 1) / group; }

// Loads of bytes wherever they start.
typedef uint32_t word1_byte __attribute__((aligned(1)));
typedef uint32_t word2_byte __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t word4_byte __attribute__((ext_vector_type(4), aligned(1)));

// Eight codes of a row from an even place on, of which the row may hold fewer: the others read as 0.
__device__ __forceinline__ uint32_t load_codes(const uint8_t *row, long long at, long long D) {
  if (at + 8 <= D) return *reinterpret_cast<const word1_byte *>(row + at / 2);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (at + 2 * i < D) w |= (uint32_t)row[at / 2 + i] << (8 * i);
  return w;
}

struct MatvecParams {
  long long R, N, D;
  const void *x;
  long long x_stride;
  const uint8_t *codes;
  long long codes_stride;
  const void *scales;
  long long scales_stride;
  const uint8_t *zeros;
  long long zeros_stride;
  void *out;
  long long out_stride;
  int out_type;
  int groups;       // of a row
  int slabs;        // of 128 entries, of a row
  int streamed;     // x goes through LDS by parts
  int chunk_log;    // log2 of the slabs of a part, which are at least as many as wavefronts share a tile
  int share_log;    // log2 of the wavefronts that share a tile by columns
  unsigned tile_blocks;  // workgroups' worth of tiles
  int block_tiles;       // that a workgroup takes at a time, where x is streamed
};
constexpr int kMatvecThreads = 512;
constexpr int kMatvecRows = 64;  // rows of x that one pass over the layer serves

template <typename X> constexpr int kStreamedPieces = 8 / sizeof(X);  // of eight columns of x that a thread has in flight

// Bytes of LDS of a workgroup: x and the groups' sums of it, and the sums of wavefronts that share tiles.
inline size_t matvec_x_bytes(int parts, int rows, int tiles, int group, int slabs) { return (size_t)slabs * ((size_t)256 * parts * rows + (size_t)(128 / group) * tiles * 64); }
inline size_t matvec_join_bytes(int tiles, int wide, int share_log) { return share_log > 0 ? (size_t)(kMatvecThreads / 64) * wide * tiles * 1024 : 0; }

// (one translation unit for each type of x)
hipError_t launch_matvec_bf16(const MatvecParams &p, int tiles, int group, int scales_type, dim3 grid, size_t lds, hipStream_t st);
hipError_t launch_matvec_f32(const MatvecParams &p, int tiles, int group, int scales_type, dim3 grid, size_t lds, hipStream_t st);

}  // namespace llc
