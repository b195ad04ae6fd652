// What the kernels of layers held in 4 bits (quantized.hip, matvec_quantized_*.hip) share.
#pragma once

#include "ends.hpp"

namespace llc {

inline bool known_group(int group) { return group == 32 || group == 64 || group == 128; }
inline long long groups_of(long long D, int group) { return (D + group - 1) / group; }

// Loads of bytes wherever they start.
typedef uint16_t half_byte __attribute__((aligned(1)));
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
  int share_log;    // log2 of the wavefronts that share a tile by columns (where x is streamed: one, or as many as a part has slabs)
  unsigned tile_blocks;  // workgroups' worth of tiles
  // where x is streamed:
  int tiles;             // of 16 rows, of up to 64
  int block_tiles;       // of 16 columns, that a workgroup takes
  char *image;           // x as LDS has it, 64 rows at a time
  long long image_stride;
};
constexpr int kMatvecThreads = 512;
constexpr int kMatvecRows = 64;  // rows of x that one pass over the layer serves

// Slabs of a part of x, where it is streamed: two parts fit LDS beside the sums of wavefronts that share tiles, and the next one the registers.
__host__ __device__ constexpr int streamed_slabs(int tiles, int parts) { return parts == 1 ? (tiles <= 2 ? 4 : 2) : tiles == 1 ? 4 : tiles == 2 ? 2 : 1; }
// Bytes of a slab of x with its groups' sums, as it is laid out.
__host__ __device__ constexpr long long slab_bytes(int parts, int tiles, int group) { return 256LL * parts * 16 * tiles + (128 / group) * tiles * 64; }

__host__ __device__ inline int pitch_of(int rows) { return rows | 1; }  // (of rows in LDS, where they are put there from memory)

// (one translation unit for each type of x)
hipError_t launch_matvec_bf16(const MatvecParams &p, int tiles, int group, int scales_type, dim3 grid, size_t lds, hipStream_t st);
hipError_t launch_matvec_f32(const MatvecParams &p, int tiles, int group, int scales_type, dim3 grid, size_t lds, hipStream_t st);

}  // namespace llc
