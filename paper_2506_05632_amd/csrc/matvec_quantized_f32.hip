// Products with a layer held in 4 bits: x in fp32, as three bf16 parts.
#include "matvec_quantized.hpp"

namespace llc {
hipError_t launch_matvec_f32(const MatvecParams &p, int tiles, int group, int scales_type, dim3 grid, size_t lds, hipStream_t st) {
  return launch_matvec<3, float>(p, tiles, group, scales_type, grid, lds, st);
}
}  // namespace llc
