// Products with a layer held in 4 bits: x in bf16.
#include "matvec_quantized.hpp"

namespace llc {
hipError_t launch_matvec_bf16(const MatvecParams &p, int tiles, int group, int scales_type, dim3 grid, size_t lds, hipStream_t st) {
  return launch_matvec<1, uint16_t>(p, tiles, group, scales_type, grid, lds, st);
}
}  // namespace llc
