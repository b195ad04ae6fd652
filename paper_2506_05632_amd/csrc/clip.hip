// The global norm over many tensors, and clipping by it.  Tensors go to a launch a table at a time (the table is a
// kernel argument, so nothing is copied to the device); every workgroup adds up its share of the table's entries, and the
// workgroups of the second launch join those partial sums, in the same order everywhere, before they scale.
#include "ends.hpp"

namespace llc {
namespace {

constexpr int kTable = 128;        // tensors a launch
constexpr int kSquareBlocks = 512; // workgroups a launch, and partial sums

struct ClipParams {
  const void *from[kTable];
  void *to[kTable];
  long long numel[kTable];
  uint8_t dtype[kTable];
  int n;
  double *partials;  // this table's
  const double *all; // every table's
  int n_all;
  float max_norm;
  float *norm;       // written by the first launch of the second kind
};

__device__ double sum_over_workgroup(double v) {
  __shared__ double s[kBlock / 64];
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
  for (int w = 1; w < kBlock / 64; ++w) v += s[w];
  return v;
}

__global__ void __launch_bounds__(kBlock) square_kernel(const ClipParams p) {
  double s = 0.0;
  for (int j = 0; j < p.n; ++j)
    for (long long i = (long long)blockIdx.x * kBlock + threadIdx.x; i < p.numel[j]; i += (long long)gridDim.x * kBlock) {
      const double v = p.dtype[j] == LLC_F32 ? (double)reinterpret_cast<const float *>(p.from[j])[i]
                                             : (double)widen(reinterpret_cast<const uint16_t *>(p.from[j])[i]);
      s += v * v;
    }
  s = sum_over_workgroup(s);
  if (threadIdx.x == 0) p.partials[blockIdx.x] = s;
}

__global__ void __launch_bounds__(kBlock) clip_kernel(const ClipParams p) {
  double s = 0.0;
  for (int i = threadIdx.x; i < p.n_all; i += kBlock) s += p.all[i];
  const double norm = sqrt(sum_over_workgroup(s));
  if (p.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = (float)norm;
  const float factor = norm > (double)p.max_norm && norm < __builtin_huge_val() ? (float)((double)p.max_norm / norm) : 1.0f;
  for (int j = 0; j < p.n; ++j) {
    if (factor == 1.0f && p.from[j] == p.to[j]) continue;
    for (long long i = (long long)blockIdx.x * kBlock + threadIdx.x; i < p.numel[j]; i += (long long)gridDim.x * kBlock) {
      if (p.dtype[j] == LLC_F32)
        reinterpret_cast<float *>(p.to[j])[i] = reinterpret_cast<const float *>(p.from[j])[i] * factor;
      else
        reinterpret_cast<uint16_t *>(p.to[j])[i] = narrow<uint16_t>(widen(reinterpret_cast<const uint16_t *>(p.from[j])[i]) * factor);
    }
  }
}

}  // namespace
}  // namespace llc

using namespace llc;

extern "C" size_t llc_clip_grad_norm_workspace_size(int64_t n) {
  if (n < 0 || n > (1 << 20)) return 0;
  return (size_t)((n + kTable - 1) / kTable + 1) * kSquareBlocks * sizeof(double);
}

extern "C" int llc_clip_grad_norm(const llc_clip_grad_norm_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  if (a->n < 0 || a->n > (1 << 20)) return LLC_E_SHAPE;
  if ((a->flags & ~LLC_FLAG_DRY_RUN) != 0 || !(a->max_norm > 0.0f)) return LLC_E_OPTION;
  if (a->norm == nullptr || (a->n > 0 && (a->grads == nullptr || a->numel == nullptr || a->dtype == nullptr))) return LLC_E_NULL;
  long long total = 0;
  for (int64_t j = 0; j < a->n; ++j) {
    if (a->numel[j] < 0 || a->numel[j] > (1LL << 40) || (total += a->numel[j]) > (1LL << 40)) return LLC_E_SHAPE;
    if (!known_type(a->dtype[j])) return LLC_E_DTYPE;
    const void *to = a->out != nullptr ? a->out[j] : a->grads[j];
    if (a->numel[j] > 0 && (a->grads[j] == nullptr || to == nullptr)) return LLC_E_NULL;
    if (!fits(a->grads[j], type_size(a->dtype[j])) || !fits(to, type_size(a->dtype[j]))) return LLC_E_ALIGN;
  }
  if (!fits(a->norm, 4)) return LLC_E_ALIGN;
  if (a->workspace == nullptr || !fits(a->workspace, 256) || a->workspace_bytes < llc_clip_grad_norm_workspace_size(a->n))
    return LLC_E_WORKSPACE;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    const int tables = a->n > 0 ? (int)((a->n + kTable - 1) / kTable) : 1;
    for (int pass = 0; pass < 2; ++pass)
      for (int t = 0; t < tables; ++t) {
        ClipParams p = {};
        const int64_t j0 = (int64_t)t * kTable;
        p.n = (int)(a->n - j0 < kTable ? a->n - j0 : kTable);
        for (int j = 0; j < p.n; ++j) {
          p.from[j] = a->grads[j0 + j];
          p.to[j] = a->out != nullptr ? a->out[j0 + j] : a->grads[j0 + j];
          p.numel[j] = a->numel[j0 + j];
          p.dtype[j] = (uint8_t)a->dtype[j0 + j];
        }
        p.partials = (double *)a->workspace + (size_t)t * kSquareBlocks;
        p.all = (const double *)a->workspace;
        p.n_all = tables * kSquareBlocks;
        p.max_norm = a->max_norm;
        p.norm = t == 0 ? a->norm : nullptr;
        if (pass == 0) square_kernel<<<kSquareBlocks, kBlock, 0, st>>>(p);
        else clip_kernel<<<kSquareBlocks, kBlock, 0, st>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
    return hipSuccess;
  });
}
