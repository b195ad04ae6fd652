// Embedding lookup with scaling, and its gradient.  One workgroup a token, or a row of the gradient.
#include "ends.hpp"

namespace llc {
namespace {

struct EmbedParams {
  long long T, N, D;
  const void *from;         // table, or the gradient of the output
  long long from_stride;
  const int32_t *tokens;
  long long tok_stride;
  float scale;
  int add;
  void *to;                 // output, or the gradient of the table
  long long to_stride;
};

template <typename A, typename B> __global__ void __launch_bounds__(kBlock) embed_kernel(const EmbedParams p) {
  for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
    const long long n = p.tokens[t * p.tok_stride];
    B *to = reinterpret_cast<B *>(p.to) + t * p.to_stride;
    const bool there = n >= 0 && n < p.N;
    const A *from = reinterpret_cast<const A *>(p.from) + (there ? n : 0) * p.from_stride;
    for (long long d = threadIdx.x; d < p.D; d += kBlock) to[d] = narrow<B>(there ? widen(from[d]) * p.scale : 0.0f);
  }
}

template <typename A, typename B> __global__ void __launch_bounds__(kBlock) embed_grad_kernel(const EmbedParams p) {
  __shared__ int s_any;
  __shared__ uint8_t s_hit[kBlock];
  for (long long item = blockIdx.x, slabs = (p.D + kBlock - 1) / kBlock; item < p.N * slabs; item += gridDim.x) {
    const long long n = item / slabs, d0 = item % slabs * kBlock;
    B *to = reinterpret_cast<B *>(p.to) + n * p.to_stride;
    const long long d = d0 + threadIdx.x;
    float sum = 0.0f;
    bool met = false;
    for (long long t0 = 0; t0 < p.T; t0 += kBlock) {
      const long long mine = t0 + threadIdx.x;
      __syncthreads();
      if (threadIdx.x == 0) s_any = 0;
      __syncthreads();
      const bool hit = mine < p.T && p.tokens[mine * p.tok_stride] == n;
      s_hit[threadIdx.x] = hit ? 1 : 0;
      if (hit) s_any = 1;
      __syncthreads();
      if (s_any == 0) continue;
      met = true;
      for (int j = 0; j < kBlock; ++j)
        if (s_hit[j] != 0 && d < p.D) sum += widen(reinterpret_cast<const A *>(p.from)[(t0 + j) * p.from_stride + d]);
    }
    if (d < p.D && (met || p.add == 0)) to[d] = narrow<B>((p.add != 0 ? widen(to[d]) : 0.0f) + sum * p.scale);
  }
}

template <typename F> hipError_t by_types(int from, int to, F launch) {
  if (from == LLC_F32) return to == LLC_F32 ? launch(float(), float()) : launch(float(), uint16_t());
  return to == LLC_F32 ? launch(uint16_t(), float()) : launch(uint16_t(), uint16_t());
}

bool sizes_ok(long long T, long long N, long long D) {
  return T >= 0 && T <= kMaxIndex && N >= 1 && N <= kMaxIndex && D >= 1 && D <= kMaxIndex;
}

unsigned blocks(long long items) { return (unsigned)(items < (1 << 20) ? items : 1 << 20); }

constexpr long long kMostRows = 1LL << 27;

}  // namespace
}  // namespace llc

using namespace llc;

extern "C" int llc_embed(const llc_embed_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  if (!sizes_ok(a->T, a->N, a->D)) return LLC_E_SHAPE;
  if ((a->flags & ~LLC_FLAG_DRY_RUN) != 0 || !std::isfinite(a->scale)) return LLC_E_OPTION;
  if (a->T == 0) return LLC_OK;
  if (a->table == nullptr || a->tokens == nullptr || a->out == nullptr) return LLC_E_NULL;
  if (a->table_stride_n < 0 || a->tok_stride < 0 || a->out_stride_t < a->D) return LLC_E_SHAPE;
  if (!known_type(a->dtype) || !known_type(a->out_dtype)) return LLC_E_DTYPE;
  if (!fits(a->table, type_size(a->dtype)) || !fits(a->out, type_size(a->out_dtype)) || !fits(a->tokens, 4)) return LLC_E_ALIGN;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  EmbedParams p = {a->T, a->N, a->D, a->table, a->table_stride_n, a->tokens, a->tok_stride, a->scale, 0, a->out, a->out_stride_t};
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    return by_types(a->dtype, a->out_dtype, [&](auto from, auto to) {
      embed_kernel<decltype(from), decltype(to)><<<blocks(p.T), kBlock, 0, st>>>(p);
      return hipGetLastError();
    });
  });
}

extern "C" size_t llc_embed_grad_workspace_size(int64_t T, int64_t N, int64_t D) {
  return sizes_ok(T, N, D) && N <= kMostRows ? 256 : 0;
}

extern "C" int llc_embed_grad(const llc_embed_grad_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  if (!sizes_ok(a->T, a->N, a->D) || a->N > kMostRows) return LLC_E_SHAPE;
  if ((a->flags & ~LLC_FLAG_DRY_RUN) != 0 || !std::isfinite(a->scale)) return LLC_E_OPTION;
  if (a->T == 0 && a->add != 0) return LLC_OK;
  if ((a->T > 0 && (a->g == nullptr || a->tokens == nullptr)) || a->grad == nullptr) return LLC_E_NULL;
  if (a->g_stride_t < 0 || a->tok_stride < 0 || a->grad_stride_n < a->D) return LLC_E_SHAPE;
  if (!known_type(a->dtype) || !known_type(a->grad_dtype)) return LLC_E_DTYPE;
  if (!fits(a->g, type_size(a->dtype)) || !fits(a->grad, type_size(a->grad_dtype)) || !fits(a->tokens, 4)) return LLC_E_ALIGN;
  if (a->workspace == nullptr || !fits(a->workspace, 256) || a->workspace_bytes < llc_embed_grad_workspace_size(a->T, a->N, a->D))
    return LLC_E_WORKSPACE;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  EmbedParams p = {a->T, a->N, a->D, a->g, a->g_stride_t, a->tokens, a->tok_stride, a->scale, a->add, a->grad, a->grad_stride_n};
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    return by_types(a->dtype, a->grad_dtype, [&](auto from, auto to) {
      embed_grad_kernel<decltype(from), decltype(to)><<<blocks(p.N * ((p.D + kBlock - 1) / kBlock)), kBlock, 0, st>>>(p);
      return hipGetLastError();
    });
  });
}
