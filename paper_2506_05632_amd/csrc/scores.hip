// Scores of tokens: their log probability, the rows' entropy and top alternatives, and the gradient of the
// first two.  One workgroup a row, one pass for the row's largest entry, one for the sums, one for each alternative.
#include "ends.hpp"

namespace llc {
namespace {

struct ScoreParams {
  long long R;
  int V, G, M;
  const void *x;
  long long stride_r;
  float temp;
  const int32_t *tokens;
  long long tok_stride_r;
  float *logp, *entropy;
  double *lse;
  int32_t *top_ids;
  float *top_logp;
  // the gradient
  const float *a;
  long long a_stride_r;
  const float *b;
  const double *lse_in;
  const float *entropy_in;
  void *grad;
  long long grad_stride_r;
};

constexpr float kInf = __builtin_huge_valf();

__device__ __forceinline__ bool with_mass(float v) { return fabsf(v) < kInf; }

// The order of the values, larger first, then of the indexes, smaller first, as one number (0: no mass).
__device__ __forceinline__ unsigned long long order_of(float v, int i) {
  if (!with_mass(v)) return 0;
  const uint32_t b = __float_as_uint(v + 0.0f);  // (-0 and 0 are equal)
  const uint32_t o = (b & 0x80000000u) != 0 ? ~b : b | 0x80000000u;
  return ((unsigned long long)o << 32) | (0xFFFFFFFFu - (uint32_t)i);
}

template <typename T, typename F> __device__ T over_workgroup(T v, F join, T *scratch) {
  for (int d = 32; d >= 1; d >>= 1) v = join(v, __shfl_xor(v, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  v = scratch[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v = join(v, scratch[w]);
  return v;
}

template <typename E> __global__ void __launch_bounds__(kBlock) score_kernel(const ScoreParams p) {
  __shared__ double s_double[kBlock / 64];
  __shared__ unsigned long long s_order[kBlock / 64];
  const long long r = blockIdx.x;
  const E *x = reinterpret_cast<const E *>(p.x) + r * p.stride_r;
  const double inv_t = 1.0 / (double)p.temp;
  const auto larger = [](unsigned long long u, unsigned long long v) { return u > v ? u : v; };
  const auto sum = [](double u, double v) { return u + v; };
  unsigned long long best = 0;
  for (int i = threadIdx.x; i < p.V; i += kBlock) best = larger(best, order_of(widen(x[i]), i));
  best = over_workgroup(best, larger, s_order);
  const bool any = best != 0;
  const double top = any ? (double)widen(x[0xFFFFFFFFu - (uint32_t)best]) : 0.0;
  double s = 0.0, d = 0.0;
  for (int i = threadIdx.x; any && i < p.V; i += kBlock) {
    const float v = widen(x[i]);
    if (!with_mass(v)) continue;
    const float y = (float)(((double)v - top) * inv_t), e = expf(y);
    s += (double)e;
    if (e > 0.0f) d += (double)e * (double)y;
  }
  s = over_workgroup(s, sum, s_double);
  d = over_workgroup(d, sum, s_double);
  const double rest = any ? log(s) : -(double)kInf;
  const double entropy = any ? rest - d / s : 0.0;
  const auto logp_of = [&](float v) { return (float)(((double)v - top) * inv_t - rest); };
  if (threadIdx.x == 0) {
    if (p.lse != nullptr) { p.lse[2 * r] = top; p.lse[2 * r + 1] = rest; }
    if (p.entropy != nullptr) p.entropy[r] = (float)entropy;
  }
  if (p.logp != nullptr) {
    for (int g = threadIdx.x; g < p.G; g += kBlock) {
      const int t = p.tokens[r * p.tok_stride_r + g];
      float out = t < 0 ? 0.0f : -kInf;
      if (t >= 0 && t < p.V && with_mass(widen(x[t]))) out = logp_of(widen(x[t]));
      p.logp[r * p.G + g] = out;
    }
  }
  unsigned long long last = ~0ull;
  for (int m = 0; m < p.M; ++m) {
    best = 0;
    for (int i = threadIdx.x; last != 0 && i < p.V; i += kBlock) {
      const unsigned long long o = order_of(widen(x[i]), i);
      if (o < last) best = larger(best, o);
    }
    last = over_workgroup(best, larger, s_order);
    if (threadIdx.x == 0) {
      const int i = last != 0 ? (int)(0xFFFFFFFFu - (uint32_t)last) : -1;
      p.top_ids[r * p.M + m] = i;
      p.top_logp[r * p.M + m] = i >= 0 ? logp_of(widen(x[i])) : -kInf;
    }
  }
}

template <typename E> __global__ void __launch_bounds__(kBlock) score_grad_kernel(const ScoreParams p) {
  const long long r = blockIdx.x;
  const E *x = reinterpret_cast<const E *>(p.x) + r * p.stride_r;
  E *out = reinterpret_cast<E *>(p.grad) + r * p.grad_stride_r;
  const int32_t *tokens = p.tokens + r * p.tok_stride_r;
  const float *a = p.a + r * p.a_stride_r;
  const double inv_t = 1.0 / (double)p.temp, top = p.lse_in[2 * r], rest = p.lse_in[2 * r + 1];
  const float b = p.b != nullptr ? p.b[r] : 0.0f, h = p.b != nullptr ? p.entropy_in[r] : 0.0f;
  double all = 0.0;
  for (int g = 0; g < p.G; ++g)
    if (tokens[g] >= 0 && tokens[g] < p.V) all += (double)a[g];
  for (int i = threadIdx.x; i < p.V; i += kBlock) {
    const float v = widen(x[i]);
    float d = 0.0f;
    if (with_mass(v)) {
      const float lp = (float)(((double)v - top) * inv_t - rest), q = expf(lp);
      d = q > 0.0f ? -q * ((float)all + b * (lp + h)) : 0.0f;
      for (int g = 0; g < p.G; ++g)
        if (tokens[g] == i) d += a[g];
      d *= (float)inv_t;
    }
    out[i] = narrow<E>(d);
  }
}

bool rows_ok(long long R, long long V, long long G, long long M) {
  return R >= 0 && R < (1LL << 24) && V >= 1 && V <= kMaxIndex && G >= 0 && G <= 65535 && M >= 0 && M <= LLC_TOP_MAX;
}

size_t rows_workspace(long long R, long long M, long long chunks) {
  return (size_t)chunks * (size_t)R * (32 + 8 * (size_t)M) + 32 * (size_t)R + 512;
}

}  // namespace
}  // namespace llc

using namespace llc;

extern "C" size_t llc_token_logprobs_workspace_size(int64_t R, int64_t V, int64_t M) {
  return rows_ok(R, V, 0, M) ? rows_workspace(R, M, 1) : 0;
}

extern "C" int llc_token_logprobs(const llc_token_logprobs_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  if (!rows_ok(a->R, a->V, a->G, a->M)) return LLC_E_SHAPE;
  if ((a->flags & ~LLC_FLAG_DRY_RUN) != 0 || a->v_chunks < 0 || a->v_chunks > 64) return LLC_E_OPTION;
  if (a->R == 0) return LLC_OK;
  if (a->x == nullptr || (a->G > 0 && (a->tokens == nullptr || a->logp == nullptr)) ||
      (a->M > 0 && (a->top_ids == nullptr || a->top_logp == nullptr)))
    return LLC_E_NULL;
  if (a->stride_r < 0 || a->tok_stride_r < 0) return LLC_E_SHAPE;
  if (!known_type(a->dtype) || (a->kind != LLC_LOGITS && a->kind != LLC_LOGW)) return LLC_E_DTYPE;
  const bool logits = a->kind == LLC_LOGITS;
  if (logits && !(std::isfinite(a->temp) && a->temp > 0.0f)) return LLC_E_TEMP;
  if (!fits(a->x, type_size(a->dtype)) || !fits(a->tokens, 4)) return LLC_E_ALIGN;
  if (a->workspace == nullptr || !fits(a->workspace, 256) ||
      a->workspace_bytes < rows_workspace(a->R, a->M, a->v_chunks > 1 ? a->v_chunks : 1))
    return LLC_E_WORKSPACE;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  ScoreParams p = {};
  p.R = a->R; p.V = (int)a->V; p.G = (int)a->G; p.M = (int)a->M;
  p.x = a->x; p.stride_r = a->stride_r; p.temp = logits ? a->temp : 1.0f;
  p.tokens = a->tokens; p.tok_stride_r = a->tok_stride_r;
  p.logp = a->logp; p.entropy = a->entropy; p.lse = a->lse; p.top_ids = a->top_ids; p.top_logp = a->top_logp;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    if (a->dtype == LLC_F32) score_kernel<float><<<(unsigned)p.R, kBlock, 0, st>>>(p);
    else score_kernel<uint16_t><<<(unsigned)p.R, kBlock, 0, st>>>(p);
    return hipGetLastError();
  });
}

extern "C" int llc_token_logprobs_grad(const llc_token_logprobs_grad_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  if (!rows_ok(a->R, a->V, a->G, 0)) return LLC_E_SHAPE;
  if ((a->flags & ~LLC_FLAG_DRY_RUN) != 0 || a->v_chunks < 0 || a->v_chunks > 64) return LLC_E_OPTION;
  if (a->R == 0) return LLC_OK;
  if (a->x == nullptr || a->grad == nullptr || (a->G > 0 && (a->tokens == nullptr || a->grad_logp == nullptr)) ||
      (a->lse_in != nullptr && a->grad_entropy != nullptr && a->entropy_in == nullptr))
    return LLC_E_NULL;
  if (a->lse_in != nullptr && (a->logp != nullptr || a->entropy != nullptr || a->lse != nullptr)) return LLC_E_OPTION;
  if (a->stride_r < 0 || a->tok_stride_r < 0 || a->grad_logp_stride_r < 0 || a->grad_stride_r < a->V) return LLC_E_SHAPE;
  if (a->x == a->grad && a->stride_r != a->grad_stride_r) return LLC_E_SHAPE;
  if (!known_type(a->dtype) || (a->kind != LLC_LOGITS && a->kind != LLC_LOGW)) return LLC_E_DTYPE;
  const bool logits = a->kind == LLC_LOGITS;
  if (logits && !(std::isfinite(a->temp) && a->temp > 0.0f)) return LLC_E_TEMP;
  if (!fits(a->x, type_size(a->dtype)) || !fits(a->grad, type_size(a->dtype)) || !fits(a->tokens, 4) || !fits(a->grad_logp, 4))
    return LLC_E_ALIGN;
  if (a->lse_in == nullptr && (a->workspace == nullptr || !fits(a->workspace, 256) ||
      a->workspace_bytes < rows_workspace(a->R, 0, a->v_chunks > 1 ? a->v_chunks : 1)))
    return LLC_E_WORKSPACE;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  ScoreParams p = {};
  p.R = a->R; p.V = (int)a->V; p.G = (int)a->G; p.M = 0;
  p.x = a->x; p.stride_r = a->stride_r; p.temp = logits ? a->temp : 1.0f;
  p.tokens = a->tokens; p.tok_stride_r = a->tok_stride_r;
  p.a = a->grad_logp; p.a_stride_r = a->grad_logp_stride_r; p.b = a->grad_entropy;
  p.grad = a->grad; p.grad_stride_r = a->grad_stride_r;
  p.logp = a->logp;
  p.lse = a->lse != nullptr ? a->lse : (double *)a->workspace;
  p.entropy = a->entropy != nullptr ? a->entropy : (float *)((double *)a->workspace + 2 * a->R);
  p.lse_in = a->lse_in != nullptr ? a->lse_in : p.lse;
  p.entropy_in = a->lse_in != nullptr ? a->entropy_in : p.entropy;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    if (a->lse_in == nullptr) {
      if (a->dtype == LLC_F32) score_kernel<float><<<(unsigned)p.R, kBlock, 0, st>>>(p);
      else score_kernel<uint16_t><<<(unsigned)p.R, kBlock, 0, st>>>(p);
      if (hipGetLastError() != hipSuccess) return hipErrorUnknown;
    }
    if (a->dtype == LLC_F32) score_grad_kernel<float><<<(unsigned)p.R, kBlock, 0, st>>>(p);
    else score_grad_kernel<uint16_t><<<(unsigned)p.R, kBlock, 0, st>>>(p);
    return hipGetLastError();
  });
}
