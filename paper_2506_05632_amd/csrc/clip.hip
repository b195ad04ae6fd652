// The global norm over many tensors, and clipping by it: memory bounds both, at two operations an entry.  Tensors go to a
// launch a table at a time; the table is a kernel argument, so nothing is copied to the device.  All tensors of a table are cut into pieces of
// 16 KB, which workgroups take whatever tensor they belong to: small tensors cost no launches and large ones no imbalance.
// Squares and their sums are fp64: exact but for the sums' rounding, and none is lost or infinite.  (In fp32 over a thread's share of a piece, with fp64 only where that
// leaves its range: 519.0 us for 520.4 of the half billion below.)  Which piece a workgroup takes and the order in which partial sums are joined follow
// from the sizes alone.
// 534 M entries in 219 tensors, bf16 but for norms' gains, into other buffers: 0.52 ms, 6.2 TB/s of the 3.2 GB read, read again and written.  Small
// lists: the host's call and two launches that wait for each other (21 tensors 11.8 us).
#include "ends.hpp"

namespace llc {
namespace {

constexpr int kTable = 140;         // tensors a launch (a launch's arguments are 4 KB at most)
constexpr int kVectors = 4;         // 16-byte loads of a thread and piece
constexpr int kPiece = kBlock * kVectors * 16;  // bytes
// Workgroups of a table's first pass, and its partial sums, at most.  (1024: 16 x 1 M fp32 29.3 us, 4096: 28.2, so 27.2; 16 x 4 M 86.3, 83.0, 82.9.)
constexpr int kSquareBlocks = 2048;
// Up to so many every workgroup of the second pass joins them itself, which spares a launch.  us a call with that launch and without: 10 x 262 144 fp32
// 12.1, 11.5; 20 x 200 000 12.2, 11.6; beyond: 16 x 1 M 26.8, 30.1; 100 x 2 M 242, 274.
constexpr int kFewPartials = 1024;
constexpr unsigned kScaleBlocks = 1u << 22;
constexpr long long kBf16 = 1LL << 62;

struct ClipParams {
  const void *from[kTable];
  void *to[kTable];
  long long numel[kTable];    // with kBf16 set for that type
  uint32_t first[kTable];     // the number of a tensor's first piece
  int n;
  uint32_t pieces;
  double *partials;   // this table's (first pass), all tables' (second)
  int n_partials;     // 0: `factor` is there
  float max_norm;
  float *factor;      // in the workspace
  float *norm;        // written by the second pass's first launch if it joins the partial sums
};

// The piece's tensor: the last whose first piece does not come after it (empty ones share theirs with the next).
__device__ __forceinline__ int tensor_of(const ClipParams &p, uint32_t piece) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int i = 0; i < kTable; i += 64) n += (int)__builtin_popcountll(__ballot(i + lane < p.n && p.first[i + lane < kTable ? i + lane : 0] <= piece));
  return n - 1;
}

__device__ double sum_over_workgroup(double v) {
  __shared__ double s[kBlock / 64];
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// A thread's vectors of a piece: vector i starts at entry (i * kBlock + thread) * kWide of the piece.
template <typename E> __device__ __forceinline__ double squares_of(const E *from, long long left) {
  constexpr int N = kWide<E>;
  float v[kVectors][N];
  const E *at = from + threadIdx.x * N;
  if (left >= (long long)kBlock * kVectors * N) {
#pragma unroll
    for (int i = 0; i < kVectors; ++i) load_some<N>(at + i * kBlock * N, v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kVectors; ++i) load_first<N>(at + i * kBlock * N, left - (i * kBlock + (int)threadIdx.x) * N, v[i]);
  }
  double d[2] = {};
#pragma unroll
  for (int i = 0; i < kVectors; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) { const double w = (double)v[i][j]; d[j & 1] = fma(w, w, d[j & 1]); }
  return d[0] + d[1];
}

__global__ void __launch_bounds__(kBlock) square_kernel(const ClipParams p) {
  double s = 0.0;
  for (uint32_t piece = blockIdx.x; piece < p.pieces; piece += gridDim.x) {
    const int j = __builtin_amdgcn_readfirstlane(tensor_of(p, piece));
    const long long numel = p.numel[j], offset = (long long)(piece - p.first[j]) * kPiece;
    if ((numel & kBf16) != 0) s += squares_of(reinterpret_cast<const uint16_t *>(p.from[j]) + offset / 2, (numel & ~kBf16) - offset / 2);
    else s += squares_of(reinterpret_cast<const float *>(p.from[j]) + offset / 4, numel - offset / 4);
  }
  s = sum_over_workgroup(s);
  if (threadIdx.x == 0) p.partials[blockIdx.x] = s;
}

__device__ __forceinline__ double sum_of_partials(const double *partials, int n, int from, int step) {
  double s = 0.0;
  for (int i = from; i < n; i += step) s += partials[i];
  return s;
}
__device__ __forceinline__ float factor_of(double norm, float max_norm) {  // (the norm as the caller sees it says whether it is finite)
  return norm > (double)max_norm && (float)norm < __builtin_huge_valf() ? (float)((double)max_norm / norm) : 1.0f;
}

// Many partial sums are joined once.
__global__ void __launch_bounds__(kBlock) norm_kernel(const double *partials, int n, float max_norm, float *factor, float *norm_out) {
  double s[8] = {};
  int i = threadIdx.x;
  for (; i + 7 * kBlock < n; i += 8 * kBlock)
#pragma unroll
    for (int u = 0; u < 8; ++u) s[u] += partials[i + u * kBlock];
  s[0] += sum_of_partials(partials, n, i, kBlock);
  const double norm = sqrt(sum_over_workgroup(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]))));
  if (threadIdx.x == 0) {
    *norm_out = (float)norm;
    *factor = factor_of(norm, max_norm);
  }
}

// A whole piece in a thread's registers, and what is left to do with it once the factor is known.
struct Piece {
  word4_any w[kVectors];
};
__device__ __forceinline__ Piece fetch_piece(const char *from) {
  Piece v;
#pragma unroll
  for (int i = 0; i < kVectors; ++i)
    v.w[i] = __builtin_nontemporal_load(reinterpret_cast<const word4_any *>(from + (i * kBlock + (int)threadIdx.x) * 16));
  return v;
}
__device__ __forceinline__ void scale_whole(const Piece &v, char *to, bool bf16, float factor) {
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    word4_any w = v.w[i];
    if (factor != 1.0f) {  // (a NaN among gradients that are only copied keeps its bits)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float a, b;
        split_pair(w[j], a, b);
        w[j] = bf16 ? narrow_pair(a * factor, b * factor) : __float_as_uint(__uint_as_float(w[j]) * factor);
      }
    }
    __builtin_nontemporal_store(w, reinterpret_cast<word4_any *>(to + (i * kBlock + (int)threadIdx.x) * 16));
  }
}
template <typename E> __device__ __forceinline__ void scale_rest(const E *from, E *to, long long left, float factor) {
  for (int i = threadIdx.x; i < left; i += kBlock) to[i] = factor != 1.0f ? narrow<E>(widen(from[i]) * factor) : from[i];
}

__global__ void __launch_bounds__(kBlock) clip_kernel(const ClipParams p) {
  // (backwards: what the first pass has read last may still be in the caches)
  uint32_t piece = p.pieces - 1 - blockIdx.x;
  int j = __builtin_amdgcn_readfirstlane(tensor_of(p, piece));
  const auto bytes_left = [&] {  // of tensor j from the piece on
    const long long numel = p.numel[j];
    return (numel & ~kBf16) * ((numel & kBf16) != 0 ? 2 : 4) - (long long)(piece - p.first[j]) * kPiece;
  };
  const auto start = [&](const void *tensor) { return reinterpret_cast<const char *>(tensor) + (long long)(piece - p.first[j]) * kPiece; };
  const auto form = [&] {
    if (p.n_partials == 0) return *p.factor;
    const double norm = sqrt(sum_over_workgroup(sum_of_partials(p.partials, p.n_partials, threadIdx.x, kBlock)));
    if (p.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = (float)norm;
    return factor_of(norm, p.max_norm);
  };
  const auto rest = [&](float factor) {
    if (factor == 1.0f && p.from[j] == p.to[j]) return;
    char *to = const_cast<char *>(start(p.to[j]));
    if ((p.numel[j] & kBf16) != 0) scale_rest((const uint16_t *)start(p.from[j]), (uint16_t *)to, bytes_left() / 2, factor);
    else scale_rest((const float *)start(p.from[j]), (float *)to, bytes_left() / 4, factor);
  };
  const auto whole = [&](const Piece &v, float factor) {
    if (factor != 1.0f || p.from[j] != p.to[j]) scale_whole(v, const_cast<char *>(start(p.to[j])), (p.numel[j] & kBf16) != 0, factor);
  };
  // The first piece is on its way while the factor is formed.  (On a way of its own: a load under a condition is waited for where the ways meet.)
  float factor;
  if (bytes_left() >= kPiece) {
    const Piece v = fetch_piece(start(p.from[j]));
    factor = form();
    whole(v, factor);
  } else {
    factor = form();
    rest(factor);
  }
  while (piece >= gridDim.x) {
    piece -= gridDim.x;
    j = __builtin_amdgcn_readfirstlane(tensor_of(p, piece));
    if (bytes_left() >= kPiece) whole(fetch_piece(start(p.from[j])), factor);
    else rest(factor);
  }
}

}  // namespace
}  // namespace llc

using namespace llc;

extern "C" size_t llc_clip_grad_norm_workspace_size(int64_t n) {
  if (n < 0 || n > (1 << 20)) return 0;
  return 256 + (size_t)((n + kTable - 1) / kTable) * kSquareBlocks * sizeof(double);  // the factor, then the partial sums
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
    const int tables = (int)((a->n + kTable - 1) / kTable);
    ClipParams p;
    p.factor = (float *)a->workspace;
    p.max_norm = a->max_norm;
    double *partials = (double *)((char *)a->workspace + 256);
    const auto fill = [&](int t) {
      const int64_t j0 = (int64_t)t * kTable;
      p.n = (int)(a->n - j0 < kTable ? a->n - j0 : kTable);
      long long pieces = 0;
      for (int j = 0; j < p.n; ++j) {
        const int64_t numel = a->numel[j0 + j];
        p.from[j] = a->grads[j0 + j];
        p.to[j] = a->out != nullptr ? a->out[j0 + j] : a->grads[j0 + j];
        p.numel[j] = numel | (a->dtype[j0 + j] == LLC_BF16 ? kBf16 : 0);
        p.first[j] = (uint32_t)pieces;
        pieces += (numel * (int64_t)type_size(a->dtype[j0 + j]) + kPiece - 1) / kPiece;  // (below 2^28 in all)
      }
      p.pieces = (uint32_t)pieces;
    };
    int n_partials = 0;
    for (int t = 0; t < tables; ++t) {
      fill(t);
      if (p.pieces == 0) continue;
      const int blocks = p.pieces < (uint32_t)kSquareBlocks ? (int)p.pieces : kSquareBlocks;
      p.partials = partials + n_partials;
      n_partials += blocks;
      square_kernel<<<blocks, kBlock, 0, st>>>(p);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    const bool scale = a->out != nullptr || a->max_norm < __builtin_huge_valf();  // (else the norm alone)
    const bool few = n_partials > 0 && n_partials <= kFewPartials && scale;
    if (!few) {
      norm_kernel<<<1, kBlock, 0, st>>>(partials, n_partials, a->max_norm, p.factor, a->norm);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    p.partials = partials;
    p.n_partials = few ? n_partials : 0;
    p.norm = few ? a->norm : nullptr;
    for (int t = tables - 1; scale && t >= 0; --t) {
      if (tables > 1) fill(t);
      if (p.pieces == 0) continue;
      clip_kernel<<<p.pieces < kScaleBlocks ? p.pieces : kScaleBlocks, kBlock, 0, st>>>(p);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      p.norm = nullptr;
    }
    return hipSuccess;
  });
}
