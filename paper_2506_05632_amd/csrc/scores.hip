// Scores of tokens: their log probability, the rows' entropy and top alternatives, and the gradient of the first two.
//
// Forward.  With a reference m, c = log2(e) / T and d_i = (x_i - m) c, a row needs S = sum 2^d_i and D = sum d_i 2^d_i: ln p_t = (x_t - m) / T - ln S
// and the entropy is ln S - ln 2 D / S.  One pass over the row forms both: a wavefront keeps its largest entry so far as its m, every lane its shares
// of S and D in fp32, scaled over when m grows (which happens a dozen times a row); lanes, wavefronts and chunks are joined in fp64.
// The same pass finds the top alternatives.  An entry is a candidate if it is above a bound that M entries of the row are known to reach: first the
// smallest, over the wavefronts, of the ceil(M / wavefronts) largest of what their lanes' first entries are (each lane's largest of 16), so that a row of 128 256 leaves
// a thousand candidates for fifty, and a tile of 16 entries a lane that has none costs one comparison a lane.  Candidates go to a list of the wavefront's in LDS as
// whole numbers that order as (value, lower index first); a full list is cut to its M largest, which raises the wavefront's bound.  At the end a
// histogram over the numbers' range finds a bound that at most kSelected of them reach, and those are ranked by comparing all with all.
// What bounds it: reading the row (10 issue slots an entry, against 16 that fp32 logits at 6.3 TB/s leave).
#include "ends.hpp"

namespace llc {
namespace {

constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.693147180559945309417232121458;
constexpr int kList = 256;      // candidates of a wavefront in LDS
constexpr int kSelected = 256;  // candidates that are ranked
constexpr int kBins = 1024;
constexpr int kPer = 16;        // entries of a lane and tile
constexpr int kMostSplit = 64;  // workgroups a row is split over

typedef unsigned long long u64;

// What a workgroup knows of a chunk of a row, when a row is split.
struct Share {
  double s, d;    // sum 2^((x - top) c), sum of (x - top) c 2^(...)
  double unused;
  float top;      // largest entry, -inf without mass
  int count;      // keys in the list behind the shares
};

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
  int chunks, chunk;  // workgroups a row is split over, entries of one
  Share *shares;      // [R][chunks]
  u64 *keys;          // [R][chunks][M]
  // the gradient
  const float *a;
  long long a_stride_r;
  const float *b;
  const double *lse_in;
  const float *entropy_in;
  void *grad;
  long long grad_stride_r;
};

__device__ __forceinline__ bool with_mass(float v) { return fabsf(v) < kInf; }
__device__ __forceinline__ uint32_t ordered(float v) {  // larger for larger values; equal for 0 and -0
  const uint32_t b = __float_as_uint(v + 0.0f);
  return (b & 0x80000000u) != 0 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float((o & 0x80000000u) != 0 ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ u64 key_of(float v, uint32_t i) { return ((u64)ordered(v) << 32) | (0xFFFFFFFFu - i); }
__device__ __forceinline__ float key_value(u64 k) { return unordered((uint32_t)(k >> 32)); }
__device__ __forceinline__ int key_index(u64 k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

__device__ __forceinline__ float wave_max(float v) {  // the same in every lane; no NaN among them
#define LLC_STEP(CTRL, ROWS) \
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(v), __float_as_uint(v), CTRL, ROWS, 0xF, false)))
  LLC_STEP(0x111, 0xF); LLC_STEP(0x112, 0xF); LLC_STEP(0x114, 0xF); LLC_STEP(0x118, 0xF);  // row_shr 1, 2, 4, 8
  LLC_STEP(0x142, 0xA); LLC_STEP(0x143, 0xC);                                              // row_bcast 15, 31
#undef LLC_STEP
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
template <int CTRL, int ROWS> __device__ __forceinline__ double from_lane(double v) {  // of the rows that do not take part: 0
  const u64 b = __builtin_bit_cast(u64, v);
  const uint32_t low = __builtin_amdgcn_update_dpp(0, (uint32_t)b, CTRL, ROWS, 0xF, false);
  const uint32_t high = __builtin_amdgcn_update_dpp(0, (uint32_t)(b >> 32), CTRL, ROWS, 0xF, false);
  return __builtin_bit_cast(double, ((u64)high << 32) | low);
}
__device__ __forceinline__ double wave_sum(double v) {  // the same in every lane
  v += from_lane<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
  v += from_lane<0x112, 0xF>(v);
  v += from_lane<0x114, 0xF>(v);
  v += from_lane<0x118, 0xF>(v);
  v += from_lane<0x142, 0xA>(v);  // row_bcast 15, 31
  v += from_lane<0x143, 0xC>(v);
  const u64 b = __builtin_bit_cast(u64, v);
  return __builtin_bit_cast(double, ((u64)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(b >> 32), 63) << 32) |
                                        (uint32_t)__builtin_amdgcn_readlane((uint32_t)b, 63));
}
__device__ __forceinline__ int lanes_below(u64 mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
__device__ __forceinline__ float max3(float a, float b, float c) {  // (NaN only if all are, or where one is a signalling one)
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// kPer entries of a lane: 16 bytes at a time, 64 lanes side by side.  `left`: entries from the lane's first on; what lies beyond is -inf.
template <typename E> __device__ __forceinline__ void load_tile(const E *x, long long left, float (&v)[kPer]) {
  constexpr int N = kWide<E>;
#pragma unroll
  for (int u = 0; u < kPer / N; ++u) {
    float w[N];
    fetch_some<N>(x + u * 64 * N, w);
#pragma unroll
    for (int i = 0; i < N; ++i) v[u * N + i] = w[i];
  }
}
template <typename E> __device__ __forceinline__ void load_tile_end(const E *x, long long left, float (&v)[kPer]) {
  constexpr int N = kWide<E>;
#pragma unroll
  for (int u = 0; u < kPer / N; ++u)
#pragma unroll
    for (int i = 0; i < N; ++i) v[u * N + i] = u * 64 * N + i < left ? widen(x[u * 64 * N + i]) : -kInf;
}

// A wavefront's sums and candidates.
template <typename E> struct Scan {
  float m = -kInf;      // largest entry so far
  float s = 0.0f, d = 0.0f;
  float bound = -kInf;  // candidates are above it
  int count = 0;        // of the list
};

// The list's M largest stay.
__device__ __forceinline__ u64 cut_list(u64 *list, int &count, int M) {
  const int lane = threadIdx.x & 63;
  u64 k[kList / 64];
#pragma unroll
  for (int i = 0; i < kList / 64; ++i) k[i] = i * 64 + lane < count ? list[i * 64 + lane] : 0;
  u64 t = 0;  // the M-th largest, bit by bit
  for (int bit = 63; bit >= 0; --bit) {
    const u64 with = t | (1ull << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < kList / 64; ++i) n += (int)__builtin_popcountll(__ballot(k[i] >= with));
    if (n >= M) t = with;
  }
  count = 0;
#pragma unroll
  for (int i = 0; i < kList / 64; ++i) {
    const bool stays = k[i] >= t && k[i] != 0;
    const u64 mask = __ballot(stays);
    if (stays) list[count + lanes_below(mask)] = k[i];
    count += (int)__builtin_popcountll(mask);
  }
  return t;
}

// One tile: `first` is the index in the row of the lane's first entry.
template <typename E> __device__ __forceinline__ void take_tile(Scan<E> &w, float (&v)[kPer], uint32_t first, float c, int M, u64 *list) {
  constexpr int N = kWide<E>;
  float half[2];  // the largest of either half of the entries
  const auto largest = [&] {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float *o = v + h * (kPer / 2);
      half[h] = max3(max3(o[0], o[1], o[2]), max3(o[3], o[4], o[5]), max3(o[6], o[7], o[7]));
    }
    return max3(half[0], half[1], half[1]);
  };
  float t = largest();
  if (__ballot(!(t <= w.bound)) != 0) {  // (a NaN comes here too)
    if (__ballot(!(t < kInf)) != 0) {    // entries without mass
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = with_mass(v[i]) ? v[i] : -kInf;
      t = largest();
    }
    if (__ballot(t > w.m) != 0) {
      const float m = wave_max(t), by = fmaxf((w.m - m) * c, -200.0f), scale = __builtin_amdgcn_exp2f(by);
      w.d = (w.d + w.s * by) * scale;
      w.s *= scale;
      w.m = m;
      if (M == 0) w.bound = m;
    }
    if (M > 0) {
      u64 lanes = __ballot(t > w.bound);
      int most = kPer * (int)__builtin_popcountll(lanes);
      if (w.count + most > kList) {
        most = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) most += (int)__builtin_popcountll(__ballot(v[i] > w.bound));
      }
      if (w.count + most <= kList) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (__ballot(half[h] > w.bound) == 0) continue;
#pragma unroll
          for (int i = h * (kPer / 2); i < (h + 1) * (kPer / 2); ++i) {
            const u64 mask = __ballot(v[i] > w.bound);
            if (mask == 0) continue;
            if (v[i] > w.bound) list[w.count + lanes_below(mask)] = key_of(v[i], first + (i / N) * 64 * N + i % N);
            w.count += (int)__builtin_popcountll(mask);
          }
        }
      } else {  // as many as may not fit: a lane's at a time, and the list is cut where it is full
        const int lane = threadIdx.x & 63;
        u64 least = 0;
        for (; lanes != 0; lanes &= lanes - 1) {
          const int from = __builtin_ctzll(lanes);
          float mine = -kInf;
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v[i]), from));
            if (lane == i) mine = o;
          }
          if (w.count + kPer > kList) least = cut_list(list, w.count, M);
          const u64 key = key_of(mine, __builtin_amdgcn_readlane(first, from) + (lane / N) * 64 * N + lane % N);
          const bool offered = mine > w.bound && key > least;
          const u64 mask = __ballot(offered);
          if (offered) list[w.count + lanes_below(mask)] = key;
          w.count += (int)__builtin_popcountll(mask);
        }
        if (least != 0) w.bound = fmaxf(w.bound, key_value(least));  // (what equals the least kept one comes after it in a later tile)
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const float d = fmaxf((v[i] - w.m) * c, -200.0f), e = __builtin_amdgcn_exp2f(d);  // (no mass: 2^-200 is 0)
    w.s += e;
    w.d = fmaf(e, d, w.d);
  }
}

// A number that n of the lanes' K ordered values each reach, and little below the n-th largest of them (its upper 16 bits); 0 if there are fewer than n.
template <int K> __device__ __forceinline__ uint32_t reached_by(const uint32_t (&o)[K], int n) {
  uint32_t t = 0;
#pragma unroll 4
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t with = t | (1u << bit);
    int reach = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) reach += (int)__builtin_popcountll(__ballot(o[i] >= with));
    if (reach >= n) t = with;
  }
  return t;
}
// What all wavefronts have said so far.
__device__ __forceinline__ uint32_t least_said(const uint32_t *said, int waves) {
  const int lane = threadIdx.x & 63;
  uint32_t v = 0xFFFFFFFFu;
  if (lane < waves) v = *(const volatile uint32_t *)&said[lane];
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(v, v, 0x111, 0xF, 0xF, false));
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(v, v, 0x112, 0xF, 0xF, false));
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(v, v, 0x114, 0xF, 0xF, false));
  v = min(v, (uint32_t)__builtin_amdgcn_update_dpp(v, v, 0x118, 0xF, 0xF, false));
  return __builtin_amdgcn_readlane(v, 15);  // (at most 16 wavefronts)
}

// The largest bound that lets through whatever orders as `o` or more.
__device__ __forceinline__ float just_below(uint32_t o) {
  return o > ordered(-kInf) ? unordered(o - (o == ordered(0.0f) ? 2 : 1)) : -kInf;  // (below 0 comes -0, its equal)
}

// A wavefront looks at its list: it says what `share` of its entries reach and, told what M of the row's entries reach then, drops the others.
// K: 64ths of the list that are in use.
template <int K> __device__ __forceinline__ float look_at_list(u64 *list, int &count, int share, uint32_t *said, int waves, int wave) {
  const int lane = threadIdx.x & 63;
  u64 k[K];
  uint32_t o[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    k[i] = i * 64 + lane < count ? list[i * 64 + lane] : 0;
    o[i] = (uint32_t)(k[i] >> 32);
  }
  const uint32_t nth = reached_by(o, share);
  if (lane == 0) said[wave] = nth;
  const uint32_t all = least_said(said, waves);
  count = 0;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const bool stays = k[i] != 0 && o[i] >= all;
    const u64 mask = __ballot(stays);
    if (stays) list[count + lanes_below(mask)] = k[i];
    count += (int)__builtin_popcountll(mask);
  }
  return just_below(all);
}

// The M largest of the lists' keys in order: emit(rank, key), key 0 where there are fewer.  Lists of `stride` keys, list i of count[i].
template <int THREADS, typename F>
__device__ __forceinline__ void select_top(const u64 *lists, int n_lists, int stride, const int *count, u64 low, u64 high, int M, F emit) {
  __shared__ int s_bins[kBins];
  __shared__ u64 s_keys[kSelected];
  __shared__ int s_wave[THREADS / 64], s_bin, s_above, s_n;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  u64 least = low;  // (M keys or all reach it)
  if (tid == 0) s_n = 0;
  __syncthreads();
  // those go to a list of their own, unless they are too many
  const auto gather = [&] {
    for (int l = wave; l < n_lists; l += THREADS / 64)
      for (int i0 = 0; i0 < count[l]; i0 += 64) {
        const u64 k = i0 + lane < count[l] ? lists[(size_t)l * stride + i0 + lane] : 0;
        const bool in = k >= least && k != 0;
        const u64 mask = __ballot(in);
        if (mask == 0) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&s_n, (int)__builtin_popcountll(mask));
        at = __builtin_amdgcn_readfirstlane(at) + lanes_below(mask);
        if (in && at < kSelected) s_keys[at] = k;
      }
  };
  gather();
  __syncthreads();
  if (s_n > kSelected) {
    int need = M, above = 0;  // `above` keys are larger than `high`
    for (;;) {
      const u64 range = high - low;
      const int bits = range == 0 ? 0 : 64 - __builtin_clzll(range), shift = bits > 10 ? bits - 10 : 0;
      for (int i = tid; i < kBins; i += THREADS) s_bins[i] = 0;
      __syncthreads();
      for (int l = wave; l < n_lists; l += THREADS / 64)
        for (int i = lane; i < count[l]; i += 64) {
          const u64 k = lists[(size_t)l * stride + i];
          if (k >= low && k <= high) atomicAdd(&s_bins[(k - low) >> shift], 1);
        }
      __syncthreads();
      // a thread takes kBins / THREADS bins, the first thread the uppermost
      constexpr int kEach = kBins / THREADS;
      int mine = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) mine += s_bins[kBins - 1 - (tid * kEach + i)];
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
      }
      if (lane == 63) s_wave[wave] = upto;
      __syncthreads();
      for (int w = 0; w < wave; ++w) upto += s_wave[w];
      if (upto >= need && upto - mine < need) {  // (one thread)
        int n = upto - mine;
        for (int i = 0; i < kEach; ++i) {
          const int bin = kBins - 1 - (tid * kEach + i), here = s_bins[bin];
          if (n + here >= need) { s_bin = bin; s_above = n; s_n = n + here; break; }
          n += here;
        }
      }
      __syncthreads();
      least = low + ((u64)s_bin << shift);
      if (above + s_n <= kSelected || shift == 0) break;
      high = least + ((1ull << shift) - 1);
      low = least;
      need -= s_above;
      above += s_above;
      __syncthreads();
    }
    __syncthreads();
    if (tid == 0) s_n = 0;
    __syncthreads();
    gather();
    __syncthreads();
  }
  const int n = s_n;
  for (int i = tid; i < n; i += THREADS) {
    const u64 k = s_keys[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += s_keys[j] > k ? 1 : 0;
    if (rank < M) emit(rank, k);
  }
  for (int m = n + tid; m < M; m += THREADS) emit(m, (u64)0);
}

// What a row's sums give, the same in every thread.
struct Row {
  double top, rest, entropy, inv_t;
  __device__ __forceinline__ float logp(float v) const { return with_mass(v) ? (float)(((double)v - top) * inv_t - rest) : -kInf; }
};
__device__ __forceinline__ Row row_of(float top, double s, double d, float temp) {
  Row r;
  const bool any = top > -kInf;
  r.top = any ? (double)top : 0.0;
  r.rest = any ? log(s) : -(double)kInf;
  r.entropy = any ? r.rest - kLn2 * d / s : 0.0;
  r.inv_t = 1.0 / (double)temp;
  return r;
}
template <typename E> __device__ __forceinline__ void write_scores(const ScoreParams &p, long long r, const Row &row, int from, int threads) {
  if (threadIdx.x == 0) {
    if (p.lse != nullptr) { p.lse[2 * r] = row.top; p.lse[2 * r + 1] = row.rest; }
    if (p.entropy != nullptr) p.entropy[r] = (float)row.entropy;
  }
  if (p.logp == nullptr) return;
  const E *x = reinterpret_cast<const E *>(p.x) + r * p.stride_r;
  for (int g = from + threadIdx.x; g < p.G; g += threads) {
    const int t = p.tokens[r * p.tok_stride_r + g];
    p.logp[r * p.G + g] = t < 0 ? 0.0f : t < p.V ? row.logp(widen(x[t])) : -kInf;
  }
}
__device__ __forceinline__ void write_top(const ScoreParams &p, long long r, const Row &row, int rank, u64 key) {
  p.top_ids[r * p.M + rank] = key != 0 ? key_index(key) : -1;
  p.top_logp[r * p.M + rank] = key != 0 ? row.logp(key_value(key)) : -kInf;
}

// Sums that the lanes hold, each relative to its own largest entry, as one relative to the largest of all.
__device__ __forceinline__ void join_shares(double &s, double &d, float mine, float top, float c) {
  const double by = mine > -kInf ? (double)fmaxf((mine - top) * c, -200.0f) : -200.0, scale = (double)__builtin_amdgcn_exp2f((float)by);  // (off by 2^-23 of a wavefront's share)
  d = wave_sum((d + s * by) * scale);
  s = wave_sum(s * scale);
}

// One workgroup a row, or a chunk of it.
template <typename E, int WAVES> __global__ void __launch_bounds__(WAVES * 64) score_kernel(const ScoreParams p) {
  constexpr int N = kWide<E>, kTile = 64 * kPer;
  __shared__ u64 s_list[WAVES * kList];
  __shared__ double s_s[WAVES], s_d[WAVES];
  __shared__ float s_m[WAVES];
  __shared__ int s_count[WAVES];
  __shared__ uint32_t s_nth[WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long r = p.chunks > 1 ? blockIdx.x / p.chunks : blockIdx.x;
  const int part = p.chunks > 1 ? (int)(blockIdx.x - r * p.chunks) : 0;
  const long long begin = (long long)part * p.chunk, end = begin + p.chunk < p.V ? begin + p.chunk : p.V;
  const E *x = reinterpret_cast<const E *>(p.x) + r * p.stride_r;
  const float c = kLog2e / p.temp;
  u64 *list = s_list + wave * kList;
  Scan<E> w;
  float v[kPer], next[kPer];
  long long at = begin + (long long)wave * kTile;
  const auto load = [&](long long from, float (&to)[kPer]) {
    if (from + kTile <= end) load_tile(x + from + lane * N, 0, to);
    else load_tile_end(x + from + lane * N, end - from - lane * N, to);
  };
  if (at < end) load(at, v);
  if (at + (long long)WAVES * kTile < end) load(at + (long long)WAVES * kTile, next);
  // tokens and their entries are on their way too
  int token = -1;
  float token_x = 0.0f;
  if (p.chunks == 1 && (int)threadIdx.x < p.G) {
    token = p.tokens[r * p.tok_stride_r + threadIdx.x];
    if (token >= 0 && token < p.V) token_x = widen(x[token]);
  }
  // A bound that M entries reach: every wavefront's share of them is among what it has seen.  First each lane's largest of the first tile; later,
  // whenever a wavefront has seen twice as much, the candidates in its list.  What a wavefront has once said stays true, so nobody waits.
  const int share = (p.M + WAVES - 1) / WAVES;
  if (p.M > 0) {
    float t = -kInf;
    if (at < end) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) t = fmaxf(t, with_mass(v[i]) ? v[i] : -kInf);
    }
    const uint32_t o[1] = {ordered(t)}, nth = share <= 64 ? reached_by(o, share) : 0;
    if (lane == 0) s_nth[wave] = nth;
    __syncthreads();
    w.bound = just_below(least_said(s_nth, WAVES));
  }
  const auto look = [&] {
    if (w.count < share) return;
    w.bound = fmaxf(w.bound, w.count <= 64 ? look_at_list<1>(list, w.count, share, s_nth, WAVES, wave)
                                           : look_at_list<kList / 64>(list, w.count, share, s_nth, WAVES, wave));
  };
  // two tiles in turn, so that one is on its way while the other is taken
  const long long step = (long long)WAVES * kTile;
  for (int tiles = 1; at < end; tiles += 2, at += 2 * step) {
    take_tile<E>(w, v, (uint32_t)(at + lane * N), c, p.M, list);
    if (at + 2 * step < end) load(at + 2 * step, v);
    if (p.M > 0 && (tiles & (tiles - 1)) == 0) look();
    if (at + step >= end) break;
    take_tile<E>(w, next, (uint32_t)(at + step + lane * N), c, p.M, list);
    if (at + 3 * step < end) load(at + 3 * step, next);
    if (p.M > 0 && (tiles & (tiles + 1)) == 0) look();
  }
  if (p.M > 0) look();
  // the wavefronts' sums
  const double ws = wave_sum((double)w.s), wd = wave_sum((double)w.d);
  if (lane == 0) { s_s[wave] = ws; s_d[wave] = wd; s_m[wave] = w.m; s_count[wave] = w.count; }
  __syncthreads();
  const int mine = lane < WAVES ? lane : 0;
  const float my_top = lane < WAVES ? s_m[mine] : -kInf, top = wave_max(my_top);
  double s = lane < WAVES ? s_s[mine] : 0.0, d = lane < WAVES ? s_d[mine] : 0.0;
  join_shares(s, d, my_top, top, c);
  int total = 0;
  for (int i = 0; i < WAVES; ++i) total += s_count[i];
  const u64 high = key_of(top > -kInf ? top : 0.0f, 0);
  u64 least = 1;
  if (p.M > 0) { const uint32_t said = least_said(s_nth, WAVES); least = (u64)(said > 0 ? said : 1) << 32; }
  if (p.chunks > 1) {
    u64 *keys = p.keys + (r * p.chunks + part) * p.M;
    if (threadIdx.x == 0) p.shares[r * p.chunks + part] = Share{s, d, 0.0, top, total < p.M ? total : p.M};
    if (p.M > 0) select_top<WAVES * 64>(s_list, WAVES, kList, s_count, least, high, p.M, [&](int rank, u64 key) { keys[rank] = key; });
    return;
  }
  const Row row = row_of(top, s, d, p.temp);
  if ((int)threadIdx.x < p.G && p.logp != nullptr) p.logp[r * p.G + threadIdx.x] = token < 0 ? 0.0f : token < p.V ? row.logp(token_x) : -kInf;
  write_scores<E>(p, r, row, WAVES * 64, WAVES * 64);
  if (p.M > 0) select_top<WAVES * 64>(s_list, WAVES, kList, s_count, least, high, p.M, [&](int rank, u64 key) { write_top(p, r, row, rank, key); });
}

// Joins a row's chunks.
template <typename E> __global__ void __launch_bounds__(kBlock) score_join_kernel(const ScoreParams p) {
  __shared__ int s_count[kMostSplit];
  const long long r = blockIdx.x;
  const Share *shares = p.shares + r * p.chunks;
  const float c = kLog2e / p.temp;
  const int lane = threadIdx.x & 63;
  Share share = {0.0, 0.0, 0.0, -kInf, 0};
  if (lane < p.chunks) share = shares[lane];
  const float top = wave_max(share.top);
  int total = share.count;
#pragma unroll
  for (int i = 32; i >= 1; i >>= 1) total += __shfl_xor(total, i);
  double s = share.s, d = share.d;
  join_shares(s, d, share.top, top, c);
  const Row row = row_of(top, s, d, p.temp);
  write_scores<E>(p, r, row, 0, kBlock);
  if (p.M == 0) return;
  if ((int)threadIdx.x < p.chunks) s_count[threadIdx.x] = share.count;
  __syncthreads();
  select_top<kBlock>(p.keys + r * p.chunks * p.M, p.chunks, p.M, s_count, 1, key_of(top > -kInf ? top : 0.0f, 0), p.M,
                     [&](int rank, u64 key) { write_top(p, r, row, rank, key); });
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

constexpr long long kMostGrid = 0xFFFFFFFFLL / kBlock;  // workgroups of a launch (those of 1024 threads: launches of fewer than 1024)

bool rows_ok(long long R, long long V, long long G, long long M) {
  return R >= 0 && R <= kMostGrid && V >= 1 && V <= kMaxIndex && G >= 0 && G <= 65535 && M >= 0 && M <= LLC_TOP_MAX;
}

static_assert(sizeof(Share) == 32, "what the interface states of the workspace");
size_t rows_workspace(long long R, long long M, long long chunks) {  // shares and keys, then (gradient) lse and entropy
  return (size_t)chunks * (size_t)R * (sizeof(Share) + 8 * (size_t)M) + 32 * (size_t)R + 512;
}

// Workgroups that a row is split over.
#ifndef SPLIT
#define SPLIT 1
#endif
int auto_split(long long R, long long V) { return SPLIT; }

// Cuts a row into `want` chunks of whole 16-byte loads.
void split_rows(ScoreParams &p, long long want) {
  const long long each = ((p.V + want - 1) / want + 15) & ~15LL;
  p.chunk = (int)(each < kMaxIndex ? each : kMaxIndex);
  p.chunks = (int)((p.V + each - 1) / each);
}

template <typename E> hipError_t launch_scores(const ScoreParams &p, hipStream_t st) {
  const unsigned blocks = (unsigned)(p.R * p.chunks);
  const long long tiles = (p.chunk + 64 * kPer - 1) / (64 * kPer);
#ifdef NW
  score_kernel<E, NW><<<blocks, NW * 64, 0, st>>>(p);
#else
  if (tiles <= 1) score_kernel<E, 1><<<blocks, 64, 0, st>>>(p);
  else if (tiles <= 4 || blocks > 512) score_kernel<E, 4><<<blocks, 256, 0, st>>>(p);
  else if (blocks > 256) score_kernel<E, 8><<<blocks, 512, 0, st>>>(p);
  else score_kernel<E, 16><<<blocks, 1024, 0, st>>>(p);
#endif
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.chunks == 1) return e;
  score_join_kernel<E><<<(unsigned)p.R, kBlock, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace
}  // namespace llc

using namespace llc;

extern "C" size_t llc_token_logprobs_workspace_size(int64_t R, int64_t V, int64_t M) {
  return rows_ok(R, V, 0, M) ? rows_workspace(R, M, auto_split(R, V)) : 0;
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
  const long long split = a->v_chunks > 0 ? a->v_chunks : auto_split(a->R, a->V);
  if (a->workspace == nullptr || !fits(a->workspace, 256) || a->workspace_bytes < rows_workspace(a->R, a->M, split)) return LLC_E_WORKSPACE;
  if (a->R * split > kMostGrid) return LLC_E_SHAPE;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  ScoreParams p = {};
  p.R = a->R; p.V = (int)a->V; p.G = (int)a->G; p.M = (int)a->M;
  p.x = a->x; p.stride_r = a->stride_r; p.temp = logits ? a->temp : 1.0f;
  p.tokens = a->tokens; p.tok_stride_r = a->tok_stride_r;
  p.logp = a->logp; p.entropy = a->entropy; p.lse = a->lse; p.top_ids = a->top_ids; p.top_logp = a->top_logp;
  split_rows(p, split);
  p.shares = (Share *)a->workspace; p.keys = (u64 *)(p.shares + p.R * p.chunks);
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] { return a->dtype == LLC_F32 ? launch_scores<float>(p, st) : launch_scores<uint16_t>(p, st); });
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
  const long long split = a->v_chunks > 0 ? a->v_chunks : auto_split(a->R, a->V);
  if (a->lse_in == nullptr && (a->workspace == nullptr || !fits(a->workspace, 256) || a->workspace_bytes < rows_workspace(a->R, 0, split)))
    return LLC_E_WORKSPACE;
  if (a->R * split > kMostGrid) return LLC_E_SHAPE;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  ScoreParams p = {};
  p.R = a->R; p.V = (int)a->V; p.G = (int)a->G; p.M = 0;
  p.x = a->x; p.stride_r = a->stride_r; p.temp = logits ? a->temp : 1.0f;
  p.tokens = a->tokens; p.tok_stride_r = a->tok_stride_r;
  p.a = a->grad_logp; p.a_stride_r = a->grad_logp_stride_r; p.b = a->grad_entropy;
  p.grad = a->grad; p.grad_stride_r = a->grad_stride_r;
  p.logp = a->logp;
  split_rows(p, split);
  p.shares = (Share *)a->workspace;
  double *kept = (double *)(p.shares + p.R * p.chunks);
  p.lse = a->lse != nullptr ? a->lse : kept;
  p.entropy = a->entropy != nullptr ? a->entropy : (float *)(kept + 2 * a->R);
  p.lse_in = a->lse_in != nullptr ? a->lse_in : p.lse;
  p.entropy_in = a->lse_in != nullptr ? a->entropy_in : p.entropy;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    if (a->lse_in == nullptr) {
      const hipError_t e = a->dtype == LLC_F32 ? launch_scores<float>(p, st) : launch_scores<uint16_t>(p, st);
      if (e != hipSuccess) return e;
    }
    if (a->dtype == LLC_F32) score_grad_kernel<float><<<(unsigned)p.R, kBlock, 0, st>>>(p);
    else score_grad_kernel<uint16_t><<<(unsigned)p.R, kBlock, 0, st>>>(p);
    return hipGetLastError();
  });
}
