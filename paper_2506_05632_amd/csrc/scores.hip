// Scores of tokens: their log probability, the rows' entropy and top alternatives, and the gradient of the first two.
//
// Forward.  With a reference m, c = log2(e) / T and d_i = (x_i - m) c, a row needs S = sum 2^d_i and D = sum d_i 2^d_i: ln p_t = (x_t - m) / T - ln S
// and the entropy is ln S - ln 2 D / S.  One pass over the row forms both: a wavefront keeps its largest entry so far as its m, every lane its shares
// of S and D, 16 entries in fp32 and those sums in fp64, scaled over when m grows (which happens a dozen times a row); lanes, wavefronts and chunks are joined in fp64.
// The same pass finds the top alternatives.  An entry is a candidate if it is above a bound that M entries of the row are known to reach: every
// wavefront says a value that its share of the M reach, at first among its lanes' first entries (each lane's largest of 16), later among the
// candidates in its list, and the smallest said is the bound.  A row of 128 256 leaves a few hundred candidates for fifty, and a tile of 16 entries a lane that has
// none costs one comparison a lane.  Candidates go to a list of the wavefront's in LDS as
// whole numbers that order as (value, lower index first); a full list is cut to its M largest, which raises the wavefront's bound.  At the end a
// histogram over the numbers' range finds a bound that at most kSelected of them reach, and those are ranked by comparing all with all.
// What bounds it: reading the rows where there are many (1024 x 128 256 fp32 with 50 alternatives 88 us, 6.0 TB/s), and otherwise how long one workgroup's steps
// take one after the other (256 x 32 000 bf16 with 20 alternatives 15 us, 8 without any).
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
struct alignas(32) Share {
  double s, d;    // sum 2^((x - top) c), sum of (x - top) c 2^(...)
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

__device__ __forceinline__ float largest3(float a, float b, float c) {  // NaN if one of them is, of either kind
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// kPer entries of a lane: 16 bytes at a time, 64 lanes side by side, as they are and as floats.
template <typename E> struct Tile {
  word4_any w[kPer / kWide<E>];
};
template <typename E> __device__ __forceinline__ void unpack(const Tile<E> &t, float (&v)[kPer]) {
#pragma unroll
  for (int u = 0; u < kPer / kWide<E>; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(E) == 2) split_pair(t.w[u][i], v[u * 8 + 2 * i], v[u * 8 + 2 * i + 1]);
      else v[u * 4 + i] = __uint_as_float(t.w[u][i]);
    }
}
// `x` is the lane's first entry; what lies `left` entries from it or further is -inf.
template <typename E> __device__ __forceinline__ Tile<E> load_tile(const E *x) {
  Tile<E> t;
#pragma unroll
  for (int u = 0; u < kPer / kWide<E>; ++u) t.w[u] = __builtin_nontemporal_load(reinterpret_cast<const word4_any *>(x + u * 64 * kWide<E>));
  return t;
}
template <typename E> __device__ __forceinline__ Tile<E> load_tile_end(const E *x, long long far) {
  constexpr int N = kWide<E>;
  const int left = far < 64 * kPer ? (int)far : 64 * kPer;
  Tile<E> t;
#pragma unroll
  for (int u = 0; u < kPer / N; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = u * 64 * N + i * (N / 4);
      if constexpr (sizeof(E) == 2)
        t.w[u][i] = (at < left ? (uint32_t)x[at] : 0xFF80u) | (at + 1 < left ? (uint32_t)x[at + 1] : 0xFF80u) << 16;
      else
        t.w[u][i] = __float_as_uint(at < left ? x[at] : -kInf);
    }
  return t;
}
// The tile whose first entry is `at` of a row (or chunk) that ends at `end`.
template <typename E> __device__ __forceinline__ Tile<E> load_at(const E *row, long long at, long long end) {
  const int lane = threadIdx.x & 63;
  if (at + 64 * kPer <= end) return load_tile(row + at + lane * kWide<E>);
  return load_tile_end(row + at + lane * kWide<E>, end - at - lane * kWide<E>);
}

// The same without a branch, for what is asked for ahead: a load that would reach beyond `end` starts at `last`, the place of the last whole one, instead.  (A
// load under a condition is waited for at once: the compiler copies what it brought, word by word, to where both ways meet.)
template <typename E> __device__ __forceinline__ uint32_t held(uint32_t from, uint32_t last) { return from < last ? from : last; }
template <typename E, bool AGAIN> __device__ __forceinline__ Tile<E> load_held(const E *row, uint32_t at, uint32_t last) {  // AGAIN: it is read a second time, soon
  constexpr int N = kWide<E>;
  Tile<E> t;
#pragma unroll
  for (int u = 0; u < kPer / N; ++u) {
    const word4_any *from = reinterpret_cast<const word4_any *>(row + held<E>(at + (u * 64 + (threadIdx.x & 63)) * N, last));
    t.w[u] = AGAIN ? *from : __builtin_nontemporal_load(from);
  }
  return t;
}
// What such loads have brought of other lanes' entries counts as nothing.
template <typename E> __device__ __forceinline__ void drop_others(Tile<E> &t, uint32_t at, uint32_t last) {
  constexpr int N = kWide<E>;
#pragma unroll
  for (int u = 0; u < kPer / N; ++u) {
    const uint32_t from = at + (u * 64 + (threadIdx.x & 63)) * N, others = from - held<E>(from, last);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      if constexpr (sizeof(E) == 2) {
        uint32_t o = t.w[u][i];
        o = 2 * i < others ? (o & 0xFFFF0000u) | 0xFF80u : o;
        t.w[u][i] = 2 * i + 1 < others ? (o & 0xFFFFu) | 0xFF800000u : o;
      } else {
        t.w[u][i] = i < others ? 0xFF800000u : t.w[u][i];
      }
    }
  }
}

// Exponents are x c less a reference that follows from the largest entry m: m c as fp32 has it.  One multiply-add forms them, exact but for its one rounding, and
// what the reference's own rounding shifts all of them by is put right at the end.  That shift has to stay small beside the range of 2^y: it is 2^-3 at most
// below 2^22, where the reference stops (from 2^31 on it may be 128).  Beyond, exponents are (x - m) c.
__device__ __forceinline__ bool has_reference(float m, float c) { return fabsf(m) * c < 0x1p22f; }
__device__ __forceinline__ float reference_of(float m, float c) {
#pragma clang fp contract(off)  // (it is rounded wherever it is used)
  return m * c;
}
// From exponents relative to what belongs to `from` to those relative to what belongs to the larger `to`.
__device__ __forceinline__ float shift_between(float from, float to, float c) {
  const bool at_from = has_reference(from, c), at_to = has_reference(to, c);
  const float by = at_from ? at_to ? reference_of(from, c) - reference_of(to, c) : -fmaf(to, c, -reference_of(from, c))
                           : at_to ? fmaf(from, c, -reference_of(to, c)) : (from - to) * c;
  return fmaxf(by, -200.0f);  // (from -inf: -200, or NaN, which is nothing to max)
}

// A wavefront's sums and candidates.
template <typename E> struct Scan {
  float m = -kInf;      // largest entry so far
  double s = 0.0, d = 0.0;  // (a tile's 16 entries are added up in fp32, tiles in fp64: a running fp32 sum of equal terms is off by 4e-6 after 4096 of them, 6e-5 after 16 384)
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

// One tile: `first` is the index in the row of the lane's first entry, and where its loads start `last` at the most.
template <typename E> __device__ __forceinline__ void take_tile(Scan<E> &w, const Tile<E> &tile, uint32_t first, uint32_t last, float c, int M, u64 *list) {
  constexpr int N = kWide<E>;
  float v[kPer];
  unpack(tile, v);
  // The largest of either half of the entries.  (A NaN has to show in it.  v_max3_f32 lets a number beside a quiet NaN through, and quiets a signalling one, which the next step
  // then takes for less than any number, with all that it was compared to: a lane would miss its largest entry, and what is put into the list would not have been counted.)
  float half[2];
  const auto largest = [&] {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float *o = v + h * (kPer / 2);
      half[h] = largest3(largest3(o[0], o[1], o[2]), largest3(o[3], o[4], o[5]), largest3(o[6], o[7], o[7]));
    }
    return largest3(half[0], half[1], half[1]);
  };
  float t = largest();
  if (__ballot(!(t <= fminf(w.bound, w.m))) != 0) {  // (a lane with a NaN comes here too; where few entries are, the bound may be above them all)
    if (__ballot(!(t < kInf)) != 0) {    // entries without mass
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = with_mass(v[i]) ? v[i] : -kInf;
      t = largest();
    }
    if (__ballot(t > w.m) != 0) {
      const float m = wave_max(t), by = shift_between(w.m, m, c), scale = __builtin_amdgcn_exp2f(by);
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
          u64 masks[kPer];  // (all comparisons first: none waits for the branch before it)
#pragma unroll
          for (int i = h * (kPer / 2); i < (h + 1) * (kPer / 2); ++i) masks[i] = __ballot(v[i] > w.bound);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = h * (kPer / 2); i < (h + 1) * (kPer / 2); ++i) {
            const u64 mask = masks[i];
            if (mask == 0) continue;
            if (v[i] > w.bound) list[w.count + lanes_below(mask)] = key_of(v[i], held<E>(first + (i / N) * 64 * N, last) + i % N);
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
          const u64 key = key_of(mine, held<E>(__builtin_amdgcn_readlane(first, from) + (lane / N) * 64 * N, last) + lane % N);
          const bool offered = mine > w.bound && key > least;
          const u64 mask = __ballot(offered);
          if (offered) list[w.count + lanes_below(mask)] = key;
          w.count += (int)__builtin_popcountll(mask);
        }
        if (least != 0) w.bound = fmaxf(w.bound, key_value(least));  // (what equals the least kept one comes after it in a later tile)
      }
    }
  }
  float s[2], sd[2];  // (two sums of either kind, so that one's additions do not wait for each other)
  const auto add = [&](int i, float d) {
    const float e = __builtin_amdgcn_exp2f(d);  // (no mass: 2^-200 is 0)
    s[i & 1] = i < 2 ? e : s[i & 1] + e;
    sd[i & 1] = i < 2 ? e * d : fmaf(e, d, sd[i & 1]);
  };
  if (has_reference(w.m, c)) {  // (not where nothing has had mass yet)
    const float reference = reference_of(w.m, c);
#pragma unroll
    for (int i = 0; i < kPer; ++i) add(i, fmaxf(fmaf(v[i], c, -reference), -200.0f));
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) add(i, fmaxf((v[i] - w.m) * c, -200.0f));
  }
  w.s += (double)(s[0] + s[1]);
  w.d += (double)(sd[0] + sd[1]);
}

// A number that n of the lanes' K ordered values each reach, and little below the n-th largest of them (its upper 16 bits); 0 if there are fewer than n.
// Two bits a step: the three counts of a step do not wait for each other.
template <int K> __device__ __forceinline__ uint32_t reached_by(const uint32_t (&o)[K], int n) {
  uint32_t t = 0;
#pragma unroll 2
  for (int bit = 30; bit >= 16; bit -= 2) {
    uint32_t best = t;
#pragma unroll
    for (uint32_t q = 1; q < 4; ++q) {
      const uint32_t with = t + (q << bit);
      int reach = 0;
#pragma unroll
      for (int i = 0; i < K; ++i) reach += (int)__builtin_popcountll(__ballot(o[i] >= with));
      if (reach >= n) best = with;
    }
    t = best;
  }
  return t;
}
// What all wavefronts have said so far.
__device__ __forceinline__ uint32_t least_said(const uint32_t *said, int waves) {
  const int lane = threadIdx.x & 63;
  uint32_t v = 0xFFFFFFFFu;
  if (lane < waves) v = __hip_atomic_load(&said[lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
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
template <int K> __device__ __forceinline__ float look_at_list(u64 *list, int &count, int share, bool speaks, uint32_t *said, int waves, int wave) {
  const int lane = threadIdx.x & 63;
  u64 k[K];
  uint32_t o[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    k[i] = i * 64 + lane < count ? list[i * 64 + lane] : 0;
    o[i] = (uint32_t)(k[i] >> 32);
  }
  if (speaks) {
    const uint32_t nth = reached_by(o, share);
    if (lane == 0) __hip_atomic_store(&said[wave], nth, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
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

// ln s, s at least 1 or near it: the exponent is taken off first and the mantissa lies around 1, so that the hardware's fp32 logarithm, of a number between
// -1/2 and 1/2, is off by 2^-24 at most; what the mantissa loses as an fp32 number is added.  (The library's fp64 logarithm keeps 40 registers of
// constants through a loop over rows.)
__device__ __forceinline__ double ln_of(double s) {
  int e = __builtin_amdgcn_frexp_exp(s);
  double m = __builtin_amdgcn_frexp_mant(s);
  const bool low = m < 0.70703125;
  m = low ? 2.0 * m : m;
  e = low ? e - 1 : e;
  const float f = (float)m;
  return kLn2 * ((double)e + (double)__builtin_amdgcn_logf(f)) + (double)((float)(m - (double)f) * __builtin_amdgcn_rcpf(f));
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
  const float c = kLog2e / temp;
  const double sum = any ? ln_of(s) : -(double)kInf;
  r.entropy = any ? sum - kLn2 * d / s : 0.0;
  r.rest = any && has_reference(top, c) ? sum + kLn2 * ((double)reference_of(top, c) - (double)top * (double)c) : sum;
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
  const double by = mine > -kInf ? (double)shift_between(mine, top, c) : -200.0, scale = (double)__builtin_amdgcn_exp2f((float)by);  // (off by 2^-23 of a wavefront's share)
  d = wave_sum((d + s * by) * scale);
  s = wave_sum(s * scale);
}

// One workgroup a row, or a chunk of it.  TINY: rows shorter than a load.
template <typename E, int WAVES, bool TINY = false> __global__ void __launch_bounds__(WAVES * 64) score_kernel(const ScoreParams p) {
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
  Tile<E> here, next;
  long long at = begin + (long long)wave * kTile;
  // (loads return in order: tokens are asked for before the row, their entries after it)
  int token = -1;
  if (p.chunks == 1 && (int)threadIdx.x < p.G) token = p.tokens[r * p.tok_stride_r + threadIdx.x];
  __builtin_amdgcn_sched_barrier(0);
  const uint32_t last = TINY ? 0u : (uint32_t)end - N;
  const auto load = [&](long long from) {
    if constexpr (TINY) return load_at(x, from, end);
    else return load_held<E, false>(x, (uint32_t)from, last);
  };
  here = load(at);
  next = load(at + WAVES * kTile);
  __builtin_amdgcn_sched_barrier(0);
  const E token_raw = x[token >= 0 && token < p.V ? token : 0];
  // A bound that M entries reach: every wavefront's share of them is among what it has seen.  First each lane's largest of the first tile; later,
  // whenever a wavefront has seen twice as much, the candidates in its list.  What a wavefront has once said stays true, so nobody waits.
  // (Of wavefronts whose first tile is whole: one with a few entries, or none, would have nothing to say.)
  const int whole = (int)((end - begin) / kTile), speakers = whole < 1 ? 1 : whole < WAVES ? whole : WAVES;
  const bool speaks = wave < speakers;
  const int share = (p.M + speakers - 1) / speakers;
  if (p.M > 0) {
    float t = -kInf;
    if (speaks || at < end) {
      Tile<E> first = here;
      if (!TINY && at + kTile > end) drop_others<E>(first, (uint32_t)at, last);
      float v[kPer];
      unpack(first, v);
#pragma unroll
      for (int i = 0; i < kPer; ++i) t = fmaxf(t, with_mass(v[i]) ? v[i] : -kInf);
    }
    const uint32_t o[1] = {ordered(t)}, nth = !speaks ? 0xFFFFFFFFu : share <= 64 ? reached_by(o, share) : 0;
    if (lane == 0) s_nth[wave] = nth;
    __syncthreads();
    w.bound = just_below(least_said(s_nth, WAVES));
  }
  const auto look = [&] {
    if (w.count < share) return;
    w.bound = fmaxf(w.bound, w.count <= 64 ? look_at_list<1>(list, w.count, share, speaks, s_nth, WAVES, wave)
                                           : look_at_list<kList / 64>(list, w.count, share, speaks, s_nth, WAVES, wave));
  };
  // A list is looked at after the wavefront's second, fourth, eighth tile, and so on, unless nothing follows; after the first too where so large a share soon
  // fills it.  (Always after the first, and never: 4 x 32 000 bf16 with 5 alternatives 12.7 us, 11.2; 300 rows with 20 19.8, 18.3; but 1024 rows with 128
  // of four wavefronts 41.0, 51.7.  From the eighth on 256 x 128 256 bf16 with 50 takes 45 for 32.)
  const int first_look = share > 16 ? 1 : 2;
  // two tiles in turn, so that one is on its way while the other is taken
  const long long step = (long long)WAVES * kTile;
  const auto take = [&](Tile<E> tile, long long from) {
    if (!TINY && from + kTile > end) drop_others<E>(tile, (uint32_t)from, last);  // (uniform)
    take_tile<E>(w, tile, (uint32_t)(from + lane * N), TINY ? 0xFFFFFFFFu : last, c, p.M, list);
  };
  for (int tiles = 1; at < end; tiles += 2, at += 2 * step) {
    take(here, at);
    here = load(at + 2 * step);
    if (at + step >= end) break;
    if (p.M > 0 && tiles >= first_look && (tiles & (tiles - 1)) == 0) look();
    take(next, at + step);
    next = load(at + 3 * step);
    if (p.M > 0 && (tiles & (tiles + 1)) == 0 && at + 2 * step < end) look();
  }
  if (p.M > 0 && w.count > kSelected / WAVES) look();  // (else what all have is soon ranked)
  // the wavefronts' sums
  const double ws = wave_sum(w.s), wd = wave_sum(w.d);
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
    if (threadIdx.x == 0) p.shares[r * p.chunks + part] = Share{s, d, top, total < p.M ? total : p.M};
    if (p.M > 0) select_top<WAVES * 64>(s_list, WAVES, kList, s_count, least, high, p.M, [&](int rank, u64 key) { keys[rank] = key; });
    return;
  }
  const Row row = row_of(top, s, d, p.temp);
  if ((int)threadIdx.x < p.G && p.logp != nullptr) p.logp[r * p.G + threadIdx.x] = token < 0 ? 0.0f : token < p.V ? row.logp(widen(token_raw)) : -kInf;
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
  Share share = {0.0, 0.0, -kInf, 0};
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
  // M keys reach the least that a chunk with M has
  const u64 *keys = p.keys + r * p.chunks * p.M;
  u64 least = lane < p.chunks && share.count == p.M ? keys[lane * p.M + p.M - 1] : 0;
#pragma unroll
  for (int i = 32; i >= 1; i >>= 1) {
    const u64 other = __shfl_xor(least, i);
    least = other > least ? other : least;
  }
  least = least != 0 ? least : 1;
  __syncthreads();
  select_top<kBlock>(keys, p.chunks, p.M, s_count, least, key_of(top > -kInf ? top : 0.0f, 0), p.M,
                     [&](int rank, u64 key) { write_top(p, r, row, rank, key); });
}

// ---- the gradient
// With y_i = (x_i - top) c - log2(e) rest, so that p_i = 2^y_i, an entry's gradient is 2^y (a + b y) and at a token's place its weight / T more.  The
// rounding of log2(e) rest to fp32 goes into a and b.  The hardware's 2^y is 0 below 2^-126, so what multiplies it is brought near 1: 2^y is taken as much larger as a and b are made
// smaller.
struct Weights {
  float top, shift, c, a, b, inv_t;
  float line;  // -(top c + shift)
  int form;    // 0: a 2^(x c + line); 1: with b; 2: whatever the values are
};
__device__ __forceinline__ Weights uniform(const Weights &w) {  // (all lanes have the same: in scalar registers)
  const auto one = [](float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); };
  return Weights{one(w.top), one(w.shift), one(w.c), one(w.a), one(w.b), one(w.inv_t), one(w.line), __builtin_amdgcn_readfirstlane(w.form)};
}
// A row's tokens and their weights: lane i has the i-th, and its share of the sum of all valid ones' weights.  (Read again for every
// tile they cost the gradient of 2048 x 32 000 bf16 3 us.)
struct RowTokens {
  int token;
  float weight;
  double share;
};
// Loads return in order, so what is known of the tokens at once is asked for before the row: their use waits for the row's loads otherwise.
struct FirstTokens {
  int token, mine;  // the lane's of the first 64, the thread's of all
  float weight;
};
__device__ __forceinline__ FirstTokens first_tokens(const ScoreParams &p, long long r) {
  const int lane = threadIdx.x & 63;
  FirstTokens t = {-1, -1, 0.0f};
  if (lane < p.G) {
    t.token = p.tokens[r * p.tok_stride_r + lane];
    t.weight = p.a[r * p.a_stride_r + lane];
  }
  if (p.logp != nullptr && (int)threadIdx.x < p.G) t.mine = p.tokens[r * p.tok_stride_r + threadIdx.x];
  __builtin_amdgcn_sched_barrier(0);
  return t;
}
__device__ __forceinline__ RowTokens tokens_of(const ScoreParams &p, long long r, const FirstTokens &first) {
  RowTokens t = {first.token, first.weight, 0.0};
  if (first.token >= 0 && first.token < p.V) t.share = (double)first.weight;
  for (int g = (int)(threadIdx.x & 63) + 64; g < p.G; g += 64) {
    const int token = p.tokens[r * p.tok_stride_r + g];
    const float weight = p.a[r * p.a_stride_r + g];
    if (token >= 0 && token < p.V) t.share += (double)weight;
  }
  return t;
}
__device__ __forceinline__ Weights weights_of(const ScoreParams &p, long long r, double share, double top, double rest, double entropy) {
  const double sum = wave_sum(share);
  const double inv_t = 1.0 / (double)p.temp;
  Weights w = {0.0f, 1000.0f, kLog2e / p.temp, 0.0f, 0.0f, (float)inv_t, 0.0f, 2};
  if (!(rest > -(double)kInf)) return w;  // (without mass all entries get 0)
  const double shift = rest / kLn2, at_top = (double)w.c * top;
  double a = -sum * inv_t, b = 0.0;
  if (p.b != nullptr) {
    b = -(double)p.b[r] * kLn2 * inv_t;
    a -= (double)p.b[r] * entropy * inv_t;
  }
  // One multiply-add an entry, x c + line, serves unless top c is so large that fp32 keeps too little of it, and what 2^y loses below 2^-126 counts only with large weights.
  const double size = fabs(a) + 128.0 * fabs(b);
  const bool plain = fabs(at_top) < 65536.0 && size < 1.0;
  const int lift = size < 1.0 ? 0 : min(__builtin_amdgcn_frexp_exp(size), 127);
  w.top = (float)top;
  w.line = (float)-(at_top + shift);
  w.shift = (float)(shift - (double)lift);
  // y as it is formed is above the true one by `over`
  const double over = plain ? at_top + shift + (double)w.line : shift - (double)lift - (double)w.shift;
  const double off = 1.0 - over * kLn2 * (1.0 - 0.5 * over * kLn2);  // 2^-over: it is 2^-8 at most
  const double scale = ldexp(off, -lift);
  a -= b * (over + (double)lift);
  w.a = (float)(a * scale);
  w.b = (float)(b * scale);
  w.form = !plain ? 2 : p.b != nullptr ? 1 : 0;
  return uniform(w);
}

// From a tile's entries to their gradients, tokens apart.
__device__ __forceinline__ void entry_gradients(const Weights &w, float (&v)[kPer]) {
  float t = largest3(v[0], v[1], v[2]);
#pragma unroll
  for (int i = 3; i + 1 < kPer; i += 2) t = largest3(t, v[i], v[i + 1]);
  t = largest3(t, v[kPer - 1], v[kPer - 1]);
  if (__ballot(!(t <= w.top)) != 0) {  // a NaN among them, +inf (and in a row without mass anything)
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = with_mass(v[i]) ? v[i] : -kInf;
  }
  if (w.form == 0) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = __builtin_amdgcn_exp2f(fmaf(v[i], w.c, w.line)) * w.a;
  } else if (w.form == 1) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float y = fmaxf(fmaf(v[i], w.c, w.line), -200.0f);
      v[i] = __builtin_amdgcn_exp2f(y) * fmaf(y, w.b, w.a);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float y = fmaxf(fmaf(v[i] - w.top, w.c, -w.shift), -200.0f);
      v[i] = __builtin_amdgcn_exp2f(y) * fmaf(y, w.b, w.a);
    }
  }
}
// And the tokens that lie in the tile.  `first(u)`: the row's entry that the lane's load u starts with; none lies before `low` or from `high` on.
template <typename E, typename F>
__device__ __forceinline__ void token_gradients(const ScoreParams &p, long long r, const Weights &w, const RowTokens &tokens, const Tile<E> &tile,
                                                float (&v)[kPer], int low, int high, F first) {
  constexpr int N = kWide<E>;
  const int lane = threadIdx.x & 63;
  int token = tokens.token;
  float weight = tokens.weight;
  for (int g0 = 0;;) {
    u64 hits = __ballot(token >= low && token < high);
    if (hits != 0) {
      float x[kPer];
      unpack(tile, x);
      for (; hits != 0; hits &= hits - 1) {
        const int from = __builtin_ctzll(hits), place = __builtin_amdgcn_readlane(token, from);
        const float more = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight * w.inv_t), from));
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (place == first(i / N) + i % N && with_mass(x[i])) v[i] += more;
      }
    }
    g0 += 64;
    if (g0 >= p.G) break;
    token = -1;
    if (g0 + lane < p.G) {
      token = p.tokens[r * p.tok_stride_r + g0 + lane];
      weight = p.a[r * p.a_stride_r + g0 + lane];
    }
  }
}
template <typename E> __device__ __forceinline__ void store_tile(E *row, long long at, long long end, const float (&v)[kPer]) {
  constexpr int N = kWide<E>;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int u = 0; u < kPer / N; ++u) {
    float o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = v[u * N + i];
    E *to = row + at + (u * 64 + lane) * N;
    if (at + 64 * kPer <= end) {
      stream_some<N>(to, o);
    } else {
      const int left = (int)(end - at) - (u * 64 + lane) * N;
      if (left > 0) stream_first<N>(to, left, o);
    }
  }
}

// From a row's lse and entropy: a wavefront takes 4 KB of it, in one tile or two.  (us with one tile, with two and with four: 2048 x 32 000 bf16 52, 46 (5.7 TB/s), 52;
// 512 x 152 064 bf16 with entropies 56, 52, 58; 768 x 128 256 fp32 with entropies 126 (6.3 TB/s), 132, 142.)
template <typename E> constexpr int kTilesOf = sizeof(E) == 2 ? 2 : 1;
template <typename E> __global__ void __launch_bounds__(kBlock) score_grad_kernel(const ScoreParams p) {
  constexpr int kTile = 64 * kPer, TILES = kTilesOf<E>;
  const long long r = blockIdx.x / p.chunks;
  const int part = (int)(blockIdx.x - r * p.chunks), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const long long begin = ((long long)part * (kBlock / 64) + wave) * kTile * TILES;
  if (begin >= p.V) return;
  const E *x = reinterpret_cast<const E *>(p.x) + r * p.stride_r;
  E *grad = reinterpret_cast<E *>(p.grad) + r * p.grad_stride_r;
  const FirstTokens asked = first_tokens(p, r);
  const auto weights = [&](const RowTokens &tokens) {
    return weights_of(p, r, tokens.share, p.lse_in[2 * r], p.lse_in[2 * r + 1], p.b != nullptr ? (double)p.entropy_in[r] : 0.0);
  };
  const auto write = [&](const Weights &w, const RowTokens &tokens, const Tile<E> &tile, long long at) {
    float v[kPer];
    unpack(tile, v);
    entry_gradients(w, v);
    const int high = (int)(at + kTile < p.V ? at + kTile : p.V);
    token_gradients(p, r, w, tokens, tile, v, (int)at, high, [&](int u) { return (int)at + (u * 64 + lane) * kWide<E>; });
    store_tile(grad, at, p.V, v);
  };
  if (begin + kTile * TILES <= p.V) {
    Tile<E> tiles[TILES];
#pragma unroll
    for (int k = 0; k < TILES; ++k) tiles[k] = load_tile(x + begin + k * kTile + lane * kWide<E>);
    __builtin_amdgcn_sched_barrier(0);
    const RowTokens tokens = tokens_of(p, r, asked);
    const Weights w = weights(tokens);
#pragma unroll
    for (int k = 0; k < TILES; ++k) write(w, tokens, tiles[k], begin + k * kTile);
  } else {
    const RowTokens tokens = tokens_of(p, r, asked);
    const Weights w = weights(tokens);
    for (long long at = begin; at < p.V; at += kTile) write(w, tokens, load_at(x, at, p.V), at);
  }
}

// Scores and gradient in one pass: a workgroup keeps a row on the chip.  Memory bounds it, and the issue of two exponentials an entry: 2048 x 32 000 bf16
// 50 us, 5.2 TB/s read and written; 768 x 128 256 fp32 with 8 tokens and entropies 152 us, as much.  (A CU's rows load, join and write in part at the same time:
// of 25 us that a bf16 row takes there, 12 pass until all of it is summed, 3 until its wavefronts know so, 7 with writing.)  What its wavefronts share:
template <typename E, int WAVES> struct RowWork {
  double s_s[WAVES], s_d[WAVES];
  float s_m[WAVES];

  // The row may be overwritten later: what its tokens need is read at the start.  (The thread's own as it is: what became of it here would be waited for.)
  static __device__ __forceinline__ E read_tokens(const ScoreParams &p, long long r, int token) {
    const E *x = reinterpret_cast<const E *>(p.x) + r * p.stride_r;
    if (p.logp != nullptr && p.G > WAVES * 64)
      for (int g = threadIdx.x; g < p.G; g += WAVES * 64) {
        const int other = p.tokens[r * p.tok_stride_r + g];
        p.logp[r * p.G + g] = other >= 0 && other < p.V ? widen(x[other]) : -kInf;
      }
    return x[token >= 0 && token < p.V ? token : 0];
  }
  // From the wavefronts' sums to the scores and what the gradient needs.
  __device__ __forceinline__ Weights join(const ScoreParams &p, long long r, const Scan<E> &w, int token, E token_raw, double share) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    double s = wave_sum(w.s), d = wave_sum(w.d);
    float token_x = token >= 0 && token < p.V ? widen(token_raw) : -kInf;
    asm volatile("" : "+v"(token_x));  // (here: not while other wavefronts already write)
    if (lane == 0) { s_s[wave] = s; s_d[wave] = d; s_m[wave] = w.m; }
    __syncthreads();
    const int mine = lane < WAVES ? lane : 0;
    const float my_top = lane < WAVES ? s_m[mine] : -kInf, top = wave_max(my_top);
    s = lane < WAVES ? s_s[mine] : 0.0;
    d = lane < WAVES ? s_d[mine] : 0.0;
    join_shares(s, d, my_top, top, kLog2e / p.temp);
    const Row row = row_of(top, s, d, p.temp);
    if (threadIdx.x == 0) {
      if (p.lse != nullptr) { p.lse[2 * r] = row.top; p.lse[2 * r + 1] = row.rest; }
      if (p.entropy != nullptr) p.entropy[r] = (float)row.entropy;
    }
    if (p.logp != nullptr)
      for (int g = threadIdx.x; g < p.G; g += WAVES * 64) {
        if (p.G > WAVES * 64) {
          token = p.tokens[r * p.tok_stride_r + g];
          token_x = p.logp[r * p.G + g];
        }
        p.logp[r * p.G + g] = token < 0 ? 0.0f : row.logp(token_x);
      }
    return weights_of(p, r, share, row.top, row.rest, row.entropy);
  }
};

// Tiles of these kernels: counted from the row's end, tile k of a wavefront is the (k * waves + wave)-th from it, in whole 16-byte loads.  One that would
// reach beyond the row starts earlier instead: its first entries are another lane's too, count there only, and get the same gradient from both.  (With a
// case for every entry of a row's end the loops below were so large that they spilled.)  In place it matters that such a tile is read before anything
// is written: it is the first of its wavefront, which is always kept.
template <typename E> struct RowTile {
  static constexpr int N = kWide<E>, kLoads = kPer / N;
  uint32_t at, last;  // the tile's first entry; where a row's last load starts (a tile that is not there: both are the same)
  __device__ __forceinline__ int first(int u) const { return (int)held<E>(at + (u * 64 + (threadIdx.x & 63)) * N, last); }
  template <bool AGAIN> __device__ __forceinline__ Tile<E> load(const E *row) const { return load_held<E, AGAIN>(row, at, last); }
  __device__ __forceinline__ void add_up(const ScoreParams &p, Scan<E> &w, const Tile<E> &tile) const {
    Tile<E> t = tile;
    if (at + 64 * kPer > (uint32_t)p.V) drop_others<E>(t, at, last);  // (uniform)
    take_tile<E>(w, t, 0, 0, kLog2e / p.temp, 0, nullptr);
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void write(const ScoreParams &p, long long r, const Weights &weights, const RowTokens &tokens, Tile<E> tile) const {
    // (the compiler would keep the floats of the first pass: twice the registers)
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      uint32_t a = tile.w[u].x, b = tile.w[u].y, c = tile.w[u].z, d = tile.w[u].w;
      asm volatile("" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
      tile.w[u] = word4_any{a, b, c, d};
    }
    float v[kPer];
    unpack(tile, v);
    entry_gradients(weights, v);
    token_gradients(p, r, weights, tokens, tile, v, (int)(at < last ? at : last), (int)min(at + 64 * kPer, (uint32_t)p.V), [&](int u) { return first(u); });
    E *row = reinterpret_cast<E *>(p.grad) + r * p.grad_stride_r;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      float o[N];
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = v[u * N + i];
      stream_some<N>(row + first(u), o);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
};

// The whole row in registers, TILES tiles a wavefront.
template <typename E, int WAVES, int TILES>
__global__ void __launch_bounds__(WAVES * 64, TILES * sizeof(E) > 8 ? 4 : TILES * sizeof(E) > 4 ? 5 : 6) score_row_kernel(const ScoreParams p, int n_tiles) {
  __shared__ RowWork<E, WAVES> work;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long r = blockIdx.x;
  const E *x = reinterpret_cast<const E *>(p.x) + r * p.stride_r;
  const auto there = [&](int k) { return k * WAVES + wave < n_tiles; };
  const uint32_t last = (uint32_t)(p.V - kWide<E>);
  const auto tile = [&](int k) { return RowTile<E>{there(k) ? (uint32_t)(n_tiles - 1 - (k * WAVES + wave)) * 64 * kPer : last, last}; };
  const FirstTokens asked = first_tokens(p, r);
  Tile<E> tiles[TILES];
#pragma unroll
  for (int k = 0; k < TILES; ++k) tiles[k] = tile(k).template load<false>(x);
  __builtin_amdgcn_sched_barrier(0);
  const E token_raw = work.read_tokens(p, r, asked.mine);
  const RowTokens tokens = tokens_of(p, r, asked);
  Scan<E> w;
#pragma unroll
  for (int k = 0; k < TILES; ++k)
    if (there(k)) tile(k).add_up(p, w, tiles[k]);
  const Weights weights = work.join(p, r, w, asked.mine, token_raw, tokens.share);
#pragma unroll
  for (int k = 0; k < TILES; ++k)
    if (there(k)) tile(k).write(p, r, weights, tokens, tiles[k]);
}

// A longer row: a part in registers, a part in LDS, and what is left is read twice, the second time from the caches.  (768 x 128 256 fp32 with four tiles in
// registers 157 us for 154 with three; five spill, 160.)
template <typename E> __global__ void __launch_bounds__(1024) score_long_row_kernel(const ScoreParams p, int n_tiles) {
  constexpr int kWaves = 16, kLoads = RowTile<E>::kLoads, kRegs = sizeof(E) == 2 ? 8 : 3, kLds = sizeof(E) == 2 ? 4 : 2;
  __shared__ RowWork<E, kWaves> work;
  __shared__ word4_any s_tiles[kLds * kWaves * kLoads * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long r = blockIdx.x;
  const E *x = reinterpret_cast<const E *>(p.x) + r * p.stride_r;
  const auto there = [&](int k) { return k * kWaves + wave < n_tiles; };
  const uint32_t last = (uint32_t)(p.V - kWide<E>);
  const auto tile = [&](int k) { return RowTile<E>{there(k) ? (uint32_t)(n_tiles - 1 - (k * kWaves + wave)) * 64 * kPer : last, last}; };
  word4_any *mine = s_tiles + wave * kLoads * 64 + lane;
  const FirstTokens asked = first_tokens(p, r);
  // (what registers keep comes last, so that they are free until then)
  int k = kRegs;
  Tile<E> next = tile(k).template load<true>(x);
  __builtin_amdgcn_sched_barrier(0);
  const E token_raw = work.read_tokens(p, r, asked.mine);
  const RowTokens tokens = tokens_of(p, r, asked);
  Scan<E> w;
  for (; there(k); ++k) {
    const Tile<E> here = next;
    next = tile(k + 1).template load<true>(x);
    if (k < kRegs + kLds) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) mine[((k - kRegs) * kWaves * kLoads + u) * 64] = here.w[u];
    }
    tile(k).add_up(p, w, here);
  }
  Tile<E> tiles[kRegs];
#pragma unroll
  for (int k = 0; k < kRegs; ++k) tiles[k] = tile(k).template load<false>(x);
#pragma unroll
  for (int k = 0; k < kRegs; ++k)
    if (there(k)) tile(k).add_up(p, w, tiles[k]);
  const Weights weights = work.join(p, r, w, asked.mine, token_raw, tokens.share);
#pragma unroll
  for (int k = 0; k < kRegs; ++k)
    if (there(k)) tile(k).write(p, r, weights, tokens, tiles[k]);
  k = kRegs + kLds;
  next = tile(k).template load<false>(x);
  for (int l = kRegs; l < kRegs + kLds && there(l); ++l) {
    Tile<E> here;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) here.w[u] = mine[((l - kRegs) * kWaves * kLoads + u) * 64];
    tile(l).write(p, r, weights, tokens, here);
  }
  for (; there(k); ++k) {
    const Tile<E> here = next;
    next = tile(k + 1).template load<false>(x);
    tile(k).write(p, r, weights, tokens, here);
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

// Workgroups that a row is split over: as many as leave each 16 000 entries, as far as there are CUs for them, if that is three or more and the row has 64 000 (the
// second launch takes some 3 us), or two and the row has 128 000.  us a call with 50 alternatives, whole and split: 1 x 128 256 fp32 27.4, 19.3 (8); 64 x 128 256
// 30.2, 24.9 (4); 85 x 128 256 bf16 30.2, 24.9 (3); 1 x 4 194 304 fp32 321, 42 (64); 64 x 64 000 22.8, 21.3 (4); in two: 107 x 128 256 bf16 30.5, 28.9, fp32 30.6,
// 29.0; 128 x 152 064 bf16 32.5, 29.6 (without alternatives 16.6, 14.1), fp32 32.4, 30.3 (18.2, 18.2); 128 x 400 000 bf16 57.7, 45.5.  Not taken: 1 x 50 257 17.2,
// 18.6 (3); 85 x 50 257 19.5, 21.6 (3); 107 x 100 000 bf16 26.4, 26.2 (2; 128 alternatives 32.4, 33.2); 128 x 64 000 22.9, 23.7 (2); 4 x 32 000 bf16 15.2, 17.2 (2).
int auto_split(long long R, long long V) {
  if (V < 64000) return 1;
  long long split = V / 16000;
  if (split > 256 / (R > 0 ? R : 1)) split = 256 / (R > 0 ? R : 1);
  if (split < 3) return split == 2 && V >= 128000 ? 2 : 1;
  return (int)(split < kMostSplit ? split : kMostSplit);
}

// (Below 2^-126 log2(e) / temp and 1 / temp leave fp32.)
bool good_temp(float t) { return std::isfinite(t) && t >= 0x1p-126f; }

// Cuts a row into `want` chunks of whole 16-byte loads.
void split_rows(ScoreParams &p, long long want) {
  const long long each = ((p.V + want - 1) / want + 15) & ~15LL;
  p.chunk = (int)(each < kMaxIndex ? each : kMaxIndex);
  p.chunks = (int)((p.V + each - 1) / each);
}

template <typename E> hipError_t launch_gradient(ScoreParams p, hipStream_t st) {
  p.chunks = (int)(((long long)p.V + kBlock * kPer * kTilesOf<E> - 1) / (kBlock * kPer * kTilesOf<E>));
  score_grad_kernel<E><<<(unsigned)(p.R * p.chunks), kBlock, 0, st>>>(p);
  return hipGetLastError();
}

// Scores and gradient in one launch: as many wavefronts as keep the row in registers.  Rows too long for that are a workgroup's too where the scores would not be
// split over more than two: under 64 000 entries, or 86 rows and more, so that a CU in three has one at least.  With fewer, or up to 128 rows so long that reading them twice costs a workgroup more than splitting them in two, scores and gradient are two or
// three launches over all CUs.  us a call, one launch and several: 70 001 fp32 of 64 rows 18.1, 18.4, of 96 18.5, 22.5, of 256 30.2, 40.9; 128 256 fp32 of 64
// rows 26.9, 23.8, of 107 27.9, 35.3, of 256 45.9, 66.1; 152 064 bf16 of 64 29.4, 19.3, of 107 26.8, 28.7, of 256 34.8, 45.3; 107 rows of 200 000 bf16 32.3,
// 34.3, of 262 144 41.2, 41.0 (with entropies 46.0, 40.9), of 400 000 60.6, 55.0; of 400 000 fp32 82.3, 86.8, of 600 000 137, 127.  False: nothing was launched.
template <typename E> bool launch_rows(const ScoreParams &p, hipStream_t st) {
  const long long tiles = ((long long)p.V + 64 * kPer - 1) / (64 * kPer);
  constexpr bool kHalf = sizeof(E) == 2;
  const unsigned rows = (unsigned)p.R;
  if (p.V < kWide<E>) return false;
  if (tiles <= 1) score_row_kernel<E, 1, 1><<<rows, 64, 0, st>>>(p, (int)tiles);
  else if (tiles <= 4) score_row_kernel<E, 4, 1><<<rows, 256, 0, st>>>(p, (int)tiles);
  else if (tiles <= 8) score_row_kernel<E, 4, 2><<<rows, 256, 0, st>>>(p, (int)tiles);
  else if (tiles <= 16) score_row_kernel<E, 4, 4><<<rows, 256, 0, st>>>(p, (int)tiles);
  else if (tiles <= 32) score_row_kernel<E, kHalf ? 4 : 8, kHalf ? 8 : 4><<<rows, kHalf ? 256 : 512, 0, st>>>(p, (int)tiles);
  else if (kHalf && tiles <= 64) score_row_kernel<E, 8, kHalf ? 8 : 4><<<rows, 512, 0, st>>>(p, (int)tiles);
  else if (p.chunks == 1 || (p.chunks == 2 && p.V < (kHalf ? 1 << 18 : 1 << 19))) score_long_row_kernel<E><<<rows, 1024, 0, st>>>(p, (int)tiles);
  else return false;
  return true;
}

template <typename E> hipError_t launch_scores(const ScoreParams &p, hipStream_t st) {
  const unsigned blocks = (unsigned)(p.R * p.chunks);
  const long long tiles = ((long long)p.chunk + 64 * kPer - 1) / (64 * kPer);
  // us a call with four wavefronts and with eight: 32 000 bf16, 50 alternatives, 256 rows 23.0, 17.7; 512 24.9, 22.8; 768 28.5, 27.5; 2048 52.7, 58.6; without
  // alternatives 768 13.4, 14.3; 128 256 fp32 256 rows 45.7, 32.8; 512 53.9, 50.4; 2048 166, 165.  (Sixteen: 16.9 and 32.5 at 256 rows, 29.7 and 59 at 512.)
  if (p.V < kWide<E>) score_kernel<E, 1, true><<<blocks, 64, 0, st>>>(p);
  else if (tiles <= 1) score_kernel<E, 1><<<blocks, 64, 0, st>>>(p);
  else if (tiles <= 4 || blocks > 512) score_kernel<E, 4><<<blocks, 256, 0, st>>>(p);
  else score_kernel<E, 8><<<blocks, 512, 0, st>>>(p);
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
  if (logits && !good_temp(a->temp)) return LLC_E_TEMP;
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
  if (logits && !good_temp(a->temp)) return LLC_E_TEMP;
  if (!fits(a->x, type_size(a->dtype)) || !fits(a->grad, type_size(a->dtype)) || !fits(a->tokens, 4) || !fits(a->grad_logp, 4))
    return LLC_E_ALIGN;
  const long long split = a->v_chunks > 0 ? a->v_chunks : auto_split(a->R, a->V);
  if (a->lse_in == nullptr && (a->workspace == nullptr || !fits(a->workspace, 256) || a->workspace_bytes < rows_workspace(a->R, 0, split)))
    return LLC_E_WORKSPACE;
  if (a->R * split > kMostGrid || a->R * ((a->V + kBlock * kPer - 1) / (kBlock * kPer)) > kMostGrid) return LLC_E_SHAPE;
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
    const bool f32 = a->dtype == LLC_F32;
    if (a->lse_in == nullptr) {
      if (a->v_chunks == 0 && (f32 ? launch_rows<float>(p, st) : launch_rows<uint16_t>(p, st))) return hipGetLastError();
      const hipError_t e = f32 ? launch_scores<float>(p, st) : launch_scores<uint16_t>(p, st);
      if (e != hipSuccess) return e;
    }
    return f32 ? launch_gradient<float>(p, st) : launch_gradient<uint16_t>(p, st);
  });
}
