// Sampling from a cut distribution with given random numbers, and the cut rows themselves.
//
// The kept entries of a row are a run of its entries in the order of their values (larger first, equal ones by index), so a
// cut is a place of that order: the key of its last entry and that entry's index.  A workgroup takes a row.
//   1. The largest entry, and with it every thread's own.
//   2. A bound that the cut cannot be below, from the threads' largest entries (the k-th largest of them has k entries at or above it) or from
//      min_p; what is at or above it goes into a list, in the order of the indexes.  In the same pass, where a share of the whole mass is asked for, the mass.
//   3. The list is sorted, its masses are summed along the order, and the cut is read off; the tokens follow from sums along the indexes.
// Rows whose kept entries the list does not hold are narrowed down instead: a histogram of the masses (or counts) by value finds the range that the cut is
// in, histograms by the keys' bits find the key, and a count of its equals the index; tokens follow from the sums of tiles of the row.
//
// Masses are exp((x - largest) / temp) in fp64: a border in a run of 128 000 entries that share the mass is hit by rounding otherwise.  Histograms add them as whole numbers,
// whose sum does not depend on the order.
#include "ends.hpp"

namespace llc {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kList = 2048;       // entries of the list
constexpr int kBuckets = 2048;    // of a histogram
constexpr int kMostTiles = 2048;  // of a row, whose masses LDS holds
constexpr int kPiece = 512;       // entries that a wavefront takes at a time, eight a lane
constexpr int kByMass = 192;      // threads' largest entries that bound the list where a share of the mass is asked for
constexpr int kByCount = 512;     // top_k up to which the list is tried
constexpr unsigned kMostRowBlocks = 1u << 20;

struct CutParams {
  long long R, V;
  const void *x;
  long long stride;
  int logits;  // the temperature counts
  float temp, top_p, min_p;
  int top_k;
  const float *row_temp, *row_top_p, *row_min_p;
  const int32_t *row_top_k;
  int S;
  const float *u;
  long long u_stride;
  int32_t *tokens;
  float *logp;
  int32_t *kept;
  void *out;
  long long out_stride;
  int pieces_tile;  // pieces of a tile
  int tiles;        // of a row
  int tiles_wave;   // of a wavefront, which has them one after the other
};

// A row's settings.
struct Cut {
  double scale;   // log2(e) / temp
  double temp;
  long long top_k;  // 0: off
  float top_p;      // 1: off
  float min_p;      // 0: off
  bool bad;
};
__device__ __forceinline__ Cut cut_of(const CutParams &p, long long r) {
  Cut c;
  const float temp = p.logits == 0 ? 1.0f : p.row_temp != nullptr ? p.row_temp[r] : p.temp;
  const float top_p = p.row_top_p != nullptr ? p.row_top_p[r] : p.top_p;
  const float min_p = p.row_min_p != nullptr ? p.row_min_p[r] : p.min_p;
  const int top_k = p.row_top_k != nullptr ? p.row_top_k[r] : p.top_k;
  c.bad = !(temp >= 0x1p-126f && temp < INFINITY) || top_p != top_p || min_p != min_p;
  c.temp = (double)temp;
  c.scale = 1.4426950408889634 / c.temp;
  c.top_k = top_k > 0 && top_k < p.V ? top_k : 0;
  c.top_p = fminf(fmaxf(top_p, 0.0f), 1.0f);
  c.min_p = fminf(fmaxf(min_p, 0.0f), 1.0f);
  return c;
}

// Values as whole numbers in their order; both zeros are one.  A distance is the largest one's less the value's.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float((key & 0x80000000u) != 0 ? key ^ 0x80000000u : ~key); }
__device__ __forceinline__ bool has_mass(float x) { return fabsf(x) < INFINITY; }

// 2^t for t <= 0, to some 2^-50 of it; 0 below 2^-1000.
__device__ __forceinline__ double exp2_down(double t) {
  const double whole = rint(t), f = (t - whole) * 0.6931471805599453;
  double y = 1.0 / 479001600.0;  // exp(f), |f| <= 0.35, by its series: f^13 / 13! is 2e-16
  y = fma(y, f, 1.0 / 39916800.0);
  y = fma(y, f, 1.0 / 3628800.0);
  y = fma(y, f, 1.0 / 362880.0);
  y = fma(y, f, 1.0 / 40320.0);
  y = fma(y, f, 1.0 / 5040.0);
  y = fma(y, f, 1.0 / 720.0);
  y = fma(y, f, 1.0 / 120.0);
  y = fma(y, f, 1.0 / 24.0);
  y = fma(y, f, 1.0 / 6.0);
  y = fma(y, f, 0.5);
  y = fma(y, f, 1.0);
  y = fma(y, f, 1.0);
  return t > -1000.0 ? ldexp(y, (int)whole) : 0.0;
}
__device__ __forceinline__ double mass_of(float x, double top, double scale) { return exp2_down(((double)x - top) * scale); }

// Sums over a workgroup and along its threads.
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}
template <typename T> __device__ __forceinline__ T wave_scan(T v, int lane) {  // inclusive
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

struct Shared {
  union {
    unsigned long long histogram[kBuckets];
    unsigned long long sorted[kList];  // distance and index
    double along[kMostTiles > kList ? kMostTiles : kList];  // masses summed along the indexes
  };
  double masses[kList];  // summed along the order
  uint32_t list_distance[kList];
  int list_index[kList];
  float largest[kThreads];
  union {
    double wave_double[kWaves];
    unsigned long long wave_whole[kWaves];
  };
  int wave_count[kWaves + 1];
  float wave_float[kWaves];
  int overflow;
  unsigned long long pick_above;
  int pick;
  long long pick_index;
};

// Over the threads' values: the sum of those before, and of all.
template <typename T> __device__ __forceinline__ T block_scan_before(T v, T *s_wave, T &all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T upto = wave_scan(v, lane);
  __syncthreads();
  if (lane == 63) s_wave[wave] = upto;
  __syncthreads();
  T before = 0;
  all = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) before = all;
    all += s_wave[w];
  }
  return before + (upto - v);
}
template <typename T> __device__ __forceinline__ T block_sum(T v, T *s_wave) {
  T all;
  block_scan_before(v, s_wave, all);
  return all;
}

// A row's entries as a wavefront has them: `f(index of the first, its eight)` for its pieces in turn; those behind the row's end are -inf.
template <typename E> __device__ __forceinline__ void load_piece(const E *row, long long at, long long V, float (&v)[8]) {
  if (at + 8 <= V) {
    load_some<8>(row + at, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = at + j < V ? widen(row[at + j]) : -INFINITY;
  }
}
template <typename E, typename F> __device__ __forceinline__ void each_piece(const E *row, const CutParams &p, int wave, int lane, F f) {
  constexpr int kAhead = 4;
  const long long first = (long long)wave * p.tiles_wave * p.pieces_tile * kPiece;
  const long long last0 = first + (long long)p.tiles_wave * p.pieces_tile * kPiece, last = last0 < p.V ? last0 : p.V;
  for (long long at = first; at < last; at += kAhead * kPiece) {  // (uniform)
    float v[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (at + i * kPiece < last) load_piece(row, at + i * kPiece + lane * 8, p.V, v[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (at + i * kPiece < last) f(at + i * kPiece + lane * 8, v[i]);
  }
}

// The least bound that at least `n` of the threads' largest entries reach (-inf where fewer have one): to a bf16 number's bits, downwards.
__device__ __forceinline__ float bound_of(const float *largest, int n) {
  const int lane = threadIdx.x & 63;
  uint32_t key[kThreads / 64];
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) key[i] = has_mass(largest[i * 64 + lane]) ? key_of(largest[i * 64 + lane]) : 0u;
  uint32_t bound = 0;
  for (uint32_t bit = 0x80000000u; bit >= 0x8000u; bit >>= 1) {
    const uint32_t to = bound | bit;
    int count = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) count += __popcll(__ballot(key[i] >= to));
    if (count >= n) bound = to;
  }
  return bound <= 0x007FFFFFu ? -INFINITY : value_of(bound);  // (keys of numbers begin above)
}

// The place of the order where the weights' sum reaches `target`: a whole number's histogram by values, then by keys.  Entries behind `distance` (and,
// at it, behind `index`) take no part.  weight(x): the entry's, a whole number.
struct Place {
  uint32_t distance;  // of the last entry
  long long index;
};
__device__ __forceinline__ int bucket_of(float x, float top, float per) {
  const float at = (top - x) * per;  // (both roundings keep the order; an infinite `per` gives NaN at the top itself, and that 0)
  return at >= (float)(kBuckets - 1) ? kBuckets - 1 : (int)fmaxf(at, 0.0f);
}
// The bucket where the sum of those up to it reaches `target`; -1: none.  `above`: the sum of those before.
__device__ __forceinline__ int pick_bucket(Shared &s, unsigned long long target, unsigned long long &above) {
  constexpr int kEach = kBuckets / kThreads;
  unsigned long long mine = 0, all;
#pragma unroll
  for (int i = 0; i < kEach; ++i) mine += s.histogram[threadIdx.x * kEach + i];
  unsigned long long before = block_scan_before(mine, s.wave_whole, all);
  if (threadIdx.x == 0) s.pick = -1;
  __syncthreads();
  if (before < target && before + mine >= target) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const unsigned long long here = s.histogram[threadIdx.x * kEach + i];
      if (before < target && before + here >= target) { s.pick = threadIdx.x * kEach + i; s.pick_above = before; }
      before += here;
    }
  }
  __syncthreads();
  above = s.pick_above;
  const int pick = s.pick;
  __syncthreads();
  return pick;
}
template <typename E, typename W>
__device__ __forceinline__ bool narrow_down(const E *row, const CutParams &p, Shared &s, float top, double temp, unsigned long long target, W weight, Place &place) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t top_key = key_of(top);
  const float per = 64.0f / (float)temp;
  uint32_t low = 0, high = top_key - key_of(-3.4028234663852886e38f);
  unsigned long long above = 0;
  for (int level = 0; low < high; ++level) {
    const uint32_t span = high - low;
    const int shift = span >= kBuckets ? 32 - __builtin_clz(span) - 11 : 0;
    __syncthreads();
    for (int i = threadIdx.x; i < kBuckets; i += kThreads) s.histogram[i] = 0;
    __syncthreads();
    each_piece(row, p, wave, lane, [&](long long, const float (&v)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!has_mass(v[j])) continue;
        const uint32_t distance = top_key - key_of(v[j]);
        if (distance < low || distance > high) continue;
        const int bucket = level == 0 ? bucket_of(v[j], top, per) : (int)((distance - low) >> shift);
        const unsigned long long w = weight(v[j]);
        if (w != 0) atomicAdd(&s.histogram[bucket], w);
      }
    });
    __syncthreads();
    unsigned long long before;
    const int bucket = pick_bucket(s, target - above, before);
    if (bucket < 0) return false;
    above += before;
    if (level == 0) {  // the bucket's ends, by halving: the buckets follow the values
      const auto first_at_least = [&](int b) {
        uint32_t a = low, z = high + 1;  // (the first distance whose bucket is b or more; distances end below 2^32 - 1)
        while (a < z) {
          const uint32_t mid = a + (z - a) / 2;
          if (bucket_of(value_of(top_key - mid), top, per) >= b) z = mid; else a = mid + 1;
        }
        return a;
      };
      const uint32_t from = first_at_least(bucket), to = bucket == kBuckets - 1 ? high : first_at_least(bucket + 1) - 1;
      low = from; high = to;
    } else {
      low += (uint32_t)bucket << shift;
      const uint32_t end = low + ((1u << shift) - 1);
      high = end < high ? end : high;
    }
  }
  // of the equals, as many as it takes
  const unsigned long long each = weight(value_of(top_key - low));
  unsigned long long count = each > 0 ? (target - above + each - 1) / each : 1;
  int equals = 0;
  const auto is_equal = [&](float x) { return has_mass(x) && top_key - key_of(x) == low; };
  each_piece(row, p, wave, lane, [&](long long, const float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) equals += is_equal(v[j]) ? 1 : 0;
  });
  for (int d = 1; d < 64; d <<= 1) equals += __shfl_xor(equals, d);
  __syncthreads();
  if (lane == 0) s.wave_count[wave] = equals;
  if (threadIdx.x == 0) s.pick_index = p.V;
  __syncthreads();
  unsigned long long before = 0;
  for (int w = 0; w < wave; ++w) before += (unsigned)s.wave_count[w];
  if (before < count && before + (unsigned)equals >= count) {  // (uniform: this wavefront has the last)
    each_piece(row, p, wave, lane, [&](long long at, const float (&v)[8]) {
      int mine = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) mine += is_equal(v[j]) ? 1 : 0;
      const int upto = wave_scan(mine, lane);
      unsigned long long here = before + (unsigned)(upto - mine);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (is_equal(v[j]) && ++here == count) s.pick_index = at + j;
      before += (unsigned)__shfl(upto, 63);
    });
  }
  __syncthreads();
  place.distance = low;
  place.index = s.pick_index;
  __syncthreads();
  return true;
}

template <typename E, bool SAMPLE> __device__ __forceinline__ void write_none(const CutParams &p, long long r, E *out) {
  if constexpr (SAMPLE) {
    for (int i = threadIdx.x; i < p.S; i += kThreads) {
      p.tokens[r * p.S + i] = -1;
      if (p.logp != nullptr) p.logp[r * p.S + i] = -INFINITY;
    }
  } else {
    for (long long i = threadIdx.x; i < p.V; i += kThreads) out[i] = narrow<E>(-INFINITY);
  }
  if (threadIdx.x == 0 && p.kept != nullptr) p.kept[r] = 0;
}

template <typename E, bool SAMPLE> __device__ __forceinline__ void cut_row(const CutParams &p, long long r, Shared &s) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const E *row = reinterpret_cast<const E *>(p.x) + r * p.stride;
  E *out = SAMPLE ? nullptr : reinterpret_cast<E *>(p.out) + r * p.out_stride;
  const Cut cut = cut_of(p, r);

  // 1. the largest
  float largest = -INFINITY;
  each_piece(row, p, wave, lane, [&](long long, const float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) largest = fmaxf(largest, has_mass(v[j]) ? v[j] : -INFINITY);
  });
  __syncthreads();  // (the last row's)
  s.largest[threadIdx.x] = largest;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) largest = fmaxf(largest, __shfl_xor(largest, d));
  if (lane == 0) s.wave_float[wave] = largest;
  if (threadIdx.x == 0) s.overflow = 0;
  __syncthreads();
  float top = -INFINITY;
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s.wave_float[w]);
  if (cut.bad || top == -INFINITY) {
    write_none<E, SAMPLE>(p, r, out);
    return;
  }
  const uint32_t top_key = key_of(top);
  const double top_wide = (double)top;
  const double least = cut.min_p > 0.0f ? cut.temp * log((double)cut.min_p) : -INFINITY;  // x - top of what min_p keeps
  const auto over_least = [&](float x) { return (double)x - top_wide >= least; };

  // 2. the list
  bool listed = false;
  int n = 0;
  double all_mass = 0.0;
  const bool by_mass = cut.top_p < 1.0f;
  // (top_p's share is of what top_k leaves, whatever min_p says: where there is a share, min_p does not shorten the list)
  const bool least_too = cut.min_p > 0.0f && !by_mass;
  const bool try_list = least_too || (cut.top_k > 0 ? cut.top_k <= kByCount : by_mass);
  if (try_list) {
    const int wanted = cut.top_k > 0 ? (cut.top_k <= kByCount ? (int)cut.top_k : 0) : by_mass ? kByMass : 0;
    const float bound = wanted > 0 ? bound_of(s.largest, wanted) : -INFINITY;
    const bool need_mass = by_mass && cut.top_k == 0;
    const int waves = (p.tiles + p.tiles_wave - 1) / p.tiles_wave;  // at work
    const int room = kList / (waves <= 1 ? 1 : waves <= 2 ? 2 : waves <= 4 ? 4 : waves <= 8 ? 8 : 16);
    int mine = 0;
    double mass = 0.0;
    each_piece(row, p, wave, lane, [&](long long at, const float (&v)[8]) {
      unsigned hits = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool there = has_mass(v[j]);
        if (need_mass) mass += there ? mass_of(v[j], top_wide, cut.scale) : 0.0;
        if (there && v[j] >= bound && (!least_too || over_least(v[j]))) hits |= 1u << j;
      }
      if (__ballot(hits != 0) != 0) {
        const int count = __popc(hits), upto = wave_scan(count, lane);
        int to = mine + upto - count;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if ((hits >> j & 1) != 0) {
            if (to < room) { s.list_distance[wave * room + to] = top_key - key_of(v[j]); s.list_index[wave * room + to] = (int)(at + j); }
            ++to;
          }
        mine += __shfl(upto, 63);
      }
    });
    if (lane == 0) {
      s.wave_count[wave] = mine;
      if (mine > room) s.overflow = 1;
    }
    if (need_mass) all_mass = block_sum(wave_sum(mass) * (lane == 0 ? 1.0 : 0.0), s.wave_double);
    __syncthreads();
    listed = s.overflow == 0;
    if (listed) {
      // to one run: a wavefront's part to where the parts before it end
      int before = 0;
      for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += s.wave_count[w];
        n += s.wave_count[w];
      }
      const int count = s.wave_count[wave];
      for (int e = lane; e < count; e += 64) s.sorted[before + e] = (unsigned long long)s.list_distance[wave * room + e] << 32 | (unsigned)s.list_index[wave * room + e];
      __syncthreads();
      for (int e = threadIdx.x; e < n; e += kThreads) { s.list_distance[e] = (uint32_t)(s.sorted[e] >> 32); s.list_index[e] = (int)(unsigned)s.sorted[e]; }
      // 3. sorted, by distance and index
      int size = 2;
      while (size < n) size <<= 1;
      __syncthreads();
      for (int e = n + threadIdx.x; e < size; e += kThreads) s.sorted[e] = ~0ULL;
      for (int run = 2; run <= size; run <<= 1)
        for (int gap = run >> 1; gap > 0; gap >>= 1) {
          __syncthreads();
          for (int t = threadIdx.x; t < size / 2; t += kThreads) {
            const int a = 2 * t - (t & (gap - 1)), b = a + gap;
            const unsigned long long va = s.sorted[a], vb = s.sorted[b];
            if ((va > vb) == ((a & run) == 0)) { s.sorted[a] = vb; s.sorted[b] = va; }
          }
        }
      __syncthreads();
      // masses summed along the order, two a thread
      constexpr int kEach = kList / kThreads;
      double m[kEach], total;
      const int e0 = threadIdx.x * kEach;
#pragma unroll
      for (int i = 0; i < kEach; ++i) m[i] = e0 + i < n ? mass_of(value_of(top_key - (uint32_t)(s.sorted[e0 + i] >> 32)), top_wide, cut.scale) : 0.0;
      double sum = block_scan_before(m[0] + m[1], s.wave_double, total);
#pragma unroll
      for (int i = 0; i < kEach; ++i) { sum += m[i]; s.masses[e0 + i] = sum; }
      __syncthreads();
      // how many of them are kept
      int first_n = cut.top_k > 0 && cut.top_k < n ? (int)cut.top_k : n;
      const double of = cut.top_k > 0 ? s.masses[first_n - 1] : all_mass;
      if (by_mass) {
        const double target = (double)cut.top_p * of;
        int a = 0, z = first_n;  // the first whose sum reaches the target
        while (a < z) {
          const int mid = (a + z) / 2;
          if (s.masses[mid] >= target) z = mid; else a = mid + 1;
        }
        if (a >= first_n) {
          if (cut.top_k > 0) a = first_n - 1;
          else listed = over_least(value_of(top_key - (uint32_t)(s.sorted[n - 1] >> 32))) ? false : listed;  // (min_p may cut in the list all the same)
        }
        first_n = a + 1 < first_n ? a + 1 : first_n;
      }
      if (cut.min_p > 0.0f) {
        int a = 0, z = first_n;  // the first that it does not keep
        while (a < z) {
          const int mid = (a + z) / 2;
          if (over_least(value_of(top_key - (uint32_t)(s.sorted[mid] >> 32)))) a = mid + 1; else z = mid;
        }
        first_n = a > 0 ? a : 1;
      }
      if (listed) {
        const unsigned long long last = s.sorted[first_n - 1];
        if (threadIdx.x == 0 && p.kept != nullptr) p.kept[r] = first_n;
        __syncthreads();
        if constexpr (SAMPLE) {
          // masses of the kept summed along the indexes
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            const int e = e0 + i;
            const bool is_kept = e < n && ((unsigned long long)s.list_distance[e] << 32 | (unsigned)s.list_index[e]) <= last;
            m[i] = is_kept ? mass_of(value_of(top_key - s.list_distance[e]), top_wide, cut.scale) : 0.0;
          }
          double along = block_scan_before(m[0] + m[1], s.wave_double, total);
#pragma unroll
          for (int i = 0; i < kEach; ++i) { along += m[i]; s.along[e0 + i] = along; }
          __syncthreads();
          total = s.along[n - 1];
          for (int i = threadIdx.x; i < p.S; i += kThreads) {
            const float u = p.u[r * p.u_stride + i];
            const double target = (double)fmaxf(u, 0.0f) * total;
            int a = 0, z = n;  // the first whose sum is over the target
            while (a < z) {
              const int mid = (a + z) / 2;
              if (s.along[mid] > target) z = mid; else a = mid + 1;
            }
            if (a >= n) {  // the last kept
              a = n - 1;
              while (a > 0 && ((unsigned long long)s.list_distance[a] << 32 | (unsigned)s.list_index[a]) > last) --a;
            }
            p.tokens[r * p.S + i] = u == u ? s.list_index[a] : -1;
            if (p.logp != nullptr)
              p.logp[r * p.S + i] = u == u ? (float)(((double)value_of(top_key - s.list_distance[a]) - top_wide) / cut.temp - log(total)) : -INFINITY;
          }
        } else {
          const uint32_t last_distance = (uint32_t)(last >> 32);
          const int last_index = (int)(unsigned)last;
          each_piece(row, p, wave, lane, [&](long long at, const float (&v)[8]) {
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint32_t d = top_key - key_of(v[j]);
              w[j] = has_mass(v[j]) && (d < last_distance || (d == last_distance && at + j <= last_index)) ? v[j] : -INFINITY;
            }
            if (at < p.V) store_first<8>(out + at, p.V - at, w);
          });
        }
        return;
      }
    }
  }

  // The list does not hold them: narrowed down.
  Place place = {0xFFFFFFFFu, p.V};
  if (cut.top_k > 0) {
    __syncthreads();
    if (!narrow_down(row, p, s, top, cut.temp, (unsigned long long)cut.top_k, [](float) { return 1ULL; }, place)) place = {0xFFFFFFFFu, p.V};
  }
  const auto inside = [&](float x, long long i) {
    const uint32_t d = top_key - key_of(x);
    return has_mass(x) && (d < place.distance || (d == place.distance && i <= place.index));
  };
  if (by_mass) {
    // The unit of the whole numbers: 2^-51 of the largest entry's mass, or more where 62 bits would not hold the row's, which is at most
    // the sum over the threads of their largest one's times their entries.
    const double most = s.largest[threadIdx.x] > -INFINITY ? mass_of(s.largest[threadIdx.x], top_wide, cut.scale) * (double)(p.tiles_wave * (long long)p.pieces_tile * 8) : 0.0;
    const double bound = block_sum(most, s.wave_double);
    int exponent = ilogb(bound) + 1;
    exponent = 62 - exponent < 51 ? 62 - exponent : 51;
    const double unit = ldexp(1.0, exponent);
    const auto whole = [&](float x) { return (unsigned long long)(mass_of(x, top_wide, cut.scale) * unit + 0.5); };
    unsigned long long mass = 0;
    each_piece(row, p, wave, lane, [&](long long at, const float (&v)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) mass += inside(v[j], at + j) ? whole(v[j]) : 0ULL;
    });
    mass = block_sum(mass, s.wave_whole);
    unsigned long long target = (unsigned long long)ceil((double)cut.top_p * (double)mass);
    if (target < 1) target = 1;
    Place by = place;
    if (narrow_down(row, p, s, top, cut.temp, target, whole, by)) place = by;
  }
  if (cut.min_p > 0.0f) {  // the last distance that it keeps
    uint32_t a = 0, z = top_key - key_of(-3.4028234663852886e38f) + 1;
    while (a < z) {
      const uint32_t mid = a + (z - a) / 2;
      if (over_least(value_of(top_key - mid))) a = mid + 1; else z = mid;
    }
    const uint32_t last = a > 0 ? a - 1 : 0;
    if (last < place.distance) place = {last, p.V};
  }
  int count = 0;
  if constexpr (SAMPLE) {
    // masses of the tiles
    __syncthreads();
    double tile = 0.0;
    int piece = 0;
    long long t = (long long)wave * p.tiles_wave;
    each_piece(row, p, wave, lane, [&](long long at, const float (&v)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = inside(v[j], at + j);
        count += in ? 1 : 0;
        tile += in ? mass_of(v[j], top_wide, cut.scale) : 0.0;
      }
      if (++piece == p.pieces_tile || at - lane * 8 + kPiece >= p.V) {
        const double sum = wave_sum(tile);
        if (lane == 0) s.masses[t] = sum;
        ++t; piece = 0; tile = 0.0;
      }
    });
    __syncthreads();
    constexpr int kEach = kMostTiles / kThreads;
    const int t0 = threadIdx.x * kEach;
    double m[kEach], total;
#pragma unroll
    for (int i = 0; i < kEach; ++i) m[i] = t0 + i < p.tiles ? s.masses[t0 + i] : 0.0;
    double along = block_scan_before(m[0] + m[1], s.wave_double, total);
#pragma unroll
    for (int i = 0; i < kEach; ++i) { along += m[i]; s.along[t0 + i] = along; }
    __syncthreads();
    total = s.along[p.tiles - 1];
    for (int i = wave; i < p.S; i += kWaves) {  // a wavefront a token
      const float u = p.u[r * p.u_stride + i];
      const double target = (double)fmaxf(u, 0.0f) * total;
      int a = 0, z = p.tiles;  // the first tile whose sum is over the target
      while (a < z) {
        const int mid = (a + z) / 2;
        if (s.along[mid] > target) z = mid; else a = mid + 1;
      }
      if (a >= p.tiles) {  // the last with mass
        a = p.tiles - 1;
        while (a > 0 && s.along[a] == s.along[a - 1]) --a;
      }
      double before = a > 0 ? s.along[a - 1] : 0.0;
      long long found = -1, last_kept = -1;
      const long long begin = (long long)a * p.pieces_tile * kPiece, end0 = begin + (long long)p.pieces_tile * kPiece, end = end0 < p.V ? end0 : p.V;
      for (long long at0 = begin; at0 < end && found < 0; at0 += kPiece) {
        const long long at = at0 + lane * 8;
        float v[8];
        load_piece(row, at, p.V, v);
        double w[8], mine = 0.0;
        long long last = -1;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool in = inside(v[j], at + j);
          w[j] = in ? mass_of(v[j], top_wide, cut.scale) : 0.0;
          mine += w[j];
          if (in) last = at + j;
        }
        const double upto = wave_scan(mine, lane);
        double here = before + (upto - mine);
        long long first = -1;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          here += w[j];
          if (first < 0 && w[j] > 0.0 && here > target) first = at + j;
        }
        const unsigned long long any = __ballot(first >= 0), some = __ballot(last >= 0);
        if (any != 0) found = __shfl(first, __builtin_ctzll(any));
        if (some != 0) last_kept = __shfl(last, 63 - __builtin_clzll(some));
        before += __shfl(upto, 63);
      }
      if (found < 0) found = last_kept;  // (rounding alone keeps the sum below the target)
      if (lane == 0) {
        const bool number = u == u && found >= 0;
        p.tokens[r * p.S + i] = number ? (int)found : -1;
        if (p.logp != nullptr) p.logp[r * p.S + i] = number ? (float)(((double)widen(row[found]) - top_wide) / cut.temp - log(total)) : -INFINITY;
      }
    }
  } else {
    each_piece(row, p, wave, lane, [&](long long at, const float (&v)[8]) {
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = inside(v[j], at + j);
        count += in ? 1 : 0;
        w[j] = in ? v[j] : -INFINITY;
      }
      if (at < p.V) store_first<8>(out + at, p.V - at, w);
    });
  }
  for (int d = 1; d < 64; d <<= 1) count += __shfl_xor(count, d);
  __syncthreads();
  if (lane == 0) s.wave_count[wave] = count;
  __syncthreads();
  if (threadIdx.x == 0 && p.kept != nullptr) {
    int sum = 0;
    for (int w = 0; w < kWaves; ++w) sum += s.wave_count[w];
    p.kept[r] = sum;
  }
}

template <typename E, bool SAMPLE> __global__ void __launch_bounds__(kThreads) cut_kernel(const CutParams p) {
  __shared__ Shared s;
  for (long long r = blockIdx.x; r < p.R; r += gridDim.x) cut_row<E, SAMPLE>(p, r, s);
}

template <typename A> int check_cut(const A *a) {
  if (a->R < 0 || a->R > (1LL << 24) - 1 || a->V < 1 || a->V > kMaxIndex) return LLC_E_SHAPE;
  if ((a->flags & ~LLC_FLAG_DRY_RUN) != 0) return LLC_E_OPTION;
  if (a->kind != LLC_LOGITS && a->kind != LLC_LOGW) return LLC_E_DTYPE;
  if (!known_type(a->dtype)) return LLC_E_DTYPE;
  if (a->kind == LLC_LOGITS && a->row_temp == nullptr && !(a->temp >= 0x1p-126f && std::isfinite(a->temp))) return LLC_E_TEMP;
  if ((a->row_top_p == nullptr && !(a->top_p > 0.0f && a->top_p <= 1.0f)) || (a->row_min_p == nullptr && !(a->min_p >= 0.0f && a->min_p <= 1.0f)) ||
      (a->row_top_k == nullptr && a->top_k < 0))
    return LLC_E_OPTION;
  return LLC_OK;
}
template <typename A> int fill_cut(const A *a, CutParams &p) {
  if (a->x == nullptr) return LLC_E_NULL;
  if (a->stride_r < 0) return LLC_E_SHAPE;
  if (!fits(a->x, type_size(a->dtype)) || !fits(a->row_temp, 4) || !fits(a->row_top_p, 4) || !fits(a->row_min_p, 4) || !fits(a->row_top_k, 4) || !fits(a->kept, 4)) return LLC_E_ALIGN;
  p.R = a->R; p.V = a->V; p.x = a->x; p.stride = a->stride_r; p.logits = a->kind == LLC_LOGITS ? 1 : 0;
  p.temp = a->temp; p.top_p = a->top_p; p.min_p = a->min_p; p.top_k = a->top_k;
  p.row_temp = a->row_temp; p.row_top_p = a->row_top_p; p.row_min_p = a->row_min_p; p.row_top_k = a->row_top_k;
  p.kept = a->kept;
  const long long pieces = (a->V + kPiece - 1) / kPiece;
  p.pieces_tile = (int)((pieces + kMostTiles - 1) / kMostTiles);
  p.tiles = (int)((pieces + p.pieces_tile - 1) / p.pieces_tile);
  p.tiles_wave = (p.tiles + kWaves - 1) / kWaves;
  return LLC_OK;
}
unsigned row_blocks(long long R) { return R < (long long)kMostRowBlocks ? (unsigned)R : kMostRowBlocks; }

}  // namespace
}  // namespace llc

using namespace llc;

extern "C" int llc_sample(const llc_sample_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  int bad = check_cut(a);
  if (bad != LLC_OK) return bad;
  if (a->S < 0 || a->S > 65535) return LLC_E_SHAPE;
  if (a->R == 0) return LLC_OK;
  if (a->S > 0 && (a->u == nullptr || a->tokens == nullptr)) return LLC_E_NULL;
  CutParams p = {};
  bad = fill_cut(a, p);
  if (bad != LLC_OK) return bad;
  if (a->u_stride_r < 0) return LLC_E_SHAPE;
  if (!fits(a->u, 4) || !fits(a->tokens, 4) || !fits(a->logp, 4)) return LLC_E_ALIGN;
  p.S = (int)a->S; p.u = a->u; p.u_stride = a->u_stride_r; p.tokens = a->tokens; p.logp = a->logp;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    if (a->dtype == LLC_F32) cut_kernel<float, true><<<row_blocks(p.R), kThreads, 0, st>>>(p);
    else cut_kernel<uint16_t, true><<<row_blocks(p.R), kThreads, 0, st>>>(p);
    return hipGetLastError();
  });
}

extern "C" int llc_truncate(const llc_truncate_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  int bad = check_cut(a);
  if (bad != LLC_OK) return bad;
  if (a->R == 0) return LLC_OK;
  if (a->out == nullptr) return LLC_E_NULL;
  CutParams p = {};
  bad = fill_cut(a, p);
  if (bad != LLC_OK) return bad;
  if (a->out_stride_r < a->V || (a->out == a->x && a->R > 1 && a->out_stride_r != a->stride_r)) return LLC_E_SHAPE;
  if (!fits(a->out, type_size(a->dtype))) return LLC_E_ALIGN;
  p.out = a->out; p.out_stride = a->out_stride_r;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    if (a->dtype == LLC_F32) cut_kernel<float, false><<<row_blocks(p.R), kThreads, 0, st>>>(p);
    else cut_kernel<uint16_t, false><<<row_blocks(p.R), kThreads, 0, st>>>(p);
    return hipGetLastError();
  });
}
