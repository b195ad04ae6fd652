// Sampling from a cut distribution with given random numbers, and the cut rows themselves.
//
// The kept entries of a row are a run of its entries in the order of their values (larger first, equal ones by index), so a
// cut is a place of that order: the key of its last entry and that entry's index.  A workgroup takes a row, two are at work on a CU, and
// most rows are read once:
//   1. Each wavefront's first entries are a sample of the row.  A value that the sample has often enough above it, or min_p's from the sample's largest,
//      bounds a list of entries that is likely to hold the kept ones.
//   2. The rest of the row goes by: its largest, the list, in the order of the indexes, and, where a share of the whole mass is
//      asked for, or no cut at all, the masses.
//   3. The list is sorted, its masses are summed along the order, and the cut is read off; the tokens follow from sums along the indexes.
// Rows whose kept entries are too many for the list, by what the sample shows or the list turns out to hold, are read twice more: a histogram of
// counts by value, 256 buckets a unit of ln, shows nearly where the cut is, and a pass with exact masses takes the sums before the buckets about it and lists what is in
// them, or counts them by tiles where thousands are equal.  That confirms the cut or not.  (256 rows of 128 256 in bf16 with settings of their own, a tenth of them so deep: 128 us, some 205 by
// histograms of masses alone; top_k of 3000 of normal rows: 86, some 106.)  What is left is narrowed down by histograms of masses (or counts) of the row, and by the keys' bits.  Tokens follow from the
// sums of tiles of the row.
//
// Masses are exp((x - reference) / temp) in fp64: a border in a run of 128 000 entries that share the mass is hit by rounding otherwise.  (An fp64 multiply-add takes
// as long as one in fp32 here; an entry takes some 23 operations, which at 128 256 entries is 19 us of a CU and about what its share of the memory takes for rows
// in bf16.)  Histograms add masses as whole numbers, whose sum does not depend on the order.
#include "ends.hpp"

namespace llc {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kRoom = 512;        // entries of the list that a wavefront has room for: as many as its part of a row of 4096 has
constexpr int kList = kRoom * kWaves;
constexpr int kFew = kThreads;    // entries that are put in order by counting
constexpr int kBuckets = 2048;    // of a histogram
constexpr int kBucketsLog = 11;
constexpr int kMostTiles = 2048;  // of a row, whose masses LDS holds
constexpr int kPiece = 512;       // entries that a wavefront takes at a time, eight a lane
constexpr int kAhead = 2;         // pieces that it has asked for (four: 300 rows of 50 257 in fp32 cut 31.3 us for 28.8)
constexpr int kSample = 2;        // pieces of a wavefront that the sample has (one: top_k 1500 of 256 rows of 128 256 in bf16 186 us for 43, top_k 40 of 1024 rows 88 for 78)
constexpr int kFine = 8192;       // buckets of the histogram of counts
constexpr float kFinePerUnit = 256.0f;  // of them for each unit of ln
constexpr int kRange = 2048;      // entries about the cut that are listed
// Entries that the list aims at where a share of the mass is asked for (eight tokens of 1024 rows of 128 256 in fp32, top_p 0.9: 162 us; 128: 186, as rows miss it, 400: 173; 256 rows
// in bf16 with settings of their own, three sets of them: 129, 133 and 101), and top_k up to which the list is tried (top_k 1500 of 256 rows: 43 us; by the range 88 of normal rows, and 310 of rows
// that fall as a power of the rank, whose cut lies deeper than the range goes).
constexpr int kByMass = 256, kByCount = 1800;
constexpr long long kMostRowBlocks = 1LL << 22;  // rows of a launch

struct CutParams {
  long long R, V, row0;
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
  float top_p;      // in (0, 1]; 1: off
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
  c.top_p = fminf(top_p, 1.0f);
  if (top_p <= 0.0f) { c.top_k = 1; c.top_p = 1.0f; }  // (no share at all leaves the first entry)
  c.min_p = fminf(fmaxf(min_p, 0.0f), 1.0f);
  return c;
}

// Values as whole numbers in their order, the largest first; both zeros are one.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ ((uint32_t)~((int32_t)u >> 31) & 0x7FFFFFFFu);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float((key & 0x80000000u) != 0 ? key : key ^ 0x7FFFFFFFu); }
constexpr uint32_t kLastKey = 0xFF7FFFFFu;  // of the least finite number
__device__ __forceinline__ bool has_mass(float x) { return fabsf(x) < INFINITY; }

// 2^t, to some 2^-51 of it (the polynomial of degree ten through the Chebyshev points of [-1/2, 1/2]; at 0 it is 1); 0 for -inf.
__device__ __forceinline__ double exp2_of(double t) {
  t = fmax(t, -1200.0);
  const double whole = rint(t), f = t - whole;
  double y = 7.072585949269224e-09;
  y = fma(y, f, 1.0208690299958306e-07);
  y = fma(y, f, 1.321544258792169e-06);
  y = fma(y, f, 1.5252657260200837e-05);
  y = fma(y, f, 0.0001540353044173605);
  y = fma(y, f, 0.0013333558230164974);
  y = fma(y, f, 0.009618129107606888);
  y = fma(y, f, 0.05550410866444772);
  y = fma(y, f, 0.24022650695910097);
  y = fma(y, f, 0.69314718055995);
  y = fma(y, f, 1.0);
  return ldexp(y, (int)whole);
}
__device__ __forceinline__ double mass_of(float x, double reference, double scale) { return exp2_of(((double)x - reference) * scale); }

// Along a wavefront's lanes, without LDS: each lane's value and those of the lanes before, joined; `none`: what joins without effect.
template <int CTRL, int ROWS, typename T> __device__ __forceinline__ T from_lane(T v, T none) {
  constexpr int kWords = sizeof(T) / 4;
  struct Words { int w[kWords]; };
  const Words a = __builtin_bit_cast(Words, v), b = __builtin_bit_cast(Words, none);
  Words r;
#pragma unroll
  for (int i = 0; i < kWords; ++i) r.w[i] = __builtin_amdgcn_update_dpp(b.w[i], a.w[i], CTRL, ROWS, 0xF, false);
  return __builtin_bit_cast(T, r);
}
template <typename T, typename F> __device__ __forceinline__ T wave_join(T v, T none, F join) {
  v = join(v, from_lane<0x111, 0xF>(v, none));  // from one lane before, within rows of 16
  v = join(v, from_lane<0x112, 0xF>(v, none));
  v = join(v, from_lane<0x114, 0xF>(v, none));
  v = join(v, from_lane<0x118, 0xF>(v, none));
  v = join(v, from_lane<0x142, 0xA>(v, none));  // the first and third row's last to the rows after
  v = join(v, from_lane<0x143, 0xC>(v, none));  // the second row's last to the third and fourth
  return v;
}
template <typename T> __device__ __forceinline__ T lane_value(T v, int lane) {  // (lane: uniform)
  constexpr int kWords = sizeof(T) / 4;
  struct Words { int w[kWords]; };
  Words a = __builtin_bit_cast(Words, v);
#pragma unroll
  for (int i = 0; i < kWords; ++i) a.w[i] = __builtin_amdgcn_readlane(a.w[i], lane);
  return __builtin_bit_cast(T, a);
}
template <typename T> __device__ __forceinline__ T wave_scan(T v) { return wave_join(v, T(0), [](T a, T b) { return a + b; }); }
template <typename T> __device__ __forceinline__ T wave_sum(T v) { return lane_value(wave_scan(v), 63); }

struct Shared {
  union {
    struct {
      alignas(16) uint32_t list_key[kList];
      int list_index[kList];
    };
    int equals[kMostTiles];  // of tiles, then summed along the indexes
    alignas(16) uint32_t fine[kFine];
  };
  union {
    unsigned long long histogram[kBuckets];
    double along[kList > kMostTiles ? kList : kMostTiles];  // masses summed along the indexes: of the list's entries, or of tiles
    double masses[kFew];                                    // summed along the order
  };
  unsigned long long few[kFew], sorted[kFew];  // key and index (kFew is a multiple of eight)
  uint32_t sample[kThreads];                   // a histogram of the sample's largest
  union {
    double wave_double[kWaves];
    unsigned long long wave_whole[kWaves];
  };
  int wave_count[kWaves];
  float wave_high[kWaves], wave_low[kWaves];
  int n_few;
  int fine_first, fine_last, fine_at;
  unsigned long long pick_above;
  int pick;
  uint32_t pick_index;
};

// Over the threads' values: the sum of those before, and of all.
template <typename T> __device__ __forceinline__ T block_scan_before(T v, T *s_wave, T &all) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T upto = wave_scan(v);
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

// A lane's entries of a piece as they lie in memory.
template <typename E> struct Raw;
template <> struct Raw<float> { float4_any a, b; };
template <> struct Raw<uint16_t> { word4_any a; };
template <typename E> __device__ __forceinline__ void load_eight(Raw<E> &r, const E *from) {
  r.a = *reinterpret_cast<const decltype(r.a) *>(from);
  if constexpr (sizeof(E) == 4) r.b = *reinterpret_cast<const decltype(r.b) *>(from + 4);
}
// Where a lane's eight of a piece begin: of the last ones, where the piece is the row's end; with an entry a lane in rows of fewer than eight.
__device__ __forceinline__ unsigned begin_of(unsigned piece, unsigned lane, unsigned V) {
  const unsigned at = piece + lane * 8;
  return V < 8 ? lane : at + 8 <= V ? at : V - 8;
}
template <typename E> __device__ __forceinline__ Raw<E> load_raw(const E *row, unsigned piece, unsigned lane, unsigned V) {
  Raw<E> r;
  if (piece + kPiece <= V) {  // (uniform)
    load_eight(r, row + piece + lane * 8);
  } else if (V >= 8) {
    load_eight(r, row + begin_of(piece, lane, V));
  } else {
    const E one = row[lane < V ? lane : 0];
    if constexpr (sizeof(E) == 4) r.a[0] = one; else r.a[0] = (uint32_t)one;
  }
  return r;
}
__device__ __forceinline__ float max_of_three(float a, float b, float c) {  // (of numbers: as it is, without a step that quiets NaNs first)
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// The entries as numbers: -inf those without mass, and those that another lane has.
template <typename E> __device__ __forceinline__ void widen_raw(const Raw<E> &r, unsigned piece, unsigned lane, unsigned V, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(E) == 4) {
      v[j] = r.a[j]; v[j + 4] = r.b[j];
    } else {
      split_pair(r.a[j], v[2 * j], v[2 * j + 1]);
    }
  }
  float nought = 0.0f;  // (times 0 nothing is left of numbers, and a NaN of anything else)
#pragma unroll
  for (int j = 0; j < 8; ++j) nought = fmaf(v[j], 0.0f, nought);
  if (__ballot(nought != 0.0f) != 0 || piece + kPiece > V) {  // (uniform: something else, or the row's end)
    const unsigned others = V < 8 ? (lane < V ? 0 : 8) : piece + lane * 8 - begin_of(piece, lane, V), mine = V < 8 ? 1 : 8;
#pragma unroll
    for (unsigned j = 0; j < 8; ++j) {
      const bool is = has_mass(v[j]) & (j >= others) & (j < mine);
      v[j] = is ? v[j] : -INFINITY;
    }
  }
}
__device__ __forceinline__ float largest_of(const float (&v)[8]) {
  return max_of_three(max_of_three(v[0], v[1], v[2]), max_of_three(v[3], v[4], v[5]), max_of_three(v[6], v[7], v[7]));
}
// A wavefront's entries.
struct Part {
  unsigned first, last;
};
__device__ __forceinline__ Part part_of(const CutParams &p, int wave) {
  const unsigned long long each = (unsigned long long)p.tiles_wave * (unsigned)p.pieces_tile * kPiece, first = (unsigned)wave * each, last = first + each, V = (unsigned long long)p.V;
  return {(unsigned)(first < V ? first : V), (unsigned)(last < V ? last : V)};
}
// Its pieces in turn, of which DEPTH are asked for ahead: f(piece, index of a lane's first, its eight).  (A load goes to the place of the piece that was taken: copies from place
// to place would wait for what was asked for last.)
template <typename E, int DEPTH> struct Ring {
  Raw<E> raw[DEPTH];
  __device__ __forceinline__ void fill(const E *row, unsigned V, Part part, int lane) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
      if (part.first + i * kPiece < part.last) raw[i] = load_raw(row, part.first + i * kPiece, lane, V);
  }
  template <typename F> __device__ __forceinline__ void run(const E *row, unsigned V, Part part, int lane, F f) {
#pragma unroll 1
    for (unsigned at0 = part.first; at0 < part.last; at0 += DEPTH * kPiece) {  // (uniform)
#pragma unroll
      for (int i = 0; i < DEPTH; ++i) {
        const unsigned at = at0 + i * kPiece;
        if (at < part.last) {
          float v[8];
          widen_raw(raw[i], at, lane, V, v);
          if (at + DEPTH * kPiece < part.last) raw[i] = load_raw(row, at + DEPTH * kPiece, lane, V);
          f(at, begin_of(at, lane, V), v);
        }
      }
    }
  }
};
template <typename E, typename F> __device__ __forceinline__ void each_piece(const E *row, const CutParams &p, Part part, int lane, F f) {
  Ring<E, 2> ring;
  ring.fill(row, (unsigned)p.V, part, lane);
  ring.run(row, (unsigned)p.V, part, lane, f);
}
// The same of a row or of the list in its place (n entries, one piece a wavefront, whose indexes are their places in the list).
struct Listed {
  const Shared *s;  // null: the row
  int n;
};
template <typename E, typename F> __device__ __forceinline__ void each_piece_of(Listed l, const E *row, const CutParams &p, Part part, int lane, int wave, F f) {
  const unsigned V = (unsigned)p.V;
  if (l.s != nullptr) part = {(unsigned)wave * kPiece, wave * kPiece < l.n ? (unsigned)wave * kPiece + 1 : (unsigned)wave * kPiece};
  constexpr int kTwo = 2;
#pragma unroll 1
  for (unsigned at0 = part.first; at0 < part.last; at0 += kTwo * kPiece) {  // (uniform)
    Raw<E> raw[kTwo];
    float v[kTwo][8];
    unsigned at[kTwo];
    if (l.s != nullptr) {
      at[0] = at0 + lane * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[0][j] = (int)at[0] + j < l.n ? value_of(l.s->list_key[at[0] + j]) : -INFINITY;
    } else {
#pragma unroll
      for (int i = 0; i < kTwo; ++i)
        if (at0 + i * kPiece < part.last) raw[i] = load_raw(row, at0 + i * kPiece, lane, V);
#pragma unroll
      for (int i = 0; i < kTwo; ++i)
        if (at0 + i * kPiece < part.last) {
          at[i] = begin_of(at0 + i * kPiece, lane, V);
          widen_raw(raw[i], at0 + i * kPiece, lane, V, v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kTwo; ++i)
      if (at0 + i * kPiece < part.last) f(at[i], v[i]);
  }
}
// The masses of a lane's entries, four at a time: all at once would take more registers than there are.
__device__ __forceinline__ double mass_of_eight(const float (&v)[8], double reference, double scale) {
  double sum = 0.0;
#pragma unroll
  for (int h = 0; h < 8; h += 4) {
    double m[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = mass_of(v[h + j], reference, scale);
    sum += (m[0] + m[1]) + (m[2] + m[3]);
    __builtin_amdgcn_sched_barrier(0);
  }
  return sum;
}

// The same, and of those before `until` among places on the histogram of counts.
__device__ __forceinline__ double mass_of_eight(const float (&v)[8], const float (&at)[8], float until, double reference, double scale, double &before) {
  double sum = 0.0;
#pragma unroll
  for (int h = 0; h < 8; h += 4) {
    double m[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = mass_of(v[h + j], reference, scale);
    sum += (m[0] + m[1]) + (m[2] + m[3]);
#pragma unroll
    for (int j = 0; j < 4; ++j) before += at[h + j] < until ? m[j] : 0.0;
    __builtin_amdgcn_sched_barrier(0);
  }
  return sum;
}

// The lanes before, and those of all: how many entries are marked.
__device__ __forceinline__ int marked_before(const bool (&hit)[8], int &all) {
  int before = 0;
  all = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned long long m = __ballot(hit[j]);
    before = __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, before));
    all += __popcll(m);
  }
  return before;
}

// The list: each wavefront's entries in a part of its own, in the order of their indexes; once they are more than it has room for, they are counted only.
struct Lister {
  int count;
  // Entries from `bound` on (a number); here: a lane's largest.  Where no lane has two, which is nearly always, a lane's one is its largest.
  __device__ __forceinline__ void add_from(float bound, Shared &s, int wave, unsigned at, const float (&v)[8], float here) {
    const unsigned long long lanes = __ballot(here >= bound);
    if (lanes == 0) return;  // (uniform)
    int mine = 0, which = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool hit = v[j] >= bound;
      mine += hit ? 1 : 0;
      which = hit ? j : which;
    }
    if (__ballot(mine > 1) == 0) {  // (uniform)
      const int to = wave * kRoom + __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, count));
      count += __popcll(lanes);
      if (mine != 0 && count <= kRoom) {
        s.list_key[to] = key_of(here);
        s.list_index[to] = (int)at + which;
      }
      return;
    }
    bool hit[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) hit[j] = v[j] >= bound;
    add(s, wave, at, v, hit);
  }
  __device__ __forceinline__ void add(Shared &s, int wave, unsigned at, const float (&v)[8], const bool (&hit)[8]) {
    int all, to = wave * kRoom + count + marked_before(hit, all);
    count += all;
    if (count > kRoom) return;  // (uniform)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (hit[j]) {
        s.list_key[to] = key_of(v[j]);
        s.list_index[to] = (int)(at + j);
        ++to;
      }
  }
};
// The wavefronts' parts to one run of n; false where one did not hold its entries.
__device__ __forceinline__ bool join_list(Shared &s, int count, int lane, int wave, int &n) {
  if (lane == 0) s.wave_count[wave] = count;
  __syncthreads();
  int before = 0;
  bool whole = true;
  n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int c = s.wave_count[w];
    if (w < wave) before += c;
    n += c;
    whole = whole && c <= kRoom;
  }
  if (!whole) return false;
  uint32_t key[kRoom / 64];
  int index[kRoom / 64];
#pragma unroll
  for (int i = 0; i < kRoom / 64; ++i)
    if (i * 64 < count) { key[i] = s.list_key[wave * kRoom + i * 64 + lane]; index[i] = s.list_index[wave * kRoom + i * 64 + lane]; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRoom / 64; ++i)
    if (i * 64 + lane < count) { s.list_key[before + i * 64 + lane] = key[i]; s.list_index[before + i * 64 + lane] = index[i]; }
  __syncthreads();
  return true;
}
// few[0..n) in order to sorted[0..n): a thread counts what is before its entry.
__device__ __forceinline__ void sort_few(Shared &s, int n) {
  __syncthreads();
  if ((int)threadIdx.x >= n && (int)threadIdx.x < ((n + 7) & ~7)) s.few[threadIdx.x] = ~0ULL;
  __syncthreads();
  if ((int)(threadIdx.x & ~63u) < n) {  // (uniform)
    const unsigned long long mine = s.few[threadIdx.x];
    int rank = 0;
    for (int i = 0; i < n; i += 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) rank += s.few[i + j] < mine ? 1 : 0;
    }
    if ((int)threadIdx.x < n) s.sorted[rank] = mine;
  }
  __syncthreads();
}
// The same of the list's first n entries, by key and place: 32 bits are compared, with the entry's key for those behind it, with the next for those before.
__device__ __forceinline__ void sort_list(Shared &s, int n) {
  const int e = threadIdx.x;
  if (e >= n && e < ((n + 31) & ~31)) s.list_key[e] = ~0u;
  __syncthreads();
  if ((int)(threadIdx.x & ~63u) < n) {  // (uniform)
    const uint32_t mine = e < n ? s.list_key[e] : 0;
    int rank = 0;
    for (int i = 0; i < n; i += 32) {  // (uniform)
      uint4 k[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) k[j] = *reinterpret_cast<const uint4 *>(s.list_key + i + 4 * j);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t to = mine + (i + 4 * j < (e & ~3) ? 1 : 0);
        rank += (k[j].x < to ? 1 : 0) + (k[j].y < to ? 1 : 0) + (k[j].z < to ? 1 : 0) + (k[j].w < to ? 1 : 0);
      }
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) {  // equals before it among its four
      const int f = (e & ~3) + j;
      rank += f < e && s.list_key[f] == mine ? 1 : 0;
    }
    if (e < n) s.sorted[rank] = (unsigned long long)mine << 32 | (unsigned)e;
  }
  __syncthreads();
}

// The place of the order where the weights' sum reaches `target`: a whole number's histogram by values, then the entries of the bucket.
struct Place {
  uint32_t key;     // of the last entry
  uint32_t index;
};
__device__ __forceinline__ int bucket_of(float x, float top, float per) {
  const float at = (top - x) * per;  // (both roundings keep the order; an infinite `per` gives NaN at the top itself, and that 0)
  return at >= (float)(kBuckets - 1) ? kBuckets - 1 : (int)fmaxf(at, 0.0f);
}
// The bucket where the sum of those up to it and of `above` reaches the target; -1: none.  before: the sum of those in front.  share > 0: the target is that share of all.
__device__ __forceinline__ int pick_bucket(Shared &s, float share, unsigned long long above, unsigned long long &target, unsigned long long &before) {
  constexpr int kEach = kBuckets / kThreads;
  unsigned long long mine = 0, all;
#pragma unroll
  for (int i = 0; i < kEach; ++i) mine += s.histogram[threadIdx.x * kEach + i];
  unsigned long long upto = above + block_scan_before(mine, s.wave_whole, all);
  if (share > 0.0f) {
    target = (unsigned long long)ceil((double)share * (double)all);
    if (target < 1) target = 1;
  }
  if (threadIdx.x == 0) s.pick = -1;
  __syncthreads();
  if (upto < target && upto + mine >= target) {
#pragma unroll 1
    for (int i = 0; i < kEach; ++i) {
      const unsigned long long here = s.histogram[threadIdx.x * kEach + i];
      if (upto < target && upto + here >= target) { s.pick = threadIdx.x * kEach + i; s.pick_above = upto - above; }
      upto += here;
    }
  }
  __syncthreads();
  before = s.pick_above;
  const int pick = s.pick;
  __syncthreads();
  return pick;
}
// Where a bucket of the histogram of counts lies: bf16 numbers are a power of two of buckets apart, which would be in few banks.
__device__ __forceinline__ int place_of(int bucket) { return bucket ^ (bucket >> 5); }
// The range of the histogram of counts that holds the cut, by count or by what the buckets' masses about are; false: none, or the last bucket's.
// (Of a bucket's entries each mass is within 2^-8.5 of its middle's, on either side; 2^-12 of the whole on either side of a share is far more than that leaves in
// rows of many entries.  The range is only where the cut is looked for.)  many: more entries than the list's masses have room for, in a single bucket then.
__device__ __forceinline__ bool pick_range(Shared &s, float share, unsigned wanted, int &first, int &last, bool &many) {
  constexpr int kEach = kFine / kThreads;
  const int b0 = threadIdx.x * kEach;
  const float rate = -1.442695f / kFinePerUnit;
  const auto weight = [&](int b) { return share > 0.0f ? (double)((float)s.fine[place_of(b)] * __builtin_amdgcn_exp2f(((float)b + 0.5f) * rate)) : (double)s.fine[place_of(b)]; };
  double mine = 0.0, all;
#pragma unroll 4
  for (int i = 0; i < kEach; ++i) mine += weight(b0 + i);
  double upto = block_scan_before(mine, s.wave_double, all);
  const double from = share > 0.0f ? fmax((double)share - 0x1p-12, 0.0) * all : (double)wanted;
  const double to = share > 0.0f ? fmin((double)share + 0x1p-12, 0.5 * (1.0 + (double)share)) * all : (double)wanted;
  const double here = share > 0.0f ? (double)share * all : (double)wanted;
  if (threadIdx.x == 0) { s.fine_first = from > 0.0 ? kFine : 0; s.fine_last = s.fine_at = kFine - 1; }
  __syncthreads();
  if (upto < to && upto + mine >= from) {
#pragma unroll 1
    for (int i = 0; i < kEach; ++i) {
      const double next = upto + weight(b0 + i);
      if (upto < from && next >= from) atomicMin(&s.fine_first, b0 + i);  // (where roundings let two cross, the first)
      if (upto < to && next >= to) atomicMin(&s.fine_last, b0 + i);
      if (upto < here && next >= here) atomicMin(&s.fine_at, b0 + i);
      upto = next;
    }
  }
  __syncthreads();
  first = s.fine_first;
  last = s.fine_last;
  int mine_within = 0, total;
#pragma unroll 4
  for (int i = 0; i < kEach; ++i) mine_within += b0 + i >= first && b0 + i <= last ? (int)s.fine[place_of(b0 + i)] : 0;
  block_scan_before(mine_within, s.wave_count, total);
  many = total > kRange;
  if (many) first = last = s.fine_at;  // the one bucket (of numbers in 16 bits, thousands may be equal)
  __syncthreads();
  return first <= last && last < kFine - 1;
}
// Weights: of an entry 1, or its mass in units, rounded.
struct Weight {
  bool counted;
  double top, scale, unit;
  __device__ __forceinline__ unsigned long long of(float x) const { return counted ? 1ULL : (unsigned long long)(mass_of(x, top, scale) * unit + 0.5); }
};
// Entries behind `until` take no part.  The target is `share` of the sum of all, or, where that is 0, `wanted`.  False: the sum of all does not reach it.
template <typename E>
__device__ __forceinline__ bool narrow_down(Listed l, const E *row, const CutParams &p, Shared &s, Part part, float top, double temp, Place until, const Weight weight,
                                            float share, unsigned long long wanted, Place &place) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float per = 64.0f / (float)temp;  // (the last bucket has what is 32 units of ln and more below the top)
  uint32_t low = key_of(top), high = kLastKey;
  unsigned long long above = 0, target = wanted;
  const auto inside = [&](uint32_t key, unsigned i) { return key < until.key || (key == until.key && i <= until.index); };
#pragma unroll 1
  for (int level = 0; level == 0 || low < high; ++level) {
    const uint32_t span = high - low;
    const int shift = span >= kBuckets ? 32 - __builtin_clz(span) - kBucketsLog : 0;
    __syncthreads();
    for (int i = threadIdx.x; i < kBuckets; i += kThreads) s.histogram[i] = 0;
    if (threadIdx.x == 0) s.n_few = 0;
    __syncthreads();
    each_piece_of(l, row, p, part, lane, wave, [&](unsigned at, const float (&v)[8]) {
      bool in[8], any = false;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t key = key_of(v[j]);
        in[j] = key >= low && key <= high && inside(key, at + j);
        any = any || in[j];
      }
      if (__ballot(any) == 0) return;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned long long w = in[j] ? weight.of(v[j]) : 0;
        if (w != 0) atomicAdd(&s.histogram[level == 0 ? bucket_of(v[j], top, per) : (int)((key_of(v[j]) - low) >> shift)], w);
      }
      if (level > 0) {
        int all, to = marked_before(in, all), from = 0;
        if (lane == 0) from = atomicAdd(&s.n_few, all);
        to += lane_value(from, 0);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (in[j]) {
            if (to < kFew) s.few[to] = (unsigned long long)key_of(v[j]) << 32 | (unsigned)(at + j);
            ++to;
          }
      }
    });
    __syncthreads();
    const int n = s.n_few;
    if (level > 0 && n <= kFew) {  // few entries: in order, they show the place
      sort_few(s, n);
      unsigned long long all;
      const int e = threadIdx.x;
      const unsigned long long w = e < n ? weight.of(value_of((uint32_t)(s.sorted[e] >> 32))) : 0, before = above + block_scan_before(w, s.wave_whole, all);
      if (threadIdx.x == 0) s.pick = n - 1;
      __syncthreads();
      if (before < target && before + w >= target) s.pick = e;
      __syncthreads();
      const unsigned long long last = s.sorted[s.pick];
      place.key = (uint32_t)(last >> 32);
      place.index = (uint32_t)last;
      __syncthreads();
      return true;
    }
    unsigned long long before;
    const int bucket = pick_bucket(s, level == 0 ? share : 0.0f, above, target, before);
    if (bucket < 0) return false;
    above += before;
    if (level == 0) {  // the bucket's ends, by halving: the buckets follow the values
      uint32_t ends[2];
#pragma unroll 1
      for (int b = 0; b < 2; ++b) {
        uint32_t a = low, z = high + 1;  // (the first key whose bucket is at least the one, or the next; keys end below 2^32 - 1)
        while (a < z) {
          const uint32_t mid = a + (z - a) / 2;
          if (bucket_of(value_of(mid), top, per) >= bucket + b) z = mid; else a = mid + 1;
        }
        if (b == 0) ends[0] = a; else ends[1] = a - 1;
      }
      low = ends[0]; high = ends[1];
      if constexpr (sizeof(E) == 2) {  // (to the keys that bf16 numbers have, of which a bucket may have a single one)
        low = low < 0x80000000u ? low | 0xFFFFu : (low + 0xFFFFu) & 0xFFFF0000u;
        high = high < 0x80000000u ? ((high + 1) & 0xFFFF0000u) - 1 : high & 0xFFFF0000u;
      }
    } else {
      low += (uint32_t)bucket << shift;
      const uint32_t end = low + ((1u << shift) - 1);
      high = end < high ? end : high;
    }
  }
  // of the equals, as many as it takes
  const unsigned long long each = weight.of(value_of(low));
  const unsigned long long count = each > 0 ? (target - above + each - 1) / each : 1;
  int equals = 0;
  unsigned long long before = 0;
#pragma unroll 1
  for (int turn = 0; turn < 2; ++turn) {  // how many each wavefront has; then the one
    if (turn == 1) {
      __syncthreads();
      if (lane == 0) s.wave_count[wave] = equals;
      if (threadIdx.x == 0) s.pick_index = (uint32_t)p.V;
      __syncthreads();
      for (int w = 0; w < wave; ++w) before += (unsigned)s.wave_count[w];
      if (before >= count || before + (unsigned)equals < count) break;  // (uniform: another wavefront has the last)
    }
    each_piece_of(l, row, p, part, lane, wave, [&](unsigned at, const float (&v)[8]) {
      bool hit[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) hit[j] = key_of(v[j]) == low;
      int all;
      unsigned long long here = before + (unsigned)marked_before(hit, all);
      if (turn == 0) {
        equals += all;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (hit[j] && ++here == count) s.pick_index = at + j;
        before += (unsigned)all;
      }
    });
  }
  __syncthreads();
  place.key = low;
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

// A value that `wanted` of the threads' largest entries of the sample reach (-inf where fewer have one); top: the largest of them.
__device__ __forceinline__ float bound_of(Shared &s, float mine, float top, float least, int wanted) {
  const float per = (float)(kThreads - 1) / (top - least);
  s.sample[threadIdx.x] = 0;
  __syncthreads();
  const int at = (int)fminf(fmaxf((top - mine) * per, 0.0f), (float)(kThreads - 1));
  if (mine > -INFINITY) atomicAdd(&s.sample[at], 1u);
  if (threadIdx.x == 0) s.pick = -1;
  __syncthreads();
  unsigned long long all;
  const unsigned long long here = s.sample[threadIdx.x], before = block_scan_before(here, s.wave_whole, all);
  if (before < (unsigned)wanted && before + here >= (unsigned)wanted) s.pick = threadIdx.x;
  __syncthreads();
  const int pick = s.pick;
  // (a bucket further down than the one: what rounding has put there is above it)
  return pick < 0 ? -INFINITY : top == least ? top : top - (float)(pick + 2) / per;
}

template <typename E, bool SAMPLE, bool RANGE> __device__ __forceinline__ void cut_row(const CutParams &p, long long r, Shared &s) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const E *row = reinterpret_cast<const E *>(p.x) + r * p.stride;
  E *out = SAMPLE ? nullptr : reinterpret_cast<E *>(p.out) + r * p.out_stride;
  const Part part = part_of(p, wave);
  // 1. the sample
  Ring<E, kAhead> ring;
  ring.fill(row, (unsigned)p.V, part, lane);
  const Cut cut = cut_of(p, r);
  const float first_u = SAMPLE && (int)threadIdx.x < p.S ? p.u[r * p.u_stride + threadIdx.x] : 0.0f;  // (of a list's tokens: waited for later)
  const bool by_mass = cut.top_p < 1.0f;
  // (top_p's share is of what top_k leaves, whatever min_p says: where there is a share, min_p does not shorten the list)
  const bool least_too = cut.min_p > 0.0f && !by_mass;
  const double least = cut.min_p > 0.0f ? cut.temp * log((double)cut.min_p) : -INFINITY;  // x - top of what min_p keeps
  const bool uncut = !by_mass && cut.top_k == 0 && cut.min_p == 0.0f;
  const bool try_list = least_too || (cut.top_k > 0 ? cut.top_k <= kByCount : by_mass);
  const bool need_mass = by_mass && cut.top_k == 0;
  const bool can_range = RANGE && (need_mass || (cut.top_k > 0 && !by_mass));
  bool deep = !try_list && can_range;  // (no list would hold the kept entries)
  float largest = -INFINITY;
#pragma unroll
  for (int i = 0; i < kSample; ++i) {
    if (part.first + i * kPiece < part.last) {
      float v[8];
      widen_raw(ring.raw[i], part.first + i * kPiece, lane, (unsigned)p.V, v);
      largest = max_of_three(largest, largest_of(v), largest);
    }
  }
  const auto block_ends = [&](float high, float low, float &top, float &end) {
    high = lane_value(wave_join(high, -INFINITY, [](float a, float b) { return fmaxf(a, b); }), 63);
    low = lane_value(wave_join(low, INFINITY, [](float a, float b) { return fminf(a, b); }), 63);
    __syncthreads();
    if (lane == 0) { s.wave_high[wave] = high; s.wave_low[wave] = low; }
    __syncthreads();
    top = s.wave_high[0]; end = s.wave_low[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) { top = fmaxf(top, s.wave_high[w]); end = fminf(end, s.wave_low[w]); }
    top = lane_value(top, 0);  // (a scalar: it is needed to the end, and vector registers are short)
  };
  float reference, sample_low;
  block_ends(largest, largest > -INFINITY ? largest : INFINITY, reference, sample_low);
  if (cut.bad) reference = -INFINITY;
  else if (reference == -INFINITY) {  // (uniform: the sample has no mass)
    float high = -INFINITY;
    each_piece(row, p, part, lane, [&](unsigned, unsigned, const float (&v)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) high = fmaxf(high, v[j]);
    });
    block_ends(high, INFINITY, reference, sample_low);
  }
  if (reference == -INFINITY) {
    write_none<E, SAMPLE>(p, r, out);
    return;
  }
  // What the sample is of the row decides how far down the list goes: so that the kept entries are in it but for some chance in a million of
  // a row in random order.  (A row that they are not in after all takes the longer way.)
  float bound = -INFINITY;
  bool by_least = false;  // the bound is min_p's
  if (try_list) {
    const long long sampled = (long long)kThreads * kSample * 8;
    const float share = p.V <= sampled ? 1.0f : (float)sampled / (float)p.V;
    const bool counted = cut.top_k > 0 && cut.top_k <= kByCount;
    if (counted || need_mass) {
      const float expected = share * (float)(counted ? (int)cut.top_k : kByMass);
      const int wanted = share == 1.0f ? (int)expected : (int)(expected + (counted ? 4.5f * sqrtf(expected) + 6.0f : 1.0f));
      bound = bound_of(s, largest, reference, sample_low, wanted);
      if (RANGE && need_mass && share < 1.0f) {  // a list that has less than half of the mass asked for in the sample is not made: of seven tenths, rows would be read once more for nothing more often (eight tokens of 1024 of 128 256 in fp32: 175 us for 162)
        float above = 0.0f, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kSample; ++i) {
          if (part.first + i * kPiece < part.last) {
            float v[8];
            widen_raw(ring.raw[i], part.first + i * kPiece, lane, (unsigned)p.V, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float m = __builtin_amdgcn_exp2f((v[j] - reference) * (float)cut.scale);
              sum += m;
              above += v[j] >= bound ? m : 0.0f;
            }
          }
        }
        above = wave_sum(above);
        sum = wave_sum(sum);
        __syncthreads();
        if (lane == 0) { s.wave_high[wave] = above; s.wave_low[wave] = sum; }
        __syncthreads();
        above = sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) { above += s.wave_high[w]; sum += s.wave_low[w]; }
        deep = above < 0.5f * cut.top_p * sum;
      }
    }
    if (least_too) {
      const float to = (float)((double)reference + least);
      const float below = to - fabsf(to) * 0x1p-23f - 1e-38f;  // (not above what min_p keeps, whatever the rounding)
      if (below > bound || !(counted || need_mass)) { by_least = true; bound = below > bound ? below : bound; }
    }
  }

  // 2. the row goes by
  float high = -INFINITY;
  double mass = 0.0;
  Lister list = {0};
  int piece = 0, count = 0;  // (count: the wavefront's kept)
  long long tile = (long long)wave * p.tiles_wave;
  const double reference_wide = (double)reference;
  const float from_number = fmaxf(bound, -3.4028234663852886e38f);
  const auto see = [&](unsigned from, unsigned at, const float (&v)[8]) {
    const float here = largest_of(v);
    high = max_of_three(high, here, high);
    if (need_mass || (SAMPLE && uncut)) mass += mass_of_eight(v, reference_wide, cut.scale);
    if (SAMPLE && uncut) {
#pragma unroll
      for (int j = 0; j < 8; ++j) count += __popcll(__ballot(v[j] > -INFINITY));
    }
    if (try_list) list.add_from(from_number, s, wave, at, v, here);
    if (SAMPLE && uncut && (++piece == p.pieces_tile || from + kPiece >= p.V)) {
      const double sum = wave_sum(mass);
      if (lane == 0) s.along[tile] = sum;
      ++tile; piece = 0; mass = 0.0;
    }
  };
  float top = reference, unused;
  if (!deep) {
    ring.run(row, (unsigned)p.V, part, lane, see);
    block_ends(high, 0.0f, top, unused);
  }
  double top_wide = (double)top;
  // (what was summed relative to the sample's largest is no number where the row's is 1024 units of log2 over that (900, which leaves room for a row's sum), as small temperatures
  // bring about: it is summed again, relative to the row's, and a share of it is not looked for in the list, which the longer way does without)
  const bool far = (top_wide - reference_wide) * cut.scale > 900.0, summed = uncut && !far;  // (summed: an uncut row's tiles are, relative to the sample's)
  const auto over_least = [&](float x) { return (double)x - top_wide >= least; };

  // 3. the list
  int n = 0;
  double all_mass = 0.0;
  if (need_mass && !deep) all_mass = block_sum(mass, s.wave_double) * exp2_of((reference_wide - top_wide) * cut.scale);
  bool listed = try_list && !deep && !(need_mass && far) && join_list(s, list.count, lane, wave, n);
  if (listed && cut.top_k > n && bound > -INFINITY && !by_least) listed = false;  // (there are more below the bound)
  Place place = {0xFFFFFFFFu, (uint32_t)p.V};  // (of the list's entries: their places in the list)
  // What the list does not show is looked for in a range about the cut, and what that does not show narrowed down in the row.
  bool ranged = false, found = uncut;
  double above_mass = 0.0;  // of the entries before the range
  int above = 0, above_mine = 0;  // (of all; of the thread's)
  int equal_kept = 0;  // of equal entries in the range, where they are many; the mass of each
  double each_equal = 0.0;
  const auto look_in_few = [&]() __attribute__((always_inline)) {
    found = true;
    const int e = threadIdx.x;
    sort_list(s, n);
    int first_n = cut.top_k > 0 && cut.top_k - above < n ? (int)cut.top_k - above : n;
    if (by_mass) {  // masses summed along the order
      const double mine = e < n ? mass_of(value_of((uint32_t)(s.sorted[e] >> 32)), top_wide, cut.scale) : 0.0;
      double total;
      const double before = block_scan_before(mine, s.wave_double, total);
      if (e < n) s.masses[e] = before + mine;
      __syncthreads();
      const double target = (double)cut.top_p * (cut.top_k > 0 ? s.masses[first_n - 1] : all_mass) - above_mass;
      int a = 0, z = first_n;  // the first whose sum reaches the target
      while (a < z) {
        const int mid = (a + z) / 2;
        if (s.masses[mid] >= target) z = mid; else a = mid + 1;
      }
      // (the list may end before; min_p may cut in it all the same)
      if (ranged) found = a < first_n && (above == 0 || target > 0.0);
      else if (a >= first_n && cut.top_k == 0 && bound > -INFINITY) found = !over_least(value_of((uint32_t)(s.sorted[n - 1] >> 32)));
      first_n = a + 1 < first_n ? a + 1 : first_n;
    }
    const unsigned long long last = s.sorted[first_n - 1];
    place = {(uint32_t)(last >> 32), (uint32_t)last};
  };
  if (!RANGE && listed && n <= kFew) look_in_few();
#pragma unroll 1
  for (int turn = deep ? 1 : 0; turn < 3 && !found; ++turn) {
    int lane = threadIdx.x & 63;
    if constexpr (RANGE) asm volatile("" : "+v"(lane));  // (or every address of a turn would be kept in registers from before the first)
    if (turn == 0 && (!listed || (!RANGE && n <= kFew))) continue;
    if (turn == 1) {
      listed = false;
      if (!can_range) continue;
      if constexpr (RANGE) {
      // a histogram of counts shows where the cut is, nearly
      // (from the row's largest on where it is known, else from 12 units of ln over the sample's; what is over that counts as if it were there, which shows the cut all the same where it
      // has nearly all of the mass)
      const float per = kFinePerUnit / (float)cut.temp, base = deep ? reference + 12.0f * kFinePerUnit / per : top;
      __syncthreads();
      for (int i = threadIdx.x * 4; i < kFine; i += kThreads * 4) *reinterpret_cast<uint4 *>(s.fine + i) = make_uint4(0, 0, 0, 0);
      __syncthreads();
      each_piece(row, p, part, lane, [&](unsigned, unsigned, const float (&v)[8]) {
        high = max_of_three(high, largest_of(v), high);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float at = (base - v[j]) * per;
          if (v[j] > -INFINITY) atomicAdd(&s.fine[place_of((int)fminf(fmaxf(at, 0.0f), (float)(kFine - 1)))], 1u);
        }
      });
      block_ends(high, 0.0f, top, unused);
      top_wide = (double)top;
      int first, last;
      bool many;
      if (!pick_range(s, by_mass ? cut.top_p : 0.0f, (unsigned)cut.top_k, first, last, many)) continue;
      if (sizeof(E) == 4 && many) continue;
      // the masses of all and of those before the range, by tiles, and a list of the range
      const float from = first > 0 ? (float)first : -INFINITY, until = (float)(last + 1);
      const bool with_mass = SAMPLE || by_mass;
      double sum = 0.0, sum_before = 0.0, tile_before = 0.0;
      int equals = 0;
      float equal_high = -INFINITY, equal_low = INFINITY;
      piece = above = 0;
      tile = (long long)wave * p.tiles_wave;
      list.count = 0;
      each_piece(row, p, part, lane, [&](unsigned from_piece, unsigned at, const float (&v)[8]) {
        float to[8];
        bool hit[8], any = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          to[j] = (base - v[j]) * per;
          above += to[j] < from ? 1 : 0;
          hit[j] = !(to[j] < from) & !(to[j] >= until);
          any = any | hit[j];
        }
        if (with_mass) sum += mass_of_eight(v, to, from, top_wide, cut.scale, tile_before);
        if (sizeof(E) == 2 && many) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            equals += hit[j] ? 1 : 0;
            equal_high = hit[j] ? fmaxf(equal_high, v[j]) : equal_high;
            equal_low = hit[j] ? fminf(equal_low, v[j]) : equal_low;
          }
        } else if (__ballot(any) != 0) {
          list.add(s, wave, at, v, hit);
        }
        if (++piece == p.pieces_tile || from_piece + kPiece >= p.V) {
          if constexpr (SAMPLE) {
            const double before = wave_sum(tile_before);
            if (lane == 0) s.along[kRange + tile] = before;
          }
          if (sizeof(E) == 2 && many) {
            equals = wave_sum(equals);
            if (lane == 0) s.equals[tile] = equals;
            equals = 0;
          }
          ++tile;
          sum_before += tile_before;
          piece = 0; tile_before = 0.0;
        }
      });
      all_mass = block_sum(sum, s.wave_double);
      above_mass = block_sum(sum_before, s.wave_double);
      const int mine = above;
      block_scan_before(mine, s.wave_count, above);
      __syncthreads();
      above_mine = mine;
      if (sizeof(E) == 2 && many) {
        block_ends(equal_high, equal_low, equal_high, equal_low);
        if (equal_high != equal_low) continue;
        // of the equals, as many as it takes: the tile with the last of them, then its index
        each_equal = mass_of(equal_high, top_wide, cut.scale);
        const double some = by_mass ? ceil(((double)cut.top_p * all_mass - above_mass) / each_equal) : (double)(cut.top_k - above);
        constexpr int kEach = kMostTiles / kThreads;
        int of[kEach], mine_equal = 0, total;
#pragma unroll
        for (int i = 0; i < kEach; ++i) { const int t = threadIdx.x * kEach + i; of[i] = t < p.tiles ? s.equals[t] : 0; mine_equal += of[i]; }
        int upto = block_scan_before(mine_equal, s.wave_count, total);
        if (!(some >= 1.0 && some <= (double)total)) continue;  // (or the range is not where the cut is)
        equal_kept = (int)some;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int t = threadIdx.x * kEach + i;
          if (upto < equal_kept && upto + of[i] >= equal_kept) { s.pick = t; s.n_few = upto; }
          upto += of[i];
          if (t < p.tiles) s.equals[t] = upto;
        }
        __syncthreads();
        const unsigned begin = (unsigned)s.pick * (unsigned)p.pieces_tile * kPiece;
        int before = s.n_few;
        if (wave == 0) {
          for (int i = 0; i < p.pieces_tile && before < equal_kept; ++i) {  // (uniform; it is within the row)
            const unsigned at0 = begin + (unsigned)i * kPiece;
            float v[8];
            bool hit[8];
            widen_raw(load_raw(row, at0, lane, (unsigned)p.V), at0, lane, (unsigned)p.V, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) hit[j] = v[j] == equal_high;
            int all, here = before + marked_before(hit, all);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (hit[j] && ++here == equal_kept) s.pick_index = begin_of(at0, lane, (unsigned)p.V) + j;
            before += all;
          }
        }
        __syncthreads();
        place = {key_of(equal_high), s.pick_index};
        found = true;
        continue;
      }
      listed = ranged = join_list(s, list.count, lane, wave, n);
      }
      if (!listed) continue;
    }
    if (turn == 2) {
      listed = ranged = false;
      above = 0;
    }
    place = {0xFFFFFFFFu, (uint32_t)p.V};
    found = true;
    if constexpr (RANGE) {
      if (listed && n <= kFew) {
        look_in_few();
        continue;
      }
    }
    const Listed in = {listed ? &s : nullptr, n};
#pragma unroll 1
    for (int by = 0; by < 2; ++by) {  // by count, then by mass
      if (by == 0 ? cut.top_k == 0 : !by_mass) continue;
      Weight weight = {by == 0, top_wide, cut.scale, 1.0};
      unsigned long long wanted = (unsigned long long)(cut.top_k - above);
      float share = 0.0f;
      if (by == 1) {
        // The unit of the whole numbers: 2^-51 of the largest entry's mass, or more where 62 bits would not hold the row's, which is at most
        // the sum over the threads of their largest one's times their entries.
        const long long entries = (long long)p.tiles_wave * p.pieces_tile * 8;
        const int room = 62 - (ilogb(block_sum(mass_of(high, top_wide, cut.scale) * (double)entries, s.wave_double)) + 1);
        weight.unit = ldexp(1.0, room < 51 ? room : 51);
        if (listed && need_mass) {
          const double target = ceil(((double)cut.top_p * all_mass - above_mass) * weight.unit);
          if (ranged && above > 0 && !(target > 0.0)) { found = false; break; }
          wanted = target > 1.0 ? (unsigned long long)target : 1;
        } else {
          share = cut.top_p;
        }
      }
      Place to;
      if (narrow_down(in, row, p, s, part, top, cut.temp, place, weight, share, wanted, to)) place = to;
      else found = !(listed && need_mass && bound > -INFINITY) && !ranged;  // (the list ends before)
    }
  }
  if (!listed) ranged = false;
  if (ranged) place.index = (uint32_t)s.list_index[place.index];
  bool tiled = ranged || equal_kept > 0;  // the tiles' masses before the range and the list are all it takes
  if (cut.min_p > 0.0f) {  // the last key that it keeps
    uint32_t a = key_of(top), z = kLastKey + 1;
    while (a < z) {
      const uint32_t mid = a + (z - a) / 2;
      if (over_least(value_of(mid))) a = mid + 1; else z = mid;
    }
    const uint32_t last = a > key_of(top) ? a - 1 : a;
    if (last < place.key) { place = {last, (uint32_t)p.V}; tiled = false; }
  }
  const auto kept_at = [&](int e) { return s.list_key[e] < place.key || (s.list_key[e] == place.key && (unsigned)e <= place.index); };
  if (listed && !ranged) {
    const int each = (n + kThreads - 1) / kThreads, e0 = threadIdx.x * each, e1 = e0 + each < n ? e0 + each : n;
    __syncthreads();
    if constexpr (SAMPLE) {
      // masses of the kept summed along the indexes
      double sum = 0.0, total;
      int mine = 0;
#pragma unroll 1
      for (int e = e0; e < e1; ++e) {
        if (kept_at(e)) { sum += mass_of(value_of(s.list_key[e]), top_wide, cut.scale); ++mine; }
        s.along[e] = sum;
      }
      const double before = block_scan_before(sum, s.wave_double, total);
#pragma unroll 1
      for (int e = e0; e < e1; ++e) s.along[e] += before;
      mine = wave_sum(mine);
      if (lane == 0) s.wave_count[wave] = mine;
      __syncthreads();
      if (threadIdx.x == 0 && p.kept != nullptr) {
        int kept = 0;
        for (int w = 0; w < kWaves; ++w) kept += s.wave_count[w];
        p.kept[r] = kept;
      }
      total = s.along[n - 1];
      const double log_total = log(total);
      for (int i = threadIdx.x; i < p.S; i += kThreads) {
        const float u = i < kThreads ? first_u : p.u[r * p.u_stride + i];
        const double target = u >= 1.0f ? (double)INFINITY : (double)fmaxf(u, 0.0f) * total;
        int a = 0, z = n;  // the first whose sum is over the target
        while (a < z) {
          const int mid = (a + z) / 2;
          if (s.along[mid] > target) z = mid; else a = mid + 1;
        }
        a = a < n ? a : n - 1;  // (none: the last kept)
        while (a > 0 && !kept_at(a)) --a;  // (sums are not equal where nothing lies between: those of two threads are rounded in different orders)
        p.tokens[r * p.S + i] = u == u ? s.list_index[a] : -1;
        if (p.logp != nullptr) p.logp[r * p.S + i] = u == u ? (float)(((double)value_of(s.list_key[a]) - top_wide) / cut.temp - log_total) : -INFINITY;
      }
    } else {
      // the row is written as nothing, then the kept entries as they were (out may be x: they are read before)
      constexpr int kEach = kList / kThreads;
      E was[kEach];
      int mine = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int e = i * kThreads + threadIdx.x;
        if (e < n && kept_at(e)) { was[i] = row[s.list_index[e]]; ++mine; }
      }
      mine = wave_sum(mine);
      if (lane == 0) s.wave_count[wave] = mine;
      __syncthreads();
      const float none[8] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY};
      for (long long at = part.first + lane * 8; at < part.last; at += kPiece) store_first<8>(out + at, p.V - at, none);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int e = i * kThreads + threadIdx.x;
        if (e < n && kept_at(e)) out[s.list_index[e]] = was[i];
      }
      if (threadIdx.x == 0 && p.kept != nullptr) {
        int kept = 0;
        for (int w = 0; w < kWaves; ++w) kept += s.wave_count[w];
        p.kept[r] = kept;
      }
    }
    return;
  }

  // The row's entries, where the list does not hold the kept ones.
  const auto inside = [&](float x, unsigned i) {
    const uint32_t key = key_of(x);
    return x > -INFINITY && (key < place.key || (key == place.key && i <= place.index));
  };
  if constexpr (SAMPLE) {
    // masses of the tiles
    const double by_wide = summed ? reference_wide : top_wide;
    __syncthreads();
    double *along = s.along + (tiled ? kRange : 0);
    if (equal_kept > 0 && tiled) {
      count = wave_sum(above_mine) + (wave == 0 ? equal_kept : 0);
    } else if (tiled) {  // masses of the range's kept, summed along the indexes
      const int each = (n + kThreads - 1) / kThreads, e0 = threadIdx.x * each, e1 = e0 + each < n ? e0 + each : n;
      double sum = 0.0, unused_total;
      int mine = above_mine;
#pragma unroll 1
      for (int e = e0; e < e1; ++e) {
        if (inside(value_of(s.list_key[e]), (unsigned)s.list_index[e])) { sum += mass_of(value_of(s.list_key[e]), top_wide, cut.scale); ++mine; }
        s.along[e] = sum;
      }
      const double before = block_scan_before(sum, s.wave_double, unused_total);
#pragma unroll 1
      for (int e = e0; e < e1; ++e) s.along[e] += before;
      count = wave_sum(mine);
    } else if (!summed) {
      double sum_tile = 0.0;
      piece = count = 0;
      tile = (long long)wave * p.tiles_wave;
      each_piece(row, p, part, lane, [&](unsigned from, unsigned at, const float (&v)[8]) {
        float kept[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool in = inside(v[j], at + j);
          count += __popcll(__ballot(in));
          kept[j] = in ? v[j] : -INFINITY;
        }
        sum_tile += mass_of_eight(kept, top_wide, cut.scale);
        if (++piece == p.pieces_tile || from + kPiece >= p.V) {
          const double sum = wave_sum(sum_tile);
          if (lane == 0) s.along[tile] = sum;
          ++tile; piece = 0; sum_tile = 0.0;
        }
      });
    }
    __syncthreads();
    constexpr int kEach = kMostTiles / kThreads;
    const int t0 = threadIdx.x * kEach;
    double m[kEach], total, sum = 0.0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) { m[i] = t0 + i < p.tiles ? along[t0 + i] : 0.0; sum += m[i]; }
    sum = block_scan_before(sum, s.wave_double, total);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      sum += m[i];
      double with = 0.0;
      if (tiled && equal_kept > 0) {
        if (t0 + i < p.tiles) with = each_equal * (double)(s.equals[t0 + i] < equal_kept ? s.equals[t0 + i] : equal_kept);
      } else if (tiled && t0 + i < p.tiles) {  // the range's up to the tile's end
        const long long end = (long long)(t0 + i + 1) * p.pieces_tile * kPiece;
        int a = 0, z = n;
        while (a < z) {
          const int mid = (a + z) / 2;
          if (s.list_index[mid] >= end) z = mid; else a = mid + 1;
        }
        if (a > 0) with = s.along[a - 1];
      }
      along[t0 + i] = sum + with;
    }
    __syncthreads();
    total = along[p.tiles - 1];
    for (int i = wave; i < p.S; i += kWaves) {  // a wavefront a token
      const float u = p.u[r * p.u_stride + i];
      double target = u >= 1.0f ? (double)INFINITY : (double)fmaxf(u, 0.0f) * total;
      int a = 0, z = p.tiles;  // the first tile whose sum is over the target
      while (a < z) {
        const int mid = (a + z) / 2;
        if (along[mid] > target) z = mid; else a = mid + 1;
      }
      a = a < p.tiles ? a : p.tiles - 1;
      long long found = -1;
      // (a tile without kept entries, which rounding alone may lead to and a number of 1 does: the last kept entry before it)
      for (; found < 0 && a >= 0; --a, target = INFINITY) {
        double before = a > 0 ? along[a - 1] : 0.0;
        long long last_kept = -1;
        const long long begin = (long long)a * p.pieces_tile * kPiece, end0 = begin + (long long)p.pieces_tile * kPiece, end = end0 < p.V ? end0 : p.V;
        for (long long at0 = begin; at0 < end && found < 0; at0 += kPiece) {
          const long long at = begin_of(at0, lane, p.V);
          float v[8];
          widen_raw(load_raw(row, at0, lane, p.V), at0, lane, p.V, v);
          double w[8], mine = 0.0;
          long long last = -1;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool in = inside(v[j], at + j);
            w[j] = mass_of(in ? v[j] : -INFINITY, by_wide, cut.scale);
            mine += w[j];
            if (in) last = at + j;
          }
          const double upto = wave_scan(mine);
          double here = before + (upto - mine);
          long long hit = -1;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            here += w[j];
            if (hit < 0 && w[j] > 0.0 && here > target) hit = at + j;
          }
          const unsigned long long any = __ballot(hit >= 0), some = __ballot(last >= 0);
          if (any != 0) found = lane_value(hit, __builtin_ctzll(any));
          if (some != 0) last_kept = lane_value(last, 63 - __builtin_clzll(some));
          before += lane_value(upto, 63);
        }
        if (found < 0) found = last_kept;  // (rounding alone keeps the sum below the target)
      }
      if (lane == 0) {
        const bool number = u == u && found >= 0;
        p.tokens[r * p.S + i] = number ? (int)found : -1;
        if (p.logp != nullptr) p.logp[r * p.S + i] = number ? (float)(((double)widen(row[found]) - by_wide) / cut.temp - log(total)) : -INFINITY;
      }
    }
  } else {
    each_piece(row, p, part, lane, [&](unsigned from, unsigned at, const float (&v)[8]) {
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = inside(v[j], at + j);
        count += __popcll(__ballot(in));
        w[j] = in ? v[j] : -INFINITY;
      }
      if (from + kPiece <= p.V) {
        store_some<8>(out + at, w);
      } else {  // (a lane's own alone)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (p.V < 8 ? j == 0 && at < p.V : at + j >= from + lane * 8) out[at + j] = narrow<E>(w[j]);
      }
    });
  }
  __syncthreads();
  if (lane == 0) s.wave_count[wave] = count;
  __syncthreads();
  if (threadIdx.x == 0 && p.kept != nullptr) {
    int sum = 0;
    for (int w = 0; w < kWaves; ++w) sum += s.wave_count[w];
    p.kept[r] = sum;
  }
  __syncthreads();
}

template <typename E, bool SAMPLE, bool RANGE> __global__ void __launch_bounds__(kThreads, 4) cut_kernel(const CutParams p) {
  __shared__ Shared s;
  cut_row<E, SAMPLE, RANGE>(p, p.row0 + blockIdx.x, s);
}
template <bool SAMPLE> hipError_t launch_cut(CutParams p, int dtype, hipStream_t st) {
  hipError_t e = hipSuccess;
  // Whether rows may look for their cut in a range;
  // the kernel that can needs more registers than there are, which costs rows that never do a tenth of their time (1024 of 128 256 in bf16, top_k 1: 72 us for 63 when both were tried).
  const bool by_mass = p.row_top_p != nullptr || p.top_p < 1.0f;
  const bool range = (by_mass && (p.row_top_k != nullptr || p.top_k == 0)) || p.row_top_k != nullptr || p.top_k > kByCount;
  for (; p.row0 < p.R && e == hipSuccess; p.row0 += kMostRowBlocks) {
    const unsigned blocks = (unsigned)(p.R - p.row0 < kMostRowBlocks ? p.R - p.row0 : kMostRowBlocks);
    if (dtype == LLC_F32) range ? cut_kernel<float, SAMPLE, true><<<blocks, kThreads, 0, st>>>(p) : cut_kernel<float, SAMPLE, false><<<blocks, kThreads, 0, st>>>(p);
    else range ? cut_kernel<uint16_t, SAMPLE, true><<<blocks, kThreads, 0, st>>>(p) : cut_kernel<uint16_t, SAMPLE, false><<<blocks, kThreads, 0, st>>>(p);
    e = hipGetLastError();
  }
  return e;
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
  return between_events(a->ev_begin, a->ev_end, st, [&] { return launch_cut<true>(p, a->dtype, st); });
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
  return between_events(a->ev_begin, a->ev_end, st, [&] { return launch_cut<false>(p, a->dtype, st); });
}
