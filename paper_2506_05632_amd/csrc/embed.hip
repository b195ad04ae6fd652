// Embedding lookup with scaling, and its gradient by sorted tokens.  Both move rows and compute next to nothing: memory
// bounds them.
//
// Gradient: grad[n] = scale * sum over t with tokens[t] == n of g[t].  Floating-point atomics would make the sums' order,
// and so their bits, a matter of timing; instead the positions are sorted by token first (a stable counting sort), and a row of the
// gradient is one wavefront's, or several wavefronts' by columns, which adds its tokens' rows up in registers in the order of their positions, in fp32, and
// writes it once.  Rows that no token names are written as zeros by a launch of their own.
// Tokens as in text name a few rows very often: a row of more than kWindow tokens is added up by windows of kWindow
// sorted positions, each a wavefront's, whose partial sums (fp32, in the workspace) a last launch joins.  A window touches at most
// two such rows, the one it starts in and the one it ends in, so two partial rows a window are room enough, and a window's place
// follows from its number: which wavefront adds what is not decided at run time.  (Of few windows the row's last wavefront at work does the joining; the order is the same.)
#include "ends.hpp"

namespace llc {
namespace {

constexpr int kWindow = 32;       // sorted positions a wavefront adds up (16: 16 384 x 4096 sums and joins 41 + 7 us for 46 + 5; all by one token x 1537 52.6 for 44.1)
constexpr int kAhead = 4;         // rows that are fetched together (8 take the registers of three wavefronts a SIMD: 65 536 tokens 402 us for 338)
constexpr int kJoinThreads = 1024;
constexpr int kFewJoins = 16;     // windows of a row that a wavefront joins by itself
constexpr int kMostRange = 896;   // rows of the table that a workgroup of the sort takes (its counters: 60 KB of LDS)
constexpr long long kMostRows = 1LL << 27;

// A sorted position: its number, the row it names, and where that row's places start and how many they are.
struct alignas(16) Place {
  int t, row, start, count;
};

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
  int team_log;             // log2 of the wavefronts that share a row's columns (divisions would take longer than a short row)
  // the gradient's
  int range;                // rows a workgroup of the sort takes
  Place *places;            // [T] the positions by token
  int32_t *starts;          // [N + 1] where a row's places start
  float *partial;           // [windows][2][D]
  int *arrived;             // [windows][team] wavefronts that are done with the long row that starts in a window; null: a launch of its own joins them
  long long windows;
  int join_each;            // windows that a wavefront of the joining launch looks at, 64 at most
  unsigned window_blocks, sum_blocks;  // of the summing launch: windows, then sorted positions
};

// ---- lookup: a wavefront, or several by columns, a token
template <typename A, typename B> __global__ void __launch_bounds__(kBlock) embed_kernel(const EmbedParams p) {
  constexpr int N = kWide<A>;
  const long long wave = (long long)blockIdx.x * (kBlock / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long t = wave >> p.team_log;
  if (t >= p.T) return;
  const long long n = p.tokens[t * p.tok_stride];
  const bool there = n >= 0 && n < p.N;
  const A *from = reinterpret_cast<const A *>(p.from) + (there ? n : 0) * p.from_stride;
  B *to = reinterpret_cast<B *>(p.to) + t * p.to_stride;
  for (long long d = ((wave & ((1 << p.team_log) - 1)) * 64 + (threadIdx.x & 63)) * N; d < p.D; d += 64LL * N << p.team_log) {
    float v[N] = {};
    if (there) load_first<N>(from + d, p.D - d, v);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= p.scale;
    if (!there) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = 0.0f;  // (not -0)
    }
    store_first<N>(to + d, p.D - d, v);
  }
}

// ---- the sort: a workgroup takes a range of rows, reads all tokens twice (they lie in the caches) and needs
// nothing from the other workgroups: where its rows start follows from how many tokens name a row below.
__device__ __forceinline__ int add_over_wave(int v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

constexpr int kSortAhead = 16;  // groups of 64 tokens that are fetched together
__device__ __forceinline__ void load_ids(const EmbedParams &p, long long t, long long until, unsigned (&id)[kSortAhead]) {
#pragma unroll
  for (int u = 0; u < kSortAhead; ++u) id[u] = t + u * 64 < until ? (unsigned)p.tokens[(t + u * 64) * p.tok_stride] : 0xFFFFFFFFu;
}

template <int WAVES> __global__ void __launch_bounds__(WAVES * 64) embed_sort_kernel(const EmbedParams p) {
  extern __shared__ int counts[];  // [WAVES][range], then where the rows' places start, [range + 1]
  __shared__ int s_wave[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), range = p.range;
  int *begins = counts + WAVES * range;
  const long long low = (long long)blockIdx.x * range;
  const int rows = (int)(p.N - low < range ? p.N - low : range);
  // a wavefront takes consecutive positions, so that the order of the positions is kept
  const long long share = ((p.T + WAVES - 1) / WAVES + 63) & ~63LL;
  const long long from = wave * share, until = from + share < p.T ? from + share : p.T;
  if (p.arrived != nullptr && blockIdx.x == 0)
    for (int i = tid; i < (int)p.windows << p.team_log; i += WAVES * 64) p.arrived[i] = 0;
  unsigned id[kSortAhead];
  load_ids(p, from + lane, until, id);
  for (int i = tid; i < WAVES * range; i += WAVES * 64) counts[i] = 0;
  __syncthreads();
  int *mine = counts + wave * range;
  int below = 0;
  for (long long t0 = from; t0 < until; t0 += 64 * kSortAhead) {
    if (t0 != from) load_ids(p, t0 + lane, until, id);
#pragma unroll
    for (int u = 0; u < kSortAhead; ++u) {
      below += id[u] < (unsigned long long)low ? 1 : 0;
      if (id[u] - (unsigned)low < (unsigned)rows) atomicAdd(&mine[id[u] - (unsigned)low], 1);
    }
  }
  below = add_over_wave(below);
  if (lane == 0) s_wave[wave] = below;
  __syncthreads();
  int base = 0;
  for (int w = 0; w < WAVES; ++w) base += s_wave[w];
  // a thread takes a row at a time: its tokens, and how many come before it
  for (int r0 = 0; r0 < rows; r0 += WAVES * 64) {
    const int r = r0 + tid;
    int total = 0;
    if (r < rows)
      for (int w = 0; w < WAVES; ++w) total += counts[w * range + r];
    int upto = total;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int at = base + upto - total;
    for (int w = 0; w < WAVES; ++w) {
      at += w < wave ? s_wave[w] : 0;
      base += s_wave[w];
    }
    if (r < rows) {
      p.starts[low + r] = at;
      begins[r] = at;
      for (int w = 0; w < WAVES; ++w) {
        const int n = counts[w * range + r];
        counts[w * range + r] = at;
        at += n;
      }
    }
  }
  if (tid == 0) {
    begins[rows] = base;
    if (low + rows == p.N) p.starts[p.N] = base;
  }
  __syncthreads();
  for (long long t0 = from; t0 < until; t0 += 64 * kSortAhead) {
    if (share > 64 * kSortAhead) load_ids(p, t0 + lane, until, id);  // (else they are still there)
#pragma unroll
    for (int u = 0; u < kSortAhead; ++u) {
      const unsigned at_row = id[u] - (unsigned)low;
      unsigned long long left = __ballot(at_row < (unsigned)rows);
      while (left != 0) {  // (uniform; one round for every row that the 64 tokens name)
        const unsigned row = __builtin_amdgcn_readlane(at_row, __builtin_ctzll(left));
        const unsigned long long same = __ballot(at_row == row);
        const int first = mine[row], begin = begins[row];  // (the first is this wavefront's own counter)
        if (at_row == row)
          p.places[first + (int)__builtin_popcountll(same & ((1ull << lane) - 1))] =
              Place{(int)(t0 + u * 64 + lane), (int)(low + row), begin, begins[row + 1] - begin};
        mine[row] = first + (int)__builtin_popcountll(same);  // (by every lane: each has read it itself)
        left &= ~same;
      }
    }
  }
}

// ---- sums
// The N columns that a lane adds up.  Every lane of a wavefront stays at work, also one whose columns lie past the end: the rows' numbers are read
// out of the lanes, and a lane that a branch has left holds nothing that could be relied on.  So a lane that the end cuts short, or that
// lies past it, adds up the row's last N columns and keeps what is its own of them.
template <int N> struct Columns {
  long long first;  // the columns that are read
  long long mine;   // the lane's own begin here (at `first`, or after it)
  long long left;   // columns from `first` on
};
// ALL: rows have N columns at least.
template <bool ALL, int N> __device__ __forceinline__ Columns<N> columns_at(long long d, long long D) {
  const long long first = ALL && d > D - N ? D - N : d;
  return Columns<N>{first, d, D - first};
}
template <bool ALL, int N, typename B> __device__ __forceinline__ void load_columns(const B *row, const Columns<N> &c, float (&v)[N]) {
  if constexpr (ALL) load_some<N>(row + c.first, v);
  else load_first<N>(row + c.first, c.left, v);
}
template <int N, bool STREAM, typename B> __device__ __forceinline__ void store_columns(B *row, const Columns<N> &c, const float (&v)[N]) {
  if (c.first == c.mine && c.left >= N) {
    if constexpr (STREAM) stream_some<N>(row + c.first, v);
    else store_some<N>(row + c.first, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (c.first + i >= c.mine && i < c.left) row[c.first + i] = narrow<B>(v[i]);
}

// The next K of the places whose positions lane i of t holds.
template <bool ALL, int K, typename A, int N>
__device__ __forceinline__ void add_some(const EmbedParams &p, const Columns<N> &c, int t, int &j, float (&sum)[N]) {
  float v[K][N];
#pragma unroll
  for (int u = 0; u < K; ++u)
    load_columns<ALL, N>(reinterpret_cast<const A *>(p.from) + (long long)__builtin_amdgcn_readlane(t, j + u) * p.from_stride, c, v[u]);
#pragma unroll
  for (int u = 0; u < K; ++u)
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] += v[u][i];
  j += K;
}
// The rows of g at n places, at most 64, in the order of the positions, which the lanes of t hold.
template <bool ALL, typename A, int N>
__device__ __forceinline__ void add_positions(const EmbedParams &p, const Columns<N> &c, int t, int n, float (&sum)[N]) {
  int j = 0;
  while (n - j >= kAhead) add_some<ALL, kAhead, A, N>(p, c, t, j, sum);
  if (n - j >= 2) add_some<ALL, 2, A, N>(p, c, t, j, sum);
  if (n - j >= 1) add_some<ALL, 1, A, N>(p, c, t, j, sum);
}

// What a row of the gradient becomes.  (ADD is known to the compiler: a load under a condition would be waited for at once.)
template <bool ADD, int N> __device__ __forceinline__ void add_scaled(const EmbedParams &p, const float (&before)[N], float (&sum)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = ADD ? fmaf(sum[i], p.scale, before[i]) : sum[i] * p.scale;
}

// A wavefront's columns of one row, or of a window's share of a row, whose n positions lane i of t holds.
template <bool ALL, typename A>
__device__ __forceinline__ void sum_window(const EmbedParams &p, float *to, int t, int n, long long d0, long long step, int lane) {
  constexpr int N = kWide<A>;
  for (long long d = d0; d < p.D; d += step) {  // (uniform)
    const Columns<N> c = columns_at<ALL, N>(d + lane * N, p.D);
    float sum[N] = {};
    add_positions<ALL, A, N>(p, c, t, n, sum);
    store_columns<N, false>(to, c, sum);
  }
}
template <bool ALL, bool ADD, typename A, typename B>
__device__ __forceinline__ void sum_row(const EmbedParams &p, B *to, int t, int n, long long d0, long long step, int lane) {
  constexpr int N = kWide<A>;
  for (long long d = d0; d < p.D; d += step) {  // (uniform)
    const Columns<N> c = columns_at<ALL, N>(d + lane * N, p.D);
    float sum[N] = {}, before[N] = {};
    if constexpr (ADD) load_columns<ALL, N>(to, c, before);
    add_positions<ALL, A, N>(p, c, t, n, sum);
    add_scaled<ADD, N>(p, before, sum);
    store_columns<N, true>(to, c, sum);
  }
}

// A wavefront's columns of a long row whose windows are all summed, the same whoever comes last.
template <bool ALL, bool ADD, typename A, typename B>
__device__ __forceinline__ void join_row(const EmbedParams &p, int row, int start, int count, long long d0, long long step, int lane) {
  constexpr int N = kWide<A>;
  const int first = start / kWindow, last = (start + count - 1) / kWindow;
  const int slot = start != first * kWindow ? 1 : 0;  // (of the first window)
  B *to = reinterpret_cast<B *>(p.to) + (long long)row * p.to_stride;
  for (long long d = d0; d < p.D; d += step) {  // (uniform)
    const Columns<N> c = columns_at<ALL, N>(d + lane * N, p.D);
    float sum[N] = {}, before[N] = {};
    if constexpr (ADD) load_columns<ALL, N>(to, c, before);
    for (int v = first; v <= last; v += kAhead) {
      float part[kAhead][N];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {  // (without a branch, the last one again where there are fewer)
        const int at = min(v + u, last);
        load_columns<ALL, N>(p.partial + (at * 2LL + (at == first ? slot : 0)) * p.D, c, part[u]);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += v + u <= last ? part[u][i] : 0.0f;
    }
    add_scaled<ADD, N>(p, before, sum);
    store_columns<N, true>(to, c, sum);
  }
}

template <typename A, typename B, bool ADD> __global__ void __launch_bounds__(kBlock) embed_sum_kernel(const EmbedParams p) {
  constexpr int N = kWide<A>;
  const int in_block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const long long wave = (long long)blockIdx.x * (kBlock / 64) + in_block, step = 64LL * N << p.team_log;
  const long long item = wave >> p.team_log, d0 = (wave & ((1 << p.team_log) - 1)) * 64 * N;
  const long long windows = (long long)p.window_blocks * (kBlock / 64) >> p.team_log,
                  sums = (long long)p.sum_blocks * (kBlock / 64) >> p.team_log;
  if (blockIdx.x < p.window_blocks) {
    const long long begin = item * kWindow;
    if (begin >= p.T) return;
    const int total = p.starts[p.N];
    const int room = (int)(p.T - begin < kWindow ? p.T - begin : kWindow);
    const Place mine = p.places[begin + (lane < room ? lane : room - 1)];  // (not written from place `total` on)
    if (begin >= total) return;
    const int n = total - begin < room ? (int)(total - begin) : room;  // the window's places
    const int a_end = __builtin_amdgcn_readlane(mine.start, 0) + __builtin_amdgcn_readlane(mine.count, 0);
    const int b_begin = __builtin_amdgcn_readlane(mine.start, n - 1);
    const bool a_long = __builtin_amdgcn_readlane(mine.count, 0) > kWindow;
    const bool b_long = b_begin > begin && __builtin_amdgcn_readlane(mine.count, n - 1) > kWindow;
    for (int slot = 0; slot < 2; ++slot) {
      if (slot == 0 ? !a_long : !b_long) continue;
      float *to = p.partial + (item * 2 + slot) * p.D;
      const int skip = slot == 0 ? 0 : (int)(b_begin - begin), upto = slot == 0 && a_end - begin < n ? (int)(a_end - begin) : n;
      const int t = __shfl(mine.t, lane + skip);
      if (p.D >= N) sum_window<true, A>(p, to, t, upto - skip, d0, step, lane);
      else sum_window<false, A>(p, to, t, upto - skip, d0, step, lane);
      if (p.arrived == nullptr) continue;
      const int from = slot == 0 ? 0 : n - 1;
      const int row = __builtin_amdgcn_readlane(mine.row, from), start = __builtin_amdgcn_readlane(mine.start, from),
                count = __builtin_amdgcn_readlane(mine.count, from), first = start / kWindow, last = (start + count - 1) / kWindow;
      __threadfence();  // (what this wavefront has written is there for the one that joins)
      int before = 0;
      if (lane == 0) before = atomicAdd(&p.arrived[(first << p.team_log) + (int)(wave & ((1 << p.team_log) - 1))], 1);
      if (__builtin_amdgcn_readfirstlane(before) != last - first) continue;
      __threadfence();
      if (p.D >= N) join_row<true, ADD, A, B>(p, row, start, count, d0, step, lane);
      else join_row<false, ADD, A, B>(p, row, start, count, d0, step, lane);
    }
    return;
  }
  // the places where a row starts
  const int total = p.starts[p.N];
  for (long long n = item - windows; n < p.T; n += sums) {
    const long long at = n + lane < p.T ? n + lane : p.T - 1;
    const Place mine = p.places[at];
    if (n >= total) return;
    const int count = __builtin_amdgcn_readfirstlane(mine.count);
    if (__builtin_amdgcn_readfirstlane(mine.start) != n || count > kWindow) continue;
    B *to = reinterpret_cast<B *>(p.to) + (long long)__builtin_amdgcn_readfirstlane(mine.row) * p.to_stride;
    if (p.D >= N) sum_row<true, ADD, A>(p, to, mine.t, count, d0, step, lane);
    else sum_row<false, ADD, A>(p, to, mine.t, count, d0, step, lane);
  }
}

// The rows without a token: 4 KB a workgroup, one store a thread, in a launch of its own with next to nothing to set up.  Memory takes such a stream best
// (1.006 GB: 149 to 152 us, 6.7 TB/s; two stores a thread 166 to 190, 64 rows a workgroup 206; in the summing launch, whose wavefronts carry more
// registers, 208).
constexpr int kZeroRows = 32768;
template <typename B>
__global__ void __launch_bounds__(kBlock) embed_zero_kernel(const int32_t *starts, B *to, long long to_stride, long long D, long long row0, long long N) {
  constexpr int kStore = kWide<B>;
  const long long row = row0 + (long long)blockIdx.z * kZeroRows + blockIdx.y;
  if (row >= N || starts[row] != starts[row + 1]) return;
  const long long d = ((long long)blockIdx.x * kBlock + threadIdx.x) * kStore;
  const float none[kStore] = {};
  if (d < D) stream_first<kStore>(to + row * to_stride + d, D - d, none);
}

// Joins the windows of long rows, 256 columns a workgroup.  A wavefront looks whether long rows start in its windows and joins the shorter ones; the longer ones are
// the workgroup's, one after the other, every sixteenth window a wavefront, in an order that follows from the row's place alone.
// A row's joined columns, all wavefronts of a workgroup.
template <bool ALL, bool ADD, typename B>
__device__ __forceinline__ void join_columns(const EmbedParams &p, float (&s_sum)[kJoinThreads / 64][64 * 4], B *to, long long first, long long last, int slot,
                                             long long d0) {
  constexpr int N = 4, kWaves = kJoinThreads / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Columns<N> c = columns_at<ALL, N>(d0 + lane * N, p.D);
  float sum[N] = {}, before[N] = {};
  if constexpr (ADD) load_columns<ALL, N>(to, c, before);
  for (long long v = first + wave; v <= last; v += kWaves * kAhead) {
    float part[kAhead][N];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {  // (without a branch, the last one again where there are fewer)
      const long long at = v + u * kWaves < last ? v + u * kWaves : last;
      load_columns<ALL, N>(p.partial + (at * 2 + (at == first ? slot : 0)) * p.D, c, part[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int j = 0; j < N; ++j) sum[j] += v + u * kWaves <= last ? part[u][j] : 0.0f;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < N; ++j) s_sum[wave][lane * N + j] = sum[j];
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int j = 0; j < N; ++j)
    for (int v = 1; v < kWaves; ++v) sum[j] += s_sum[v][lane * N + j];
  add_scaled<ADD, N>(p, before, sum);
  store_columns<N, true>(to, c, sum);
}
template <typename B, bool ADD> __global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(const EmbedParams p) {
  constexpr int N = 4, kWaves = kJoinThreads / 64;
  __shared__ float s_sum[kWaves][64 * N];
  __shared__ Place s_row[64 + 1];  // (rows that start in the workgroup's windows, each more than kFewJoins of them long)
  __shared__ int s_n;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  Place mine = {0, -1, 0, 0};
  const long long begin = (((long long)blockIdx.x * kWaves + wave) * p.join_each + lane) * kWindow;
  if (lane < p.join_each && begin < p.T) {
    const int total = p.starts[p.N];
    const int until = p.T - begin < kWindow ? (int)p.T : (int)begin + kWindow;
    Place last = p.places[until - 1];
    if (total < until && total > begin) last = p.places[total - 1];  // (places are written up to `total`)
    if (total > begin && last.start >= begin && last.count > kWindow) mine = last;
  }
  const long long d0 = (long long)blockIdx.y * 64 * N, step = (long long)gridDim.y * 64 * N;
  for (unsigned long long left = __ballot(mine.row >= 0); left != 0; left &= left - 1) {  // (uniform)
    const int from = __builtin_ctzll(left);
    const Place row = {0, (int)__builtin_amdgcn_readlane(mine.row, from), (int)__builtin_amdgcn_readlane(mine.start, from),
                       (int)__builtin_amdgcn_readlane(mine.count, from)};
    if (row.count > kFewJoins * kWindow) {
      if (lane == 0) s_row[atomicAdd(&s_n, 1)] = row;
    } else if (p.D >= N) {
      join_row<true, ADD, float, B>(p, row.row, row.start, row.count, d0, step, lane);
    } else {
      join_row<false, ADD, float, B>(p, row.row, row.start, row.count, d0, step, lane);
    }
  }
  __syncthreads();
  const int n = s_n;
  for (int i = 0; i < n; ++i) {  // (uniform)
    const Place row = s_row[i];
    const long long first = row.start / kWindow, last = ((long long)row.start + row.count - 1) / kWindow;
    const int slot = row.start != first * kWindow ? 1 : 0;  // (of its first window)
    B *to = reinterpret_cast<B *>(p.to) + (long long)row.row * p.to_stride;
    for (long long d = d0; d < p.D; d += step) {
      if (p.D >= N) join_columns<true, ADD>(p, s_sum, to, first, last, slot, d);
      else join_columns<false, ADD>(p, s_sum, to, first, last, slot, d);
    }
  }
}

template <typename F> hipError_t by_types(int from, int to, F launch) {
  if (from == LLC_F32) return to == LLC_F32 ? launch(float(), float()) : launch(float(), uint16_t());
  return to == LLC_F32 ? launch(uint16_t(), float()) : launch(uint16_t(), uint16_t());
}

bool sizes_ok(long long T, long long N, long long D) {
  return T >= 0 && T <= kMaxIndex && N >= 1 && N <= kMaxIndex && D >= 1 && D <= kMaxIndex;
}

// log2 of the wavefronts that share a row: as many as have columns, up to a workgroup's four.
int team_log_of(long long D, int from) {
  const long long slabs = (D * (long long)type_size(from) + 1023) / 1024;
  return slabs >= 4 ? 2 : slabs >= 2 ? 1 : 0;
}

// Up to that many windows the last of a long row's wavefronts joins it, which spares a launch; that wavefront's sums follow each other, so the joins of
// more windows are workgroups' of their own.  us a call, bf16 rows of 1537 into fp32, with the launch and without: 1001 tokens that hardly
// repeat 14.3, 10.5; three in ten by one token 15.2, 15.5; all by one token 15.7, 19.2.  4096 tokens, when the launch took 5 us more: 21.2, 17.6; 22.2, 25.7; 21.7,
// 44.5.  (A tree of such joins, without the other launch at all: 16 384 x 4096 bf16, a quarter by one token, 147 us for the sums, where sums and joins take 46 and
// 5: every fence writes back what the L2 holds.)
constexpr int kFewWindows = 32;

struct GradLayout {
  size_t places, starts, arrived, partial, total;
};
GradLayout grad_layout(long long T, long long N, long long D) {
  const auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  GradLayout l;
  size_t at = 0;
  l.places = at; at += up((size_t)T * sizeof(Place));
  l.starts = at; at += up((size_t)(N + 1) * 4);
  l.arrived = at; at += T > kWindow && T <= kFewWindows * kWindow ? up(kFewWindows * 4 * 4) : 0;
  l.partial = at; at += T > kWindow ? up((size_t)((T + kWindow - 1) / kWindow) * 2 * (size_t)D * 4) : 0;
  l.total = at;
  return l;
}

constexpr long long kMostBlocks = 0xFFFFFFFFLL / kBlock;  // of a launch
constexpr long long kRowBlocks = 1LL << 22;  // of a launch's that take rows (they take several where there are more)

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
  EmbedParams p = {};
  p.T = a->T; p.N = a->N; p.D = a->D;
  p.from = a->table; p.from_stride = a->table_stride_n; p.tokens = a->tokens; p.tok_stride = a->tok_stride;
  p.scale = a->scale; p.to = a->out; p.to_stride = a->out_stride_t;
  p.team_log = team_log_of(a->D, a->dtype);
  const long long blocks = ((a->T << p.team_log) + kBlock / 64 - 1) / (kBlock / 64);
  if (blocks > kMostBlocks) return LLC_E_SHAPE;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    return by_types(a->dtype, a->out_dtype, [&](auto from, auto to) {
      embed_kernel<decltype(from), decltype(to)><<<(unsigned)blocks, kBlock, 0, st>>>(p);
      return hipGetLastError();
    });
  });
}

extern "C" size_t llc_embed_grad_workspace_size(int64_t T, int64_t N, int64_t D) {
  return sizes_ok(T, N, D) && N <= kMostRows ? grad_layout(T, N, D).total : 0;
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
  const GradLayout l = grad_layout(a->T, a->N, a->D);
  if (a->workspace == nullptr || !fits(a->workspace, 256) || a->workspace_bytes < l.total) return LLC_E_WORKSPACE;
  EmbedParams p = {};
  p.T = a->T; p.N = a->N; p.D = a->D;
  p.from = a->g; p.from_stride = a->g_stride_t; p.tokens = a->tokens; p.tok_stride = a->tok_stride;
  p.scale = a->scale; p.add = a->add; p.to = a->grad; p.to_stride = a->grad_stride_n;
  p.team_log = team_log_of(a->D, a->dtype);
  char *work = (char *)a->workspace;
  p.places = (Place *)(work + l.places); p.starts = (int32_t *)(work + l.starts);
  p.partial = (float *)(work + l.partial);
  // (a workgroup of the sort on every CU, as long as its counters fit)
  p.range = (int)((a->N + 255) / 256 < kMostRange ? (a->N + 255) / 256 : kMostRange);
  const long long sort_blocks = (a->N + p.range - 1) / p.range;
  p.windows = a->T > kWindow ? (a->T + kWindow - 1) / kWindow : 0;
  p.arrived = p.windows > 0 && p.windows <= kFewWindows ? (int *)(work + l.arrived) : nullptr;
  const long long a_block = kBlock / 64, window_blocks = ((p.windows << p.team_log) + a_block - 1) / a_block;
  const auto row_blocks = [&](long long rows) {
    const long long blocks = ((rows << p.team_log) + a_block - 1) / a_block;
    return blocks < kRowBlocks ? blocks : kRowBlocks;
  };
  const long long sum_blocks = row_blocks(a->T), chunks = (a->D * (long long)type_size(a->grad_dtype) + 4095) / 4096;
  if (window_blocks > kMostBlocks - kRowBlocks) return LLC_E_SHAPE;
  p.window_blocks = (unsigned)window_blocks; p.sum_blocks = (unsigned)sum_blocks;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    // Few tokens: four wavefronts take them in one go, and are sooner done than sixteen.  (us a call with four and with sixteen, rows of 256: 256 tokens
    // 12.3, 13.4; 4096 14.0, 14.6; 8192 18.6, 16.0; 16 384 26.6, 18.8.)
    if (a->T <= 4 * 64 * kSortAhead)
      embed_sort_kernel<4><<<(unsigned)sort_blocks, 256, ((size_t)4 * p.range + p.range + 1) * 4, st>>>(p);
    else
      embed_sort_kernel<16><<<(unsigned)sort_blocks, 1024, ((size_t)16 * p.range + p.range + 1) * 4, st>>>(p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return by_types(a->dtype, a->grad_dtype, [&](auto from, auto to) {
      using B = decltype(to);
      const long long most_rows = kRowBlocks / chunks < 1 ? 1 : kRowBlocks / chunks;  // of a launch
      for (long long row0 = 0; p.add == 0 && row0 < p.N && e == hipSuccess; row0 += most_rows) {
        const long long rows = p.N - row0 < most_rows ? p.N - row0 : most_rows;
        const dim3 grid((unsigned)chunks, (unsigned)(rows < kZeroRows ? rows : kZeroRows), (unsigned)((rows + kZeroRows - 1) / kZeroRows));
        embed_zero_kernel<B><<<grid, kBlock, 0, st>>>(p.starts, (B *)p.to, p.to_stride, p.D, row0, row0 + rows);
        e = hipGetLastError();
      }
      if (e != hipSuccess || p.T == 0) return e;
      const unsigned sums = (unsigned)(window_blocks + sum_blocks);
      if (p.add != 0) embed_sum_kernel<decltype(from), B, true><<<sums, kBlock, 0, st>>>(p);
      else embed_sum_kernel<decltype(from), B, false><<<sums, kBlock, 0, st>>>(p);
      e = hipGetLastError();
      if (e != hipSuccess || p.windows == 0 || p.arrived != nullptr) return e;
      // (a workgroup a CU, where that leaves a wavefront 64 windows: more of them wait for each other)
      const long long slabs = (a->D + 255) / 256, columns = slabs < 64 ? slabs : 64, waves = kJoinThreads / 64;
      const long long each = (p.windows * columns + 256 * waves - 1) / (256 * waves);
      EmbedParams q = p;
      q.join_each = (int)(each < 64 ? each : 64);
      const dim3 grid((unsigned)((p.windows + q.join_each * waves - 1) / (q.join_each * waves)), (unsigned)columns);
      if (p.add != 0) embed_join_kernel<B, true><<<grid, kJoinThreads, 0, st>>>(q);
      else embed_join_kernel<B, false><<<grid, kJoinThreads, 0, st>>>(q);
      return hipGetLastError();
    });
  });
}
