// Layers held in 4 bits: making one, looking rows of it up, and the host side of the products with it.  The first two move data and compute next to
// nothing beside it: memory bounds them.  A lane takes eight neighbouring columns (a word of codes), a wavefront 512, four times over (128 256 x 2048 in
// fp32, groups of 64 with zeros: 230 us, 5.2 TB/s; all its rows back in bf16 after it: 131 us, 5.1 TB/s; again, the codes still in the caches: 95).
#include "quantized.hpp"

namespace llc {
namespace {

constexpr int kPieces = 4;                    // of 512 columns that a wavefront has in flight
constexpr int kUnit = 512 * kPieces;
constexpr long long kMostUnitBlocks = 1LL << 22;  // of a launch; its workgroups take several units each where there are more
constexpr long long kMostUnits = 1LL << 31;

struct QuantizedParams {
  long long N, D;           // rows (tokens of the lookup) and columns
  long long table;          // rows of the lookup's table
  unsigned units_row;       // units of a row
  long long units;
  const void *w;
  long long w_stride;
  uint8_t *codes;
  long long codes_stride;
  void *scales;
  long long scales_stride;
  uint8_t *zeros;
  long long zeros_stride;
  const int32_t *tokens;
  long long tok_stride;
  float scale;
  void *out;
  long long out_stride;
};

template <int CTRL> __device__ __forceinline__ float dpp_max(float v) {
  return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true)));
}
template <int LANES> __device__ __forceinline__ float max_lanes(float v) {  // over 4, 8 or 16 neighbours, in each of them
  v = dpp_max<0xB1>(v);
  v = dpp_max<0x4E>(v);
  if constexpr (LANES >= 8) v = dpp_max<0x141>(v);
  if constexpr (LANES >= 16) v = dpp_max<0x140>(v);
  return v;
}

// The whole number nearest to w / s, ties to even, for a quotient of at most some 16: a product with the rounded reciprocal finds it within one, and the sign of w - (n + 1/2) s,
// which a fused multiply-add rounds rightly, decides.  (fp32 division, ten operations, makes ties of quotients that are none: half of a group's
// largest entry is three and a half times its scale but for the scale's rounding.)
__device__ __forceinline__ float nearest(float w, float s, float inverse) {
  const float n = floorf(fminf(fmaxf(w * inverse, -20.0f), 20.0f));
  const float d = fmaf(-(n + 0.5f), s, w);
  return d > 0.0f ? n + 1.0f : d < 0.0f ? n : n + (float)((int)n & 1);
}

template <int G, typename A, typename S, bool ZEROS> __global__ void __launch_bounds__(kBlock) quantize_kernel(const QuantizedParams p) {
  const int lane = threadIdx.x & 63;
  for (long long unit = (long long)blockIdx.x * (kBlock / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); unit < p.units;
       unit += (long long)gridDim.x * (kBlock / 64)) {
    const long long n = unit / p.units_row, first = (unit - n * p.units_row) * kUnit + lane * 8;
    const A *row = reinterpret_cast<const A *>(p.w) + n * p.w_stride;
    float v[kPieces][8];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const long long at = first + i * 512;
      if (at < p.D) {
        load_first<8>(row + at, p.D - at, v[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const long long at = first + i * 512;
      float low = 0.0f, high = 0.0f;  // (of -w where there are zeros)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float f = fabsf(v[i][j]) < INFINITY ? v[i][j] : 0.0f;
        high = fmaxf(high, ZEROS ? f : fabsf(f));
        if constexpr (ZEROS) low = fmaxf(low, -f);
      }
      high = max_lanes<G / 8>(high);
      if constexpr (ZEROS) low = max_lanes<G / 8>(low);
      float scale;
      if constexpr (ZEROS) scale = high + low < INFINITY ? (high + low) / 15.0f : (0.5f * high + 0.5f * low) / 7.5f;
      else scale = high / 7.0f;
      const S kept = narrow<S>(scale);
      scale = widen(kept);
      // (scales whose reciprocal would not be a number: both sides are raised, exactly)
      const float lift = scale < 0x1p-100f ? 0x1p64f : 1.0f, s = scale * lift, inverse = __builtin_amdgcn_rcpf(s);
      float zero = 8.0f;
      if constexpr (ZEROS) zero = scale > 0.0f ? fminf(nearest(low * lift, s, inverse), 15.0f) : 8.0f;
      if (at >= p.D) continue;
      uint32_t word = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float q = nearest(v[i][j] * lift, s, inverse) + zero;
        q = fminf(fmaxf(q, 0.0f), 15.0f);
        q = scale > 0.0f && v[i][j] == v[i][j] ? q : zero;
        word |= (at + j < p.D ? (uint32_t)q : 0u) << (4 * j);
      }
      uint8_t *to = p.codes + n * p.codes_stride + at / 2;
      if (at + 8 <= p.D) {
        *reinterpret_cast<word1_byte *>(to) = word;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at + 2 * j < p.D) to[j] = (uint8_t)(word >> (8 * j));
      }
      if (at % G == 0) {
        reinterpret_cast<S *>(p.scales)[n * p.scales_stride + at / G] = kept;
        if constexpr (ZEROS) p.zeros[n * p.zeros_stride + at / G] = (uint8_t)zero;
      }
    }
  }
}

template <int G, typename S, typename B> __global__ void __launch_bounds__(kBlock) embed_quantized_kernel(const QuantizedParams p) {
  const int lane = threadIdx.x & 63;
  for (long long unit = (long long)blockIdx.x * (kBlock / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); unit < p.units;
       unit += (long long)gridDim.x * (kBlock / 64)) {
    const long long t = unit / p.units_row, first = (unit - t * p.units_row) * kUnit + lane * 8;
    const long long n = p.tokens[t * p.tok_stride];
    const bool there = n >= 0 && n < p.table;
    const uint8_t *codes = p.codes + (there ? n : 0) * p.codes_stride;
    const S *scales = reinterpret_cast<const S *>(p.scales) + (there ? n : 0) * p.scales_stride;
    const uint8_t *zeros = p.zeros != nullptr ? p.zeros + (there ? n : 0) * p.zeros_stride : nullptr;
    B *to = reinterpret_cast<B *>(p.out) + t * p.out_stride;
    uint32_t word[kPieces];
    float scale[kPieces], zero[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const long long at = first + i * 512;
      word[i] = 0; scale[i] = 0.0f; zero[i] = 8.0f;
      if (at < p.D) {
        word[i] = load_codes(codes, at, p.D);
        scale[i] = widen(scales[at / G]);
        if (zeros != nullptr) zero[i] = (float)zeros[at / G];
      }
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const long long at = first + i * 512;
      if (at >= p.D) continue;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w = p.scale * (scale[i] * ((float)((word[i] >> (4 * j)) & 15) - zero[i]));
        v[j] = there ? w : 0.0f;
      }
      stream_first<8>(to + at, p.D - at, v);
    }
  }
}

template <typename F> hipError_t by_group(int group, F launch) {
  if (group == 128) return launch(std::integral_constant<int, 128>());
  if (group == 64) return launch(std::integral_constant<int, 64>());
  return launch(std::integral_constant<int, 32>());
}
template <typename F> hipError_t by_type(int type, F launch) { return type == LLC_F32 ? launch(float()) : launch(uint16_t()); }

// A layer's sizes and rows, the same in every call.
int check_layer(long long D, int group, const void *codes, long long codes_stride, const void *scales, int scales_dtype, long long scales_stride, const void *zeros,
                long long zeros_stride) {
  if (codes == nullptr || scales == nullptr) return LLC_E_NULL;
  const long long groups = groups_of(D, group);
  if (codes_stride < (D + 1) / 2 || scales_stride < groups || (zeros != nullptr && zeros_stride < groups)) return LLC_E_SHAPE;
  if (!known_type(scales_dtype)) return LLC_E_DTYPE;
  return fits(scales, type_size(scales_dtype)) ? LLC_OK : LLC_E_ALIGN;
}
bool units_of(QuantizedParams &p) {
  p.units_row = (unsigned)((p.D + kUnit - 1) / kUnit);
  p.units = p.N * p.units_row;
  return p.units <= kMostUnits;
}
unsigned unit_blocks(const QuantizedParams &p) {
  const long long blocks = (p.units + kBlock / 64 - 1) / (kBlock / 64);
  return (unsigned)(blocks < kMostUnitBlocks ? blocks : kMostUnitBlocks);
}

}  // namespace
}  // namespace llc

using namespace llc;

extern "C" int llc_quantize(const llc_quantize_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  if (a->N < 0 || a->N > kMaxIndex || a->D < 1 || a->D > kMaxIndex) return LLC_E_SHAPE;
  if ((a->flags & ~LLC_FLAG_DRY_RUN) != 0 || !known_group(a->group)) return LLC_E_OPTION;
  if (a->N == 0) return LLC_OK;
  if (a->w == nullptr) return LLC_E_NULL;
  const int bad = check_layer(a->D, a->group, a->codes, a->codes_stride_n, a->scales, a->scales_dtype, a->scales_stride_n, a->zeros, a->zeros_stride_n);
  if (bad != LLC_OK) return bad;
  if (a->w_stride_n < 0) return LLC_E_SHAPE;
  if (!known_type(a->dtype)) return LLC_E_DTYPE;
  if (!fits(a->w, type_size(a->dtype))) return LLC_E_ALIGN;
  QuantizedParams p = {};
  p.N = a->N; p.D = a->D; p.w = a->w; p.w_stride = a->w_stride_n; p.codes = a->codes; p.codes_stride = a->codes_stride_n;
  p.scales = a->scales; p.scales_stride = a->scales_stride_n; p.zeros = a->zeros; p.zeros_stride = a->zeros_stride_n;
  if (!units_of(p)) return LLC_E_SHAPE;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    return by_group(a->group, [&](auto group) {
      return by_type(a->dtype, [&](auto from) {
        return by_type(a->scales_dtype, [&](auto scale) {
          constexpr int G = decltype(group)::value;
          if (p.zeros != nullptr) quantize_kernel<G, decltype(from), decltype(scale), true><<<unit_blocks(p), kBlock, 0, st>>>(p);
          else quantize_kernel<G, decltype(from), decltype(scale), false><<<unit_blocks(p), kBlock, 0, st>>>(p);
          return hipGetLastError();
        });
      });
    });
  });
}

extern "C" int llc_embed_quantized(const llc_embed_quantized_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  if (a->T < 0 || a->T > kMaxIndex || a->N < 1 || a->N > kMaxIndex || a->D < 1 || a->D > kMaxIndex) return LLC_E_SHAPE;
  if ((a->flags & ~LLC_FLAG_DRY_RUN) != 0 || !known_group(a->group) || !std::isfinite(a->scale)) return LLC_E_OPTION;
  if (a->T == 0) return LLC_OK;
  if (a->tokens == nullptr || a->out == nullptr) return LLC_E_NULL;
  const int bad = check_layer(a->D, a->group, a->codes, a->codes_stride_n, a->scales, a->scales_dtype, a->scales_stride_n, a->zeros, a->zeros_stride_n);
  if (bad != LLC_OK) return bad;
  if (a->tok_stride < 0 || a->out_stride_t < a->D) return LLC_E_SHAPE;
  if (!known_type(a->out_dtype)) return LLC_E_DTYPE;
  if (!fits(a->out, type_size(a->out_dtype)) || !fits(a->tokens, 4)) return LLC_E_ALIGN;
  QuantizedParams p = {};
  p.N = a->T; p.D = a->D; p.table = a->N; p.codes = const_cast<uint8_t *>(a->codes); p.codes_stride = a->codes_stride_n;
  p.scales = const_cast<void *>(a->scales); p.scales_stride = a->scales_stride_n; p.zeros = const_cast<uint8_t *>(a->zeros); p.zeros_stride = a->zeros_stride_n;
  p.tokens = a->tokens; p.tok_stride = a->tok_stride; p.scale = a->scale; p.out = a->out; p.out_stride = a->out_stride_t;
  if (!units_of(p)) return LLC_E_SHAPE;
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    return by_group(a->group, [&](auto group) {
      return by_type(a->scales_dtype, [&](auto scale) {
        return by_type(a->out_dtype, [&](auto to) {
          embed_quantized_kernel<decltype(group)::value, decltype(scale), decltype(to)><<<unit_blocks(p), kBlock, 0, st>>>(p);
          return hipGetLastError();
        });
      });
    });
  });
}

namespace llc {
namespace {

struct MatvecPlan {
  int tiles, parts, streamed, share_log, block_tiles;
  unsigned tile_blocks, blocks, passes;
  size_t lds;
  long long image_stride;
  size_t workspace;
};
MatvecPlan plan_matvec(long long R, long long N, long long D, int group, int dtype) {
  MatvecPlan m = {};
  const int rows = (int)(R < kMatvecRows ? R : kMatvecRows), slabs = (int)((D + 127) / 128);
  m.tiles = (rows + 15) / 16;
  m.parts = dtype == LLC_F32 ? 3 : 1;
  m.passes = (unsigned)((R + kMatvecRows - 1) / kMatvecRows);
  const long long column_tiles = (N + 15) / 16;
  constexpr int waves = kMatvecThreads / 64;
  constexpr size_t kLds = 156 << 10;  // that a workgroup may have, of a CU's 160 KB
  const auto join_bytes = [&](int wide, int log) { return log > 0 ? (size_t)waves * wide * m.tiles * 1024 : 0; };
  // Wavefronts share tiles of few columns until some 2048 of them are at work, eight a CU.
  const auto share_for = [&](int wide, int most) {
    int log = 0;
    while (log < 3 && (column_tiles << log) < 2048LL * wide && (2 << log) <= most) ++log;
    return log;
  };
  m.share_log = share_for(1, slabs);
  m.lds = (size_t)slabs * ((size_t)256 * m.parts * pitch_of(rows) + (size_t)(128 / group) * 64) + join_bytes(1, m.share_log);
  m.streamed = m.tiles == 1 && m.lds <= kLds ? 0 : 1;
  if (m.streamed == 0) {
    const int each = waves >> m.share_log;
    m.tile_blocks = (unsigned)((column_tiles + each - 1) / each);
    const unsigned resident = 256u * (m.lds <= kLds / 2 ? 2 : 1);
    const unsigned turns = (m.tile_blocks + resident - 1) / resident;  // (as many blocks for each workgroup, or one less)
    m.blocks = (m.tile_blocks + turns - 1) / turns;
    return m;
  }
  const size_t slab = (size_t)slab_bytes(m.parts, m.tiles, group);
  const int part = streamed_slabs(m.tiles, m.parts), part_log = part == 4 ? 2 : part == 2 ? 1 : 0;
  m.share_log = column_tiles < 2048 && part <= slabs ? part_log : 0;
  m.lds = 2 * slab * (size_t)part + join_bytes(2, m.share_log);
  const long long each = 2 * (waves >> m.share_log), turns = (column_tiles + 256 * each - 1) / (256 * each);
  m.block_tiles = (int)((column_tiles + 256 * turns - 1) / (256 * turns));
  m.tile_blocks = m.blocks = (unsigned)((column_tiles + m.block_tiles - 1) / m.block_tiles);
  m.image_stride = (long long)(((size_t)slabs * slab + 255) & ~(size_t)255);
  m.workspace = (size_t)m.image_stride * m.passes;
  return m;
}
// (a launch takes fewer than 2^32 threads: of the layout of x, and, of the products, for every 64 rows a workgroup for at least 13 tiles of 16 columns)
bool matvec_sizes_ok(long long R, long long N, long long D) {
  return R >= 0 && R <= (1LL << 17) && N >= 1 && N <= kMaxIndex && D >= 1 && D <= (1LL << 27) && R * D <= (1LL << 34) && (R <= 16 || (R + 63) / 64 * ((N + 15) / 16) <= 1LL << 25);
}

}  // namespace
}  // namespace llc

extern "C" size_t llc_matvec_quantized_workspace_size(int64_t R, int64_t N, int64_t D, int32_t group, int32_t dtype) {
  if (!matvec_sizes_ok(R, N, D) || R == 0 || !known_group(group) || !known_type(dtype)) return 0;
  return plan_matvec(R, N, D, group, dtype).workspace;
}

extern "C" int llc_matvec_quantized(const llc_matvec_quantized_args *a) {
  if (a == nullptr) return LLC_E_NULL;
  if (!matvec_sizes_ok(a->R, a->N, a->D)) return LLC_E_SHAPE;
  if ((a->flags & ~LLC_FLAG_DRY_RUN) != 0 || !known_group(a->group)) return LLC_E_OPTION;
  if (a->R == 0) return LLC_OK;
  if (a->x == nullptr || a->out == nullptr) return LLC_E_NULL;
  const int bad = check_layer(a->D, a->group, a->codes, a->codes_stride_n, a->scales, a->scales_dtype, a->scales_stride_n, a->zeros, a->zeros_stride_n);
  if (bad != LLC_OK) return bad;
  if (a->x_stride_r < 0 || a->out_stride_r < a->N) return LLC_E_SHAPE;
  if (!known_type(a->dtype) || !known_type(a->out_dtype)) return LLC_E_DTYPE;
  if (!fits(a->x, type_size(a->dtype)) || !fits(a->out, type_size(a->out_dtype))) return LLC_E_ALIGN;
  const MatvecPlan m = plan_matvec(a->R, a->N, a->D, a->group, a->dtype);
  if (m.workspace > 0 && (a->workspace == nullptr || !fits(a->workspace, 256) || a->workspace_bytes < m.workspace)) return LLC_E_WORKSPACE;
  MatvecParams p = {};
  p.R = a->R; p.N = a->N; p.D = a->D; p.x = a->x; p.x_stride = a->x_stride_r;
  p.codes = a->codes; p.codes_stride = a->codes_stride_n; p.scales = a->scales; p.scales_stride = a->scales_stride_n;
  p.zeros = a->zeros; p.zeros_stride = a->zeros_stride_n; p.out = a->out; p.out_stride = a->out_stride_r; p.out_type = a->out_dtype;
  p.groups = (int)groups_of(a->D, a->group);
  p.slabs = (int)((a->D + 127) / 128);
  p.streamed = m.streamed; p.share_log = m.share_log; p.tile_blocks = m.tile_blocks; p.tiles = m.tiles; p.block_tiles = m.block_tiles;
  p.image = (char *)a->workspace; p.image_stride = m.image_stride;
  const dim3 grid(m.blocks, m.passes);
  if ((a->flags & LLC_FLAG_DRY_RUN) != 0) return LLC_OK;
  hipStream_t st = (hipStream_t)a->stream;
  return between_events(a->ev_begin, a->ev_end, st, [&] {
    return a->dtype == LLC_F32 ? launch_matvec_f32(p, m.tiles, a->group, a->scales_dtype, grid, m.lds, st)
                               : launch_matvec_bf16(p, m.tiles, a->group, a->scales_dtype, grid, m.lds, st);
  });
}
