// A linear layer's weight gradient from its output's gradient dY [tokens][n]
// and its input X [tokens][k] kept in 8 bits:
//
//   dW[n][k] (+)= sum over t of dY[t][n] * (X[t][k] * scale[k] + shift[k])
//             =  scale[k] * (dY^T X)[n][k] + shift[k] * s[n],   s[n] = sum over t of dY[t][n]
//   dbias[n] (+)= s[n]
//
// so the columns' scale and shift cost the main loop nothing.  Bound by the
// matrix cores: 2 n k flops a token.  A kept element is 4 significant bits
// times a power of two, so it is exact in bf16 (below 2^-126 as far as its
// subnormals hold it); a bf16 dY enters as it is, an fp32 dY as the sum of three
// bf16 parts (8 of its 24 bits each), which keeps every product exact.  Sums are
// fp32; scale and shift are applied to the two sums, so where X * scale and shift
// cancel the error stays that of each.
//
// Both operands lie with the tokens, over which the product sums, as rows: a
// tile goes to LDS as it lies and the transposing LDS reads give each lane the
// eight tokens of its column that the matrix instruction takes.
#include <algorithm>

#include "lc_ops_device.h"

namespace lc {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr uint32_t kTile = 128;     // of n and of k
constexpr uint32_t kStep = 32;      // tokens in LDS at a time
constexpr uint32_t kThreads = 256;  // four waves of 64 x 64
constexpr uint32_t kPitch = kTile + 16;  // elements from token to token in LDS
constexpr uint32_t kOut = 64 + 4;        // floats from row to row on their way out

struct Codes16 {
  u32x4 codes;
  uint32_t code;
};

typedef u32x4 __attribute__((aligned(1))) u32x4_any1;
typedef const __attribute__((address_space(1))) u32x4_any1 gc_u32x4_any1;

// Sixteen codes of one block of a row and the block's power; zeros outside.
__device__ __forceinline__ Codes16 load_codes16(const Kept& x, uint64_t row, uint32_t col, int n) {
  Codes16 r;
  r.codes = u32x4{0, 0, 0, 0};
  r.code = 127;
  if (n <= 0) return r;
  const uint64_t p = x.codes + row * x.code_stride + col;
  if (n >= 16) {
    r.codes = *(gc_u32x4_any1*)p;
  } else {
#pragma unroll
    for (int i = 0; i < 15; ++i)
      if (i < n) r.codes[i / 4] |= static_cast<uint32_t>(*(gc_u8*)(p + i)) << (8 * (i & 3));
  }
  r.code = *(gc_u8*)(x.scales + row * x.scale_stride + col / kActBlock);
  return r;
}

// Sixteen codes moved down by s, zeros behind them.
__device__ __forceinline__ void move_down16(u32x4& v, uint32_t s) {
  uint64_t lo = v[0] | static_cast<uint64_t>(v[1]) << 32, hi = v[2] | static_cast<uint64_t>(v[3]) << 32;
  if (s & 8) {
    lo = hi;
    hi = 0;
  }
  const uint32_t bits = s % 8 * 8;
  if (bits) {
    lo = lo >> bits | hi << (64 - bits);
    hi >>= bits;
  }
  v = u32x4{static_cast<uint32_t>(lo), static_cast<uint32_t>(lo >> 32), static_cast<uint32_t>(hi), static_cast<uint32_t>(hi >> 32)};
}

// Four bytes to four bf16, times 2^(code - 127); exact, and code 255 gives NaN.
__device__ __forceinline__ u32x2 decode4(uint32_t b, float scale) {
  const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
  const auto hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// Two fp32 values as three pairs of bf16 parts, of 8 bits each, whose sums they
// are; of what is not finite the first part says so alone.
__device__ __forceinline__ void split3(float a, float b, uint32_t (&part)[3]) {
  float v[2] = {a, b};
  uint32_t top[2];
  part[0] = part[1] = part[2] = 0;
#pragma unroll
  for (int p = 0; p < 3; ++p) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      top[i] = __float_as_uint(v[i]);
      if (p == 0) top[i] = v[i] != v[i] ? 0x7FC00000u : top[i];  // its low bits may be all that says NaN
      const float rest = v[i] - __uint_as_float(top[i] & 0xffff0000u);
      v[i] = p > 0 || fabsf(v[i]) < __builtin_inff() ? rest : 0.0f;
    }
    part[p] = top[0] >> 16 | (top[1] & 0xffff0000u);
  }
}

template <int DT>
constexpr int kPlanes = DT == kBf16 ? 1 : 3;

// Eight tokens of the lane's column out of LDS rows [t0, t0 + 32): the operand
// of a 16 x 16 x 32 product for the 16 columns at `col`.
__device__ __forceinline__ bf16x8 read_cols(const uint16_t* tile, uint32_t col, uint32_t lane) {
  const uint32_t row = lane / 16 * 8 + lane % 16 / 4;
  const uint16_t* p = tile + row * kPitch + col + lane % 4 * 4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * kPitch));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// How a product is cut: `full` tiles of the whole sum over the tokens, then the
// others in `splits` parts each, whose sums wgrad_join_kernel adds.
struct WgradTiles {
  uint32_t tile;         // columns of n and of k
  uint32_t tn, tk;       // tiles of n and k
  uint32_t splits;
  uint32_t full, tiles;  // tiles of the whole sum, and all: dW's 2^46 bytes hold fewer than 2^32
  uint64_t per_split;    // tokens a part, a multiple of kStep
  float* part;           // [tiles - full][splits][tile][tile]
  float* sums;           // [sum_parts][n] column sums of dY
  uint32_t sum_parts;
  bool big;              // wgrad_big_kernel's tiles
  bool ragged;           // of rows that end inside 16 bytes
};

struct WgradItem {
  uint32_t tile, split, n0, k0;
  bool whole;
  uint64_t t_begin, t_end;
};
// Eight tiles of n by all of k follow each other, so that blocks that run side
// by side read the same columns.
__device__ __forceinline__ void wgrad_place(const WgradTiles& s, uint32_t tile, uint32_t& n0, uint32_t& k0) {
  const uint32_t group = tile / (8 * s.tk), in_g = tile - group * 8 * s.tk;
  const uint32_t wide = s.tn - group * 8 < 8 ? s.tn - group * 8 : 8, k = in_g / wide;
  n0 = (group * 8 + in_g - k * wide) * s.tile;
  k0 = k * s.tile;
}
// Item b of the grid.  The whole tiles run first, then the parts; each in
// contiguous eighths for the XCDs.  A part's tiles of 256 follow each other, so
// that an XCD's blocks read the same tokens (16384 tokens x 1024 x 1024: 62.3 us;
// a tile's parts after each other 67), of 128 a tile's parts (2048 x 1024 x 1024
// fp32: 33.8 us, the other way 36.9).
__device__ __forceinline__ WgradItem wgrad_item(const WgradTiles& s, uint64_t rows, uint32_t b) {
  WgradItem w;
  w.whole = b < s.full;
  if (w.whole) {
    w.tile = s.full <= gridDim.x ? remap_xcd(b, s.full) : b;
    w.split = 0;
    w.t_begin = 0;
    w.t_end = rows;
  } else {
    const uint32_t cut = s.tiles - s.full, parts = cut * s.splits;
    const uint32_t i = s.full + parts <= gridDim.x ? remap_xcd(b - s.full, parts) : b - s.full;
    w.split = s.big ? i / cut : i % s.splits;
    w.tile = s.full + (s.big ? i % cut : i / s.splits);
    w.t_begin = w.split * s.per_split;
    w.t_end = w.t_begin + s.per_split < rows ? w.t_begin + s.per_split : rows;
  }
  wgrad_place(s, w.tile, w.n0, w.k0);
  return w;
}
// Row n of a part's sums.
__device__ __forceinline__ float* wgrad_part(const WgradTiles& s, uint32_t tile, uint32_t split, uint32_t n) {
  return s.part + ((static_cast<uint64_t>(tile - s.full) * s.splits + split) * s.tile + n) * s.tile;
}

// What a lane's eight columns of k have besides their sums.
struct WgradCols {
  uint32_t k;
  int in;  // of the eight, that exist
  float scale[8], shift[8];
};
__device__ __forceinline__ WgradCols wgrad_cols(const Wgrad& a, uint32_t k, bool whole) {
  WgradCols c;
  c.k = k;
  c.in = static_cast<int>(a.k) - static_cast<int>(k);
  load_params8(whole ? a.col_scale : 0, a.param_dtype, k / 8, c.in, 1.0f, c.scale);
  load_params8(whole ? a.col_shift : 0, a.param_dtype, k / 8, c.in, 0.0f, c.shift);
  return c;
}
// The whole sums of row n at these columns, into dW.
__device__ __forceinline__ void wgrad_write8(const Wgrad& a, uint64_t n, const WgradCols& c, float sum, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= c.scale[e];
  if (a.col_shift) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += sum * c.shift[e];
  }
  const uint64_t at = n * a.dw.stride + c.k;
  float w[8];
  if (a.dw_dtype == kBf16) {
    const uint64_t p = a.dw.data + 2 * at;
    if (a.accumulate) {
      unpack8<kBf16>(load8_raw<kBf16>(p, c.in), w);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += w[e];
    }
    store8<kBf16>(p, v, c.in);
  } else {
    const uint64_t p = a.dw.data + 4 * at;
    if (a.accumulate) {
      unpack8<kF32>(load8_raw<kF32>(p, c.in), w);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += w[e];
    }
    store8<kF32>(p, v, c.in);
  }
}
// Row `ln` of the tile from the columns' first on: into the part of a split
// tile, else into dW.
__device__ __forceinline__ void wgrad_out8(const Wgrad& a, const WgradTiles& s, const WgradItem& w, const WgradCols& c,
                                           uint32_t ln, float sum, float (&v)[8]) {
  if (!w.whole) store8<kF32>(reinterpret_cast<uint64_t>(wgrad_part(s, w.tile, w.split, ln) + (c.k - w.k0)), v, 8);
  else if (w.n0 + ln < a.n && c.in > 0) wgrad_write8(a, w.n0 + ln, c, sum, v);
}
__device__ __forceinline__ void wgrad_write_bias(const Wgrad& a, uint64_t n, float sum) {
  if (a.accumulate) sum += load_param(a.dbias, n, a.dw_dtype);
  store_param(a.dbias, n, a.dw_dtype, sum);
}

// The next `rows` of an operand, 32 at most: an offset past the last one's end
// (and what may be read behind it) reads zeros; past another's end it reads the
// row behind it, whose columns are not stored.  The hardware looks at four bytes
// at a time: those that the end divides read zeros, too.
__device__ __forceinline__ tile_t step_tile(uint64_t base, int rows, uint32_t pitch, uint32_t width) {
  const uint32_t bytes = static_cast<uint32_t>(rows - 1) * pitch + width;
  return make_tile(reinterpret_cast<const void*>(base), rows > 0 ? bytes : 0u);
}
// The whole offset is in the operand that the bounds check covers; the scalar
// one is left at zero, for it need not count there.
template <typename T>
__device__ __forceinline__ T ld_step(tile_t t, uint32_t off) {
  if constexpr (sizeof(T) == 16) return __builtin_amdgcn_raw_buffer_load_b128(t, off, 0, 0);
  else return __builtin_amdgcn_raw_buffer_load_b8(t, off, 0, 0);
}

// ANY: rows of any length and stride, read an element at a time where they end;
// else of 8 columns of n and 16 of k at least, as far as 32-bit offsets reach.
template <int DT, bool SUMS, bool ANY>
__global__ __launch_bounds__(kThreads, 2) void wgrad_kernel(Wgrad a, WgradTiles s) {
  constexpr int P = kPlanes<DT>;
  constexpr uint32_t kIn = 2 * (P + 1) * kStep * kPitch * 2, kOutBytes = 4 * 64 * kOut * 4;
  __shared__ __align__(16) uint8_t lds[kIn > kOutBytes ? kIn : kOutBytes];  // two steps; then the waves' 64 rows of 64
  auto* const dys = reinterpret_cast<uint16_t(*)[P][kStep * kPitch]>(lds);
  auto* const xs = reinterpret_cast<uint16_t(*)[kStep * kPitch]>(lds + 2 * P * kStep * kPitch * 2);
  __shared__ float colsum[SUMS ? kThreads / 16 : 1][kTile];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t items = s.full + (s.tiles - s.full) * s.splits;
  for (uint32_t b = blockIdx.x; b < items; b += gridDim.x) {
    const WgradItem w = wgrad_item(s, a.rows, b);
    const uint32_t n0 = w.n0, k0 = w.k0;
    const uint64_t t_begin = w.t_begin, t_end = w.t_end;
    // a thread's share of a step: two groups of eight of dY, sixteen codes of X
    const uint32_t dc = tid % 16, dr = tid / 16;
    const int d_in = static_cast<int>(a.n) - static_cast<int>(n0 + 8 * dc);
    const uint32_t xc = tid % 8, xr = tid / 8;
    const int x_in = static_cast<int>(a.k) - static_cast<int>(k0 + 16 * xc);
    // a group that reaches past its row's end is read from before it, and moved
    // down on its way to LDS; one that lies past it reads what no one stores
    const uint32_t d_at = ANY || n0 + 8 * dc + 8 <= a.n ? n0 + 8 * dc : a.n - 8;
    const uint32_t x_at = ANY || k0 + 16 * xc + 16 <= a.k ? k0 + 16 * xc : a.k - 16;
    const uint32_t d_move = n0 + 8 * dc - d_at, x_move = k0 + 16 * xc - x_at;
    const uint32_t s_at = x_in > 0 ? (k0 + 16 * xc) / kActBlock : 0;
    const uint32_t d_pitch = static_cast<uint32_t>(a.dy.stride * kEsz<DT>), x_pitch = static_cast<uint32_t>(a.x.code_stride);
    const uint32_t s_pitch = static_cast<uint32_t>(a.x.scale_stride);
    const uint32_t d_from = dr * d_pitch + d_at * kEsz<DT>, x_from = xr * x_pitch + x_at, s_from = xr * s_pitch + s_at;
    struct Stage {
      Raw8<DT> d[2];
      Codes16 c;
    };
    float sum[8] = {};
    // Step t, zeros for the rows behind the last: loads without a condition, or
    // the compiler waits for the newest of them where it needs the oldest.
    auto load = [&](Stage& g, uint64_t t) {
      if constexpr (ANY) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint64_t r = t + dr + 16 * i;
          g.d[i] = load8_raw<DT>(a.dy.data + (r * a.dy.stride + d_at) * kEsz<DT>, r < t_end ? d_in : 0);
        }
        g.c = load_codes16(a.x, t + xr, x_at, t + xr < t_end ? x_in : 0);
      } else {
        const int rows = t + kStep <= t_end ? static_cast<int>(kStep) : t < t_end ? static_cast<int>(t_end - t) : 0;
        const tile_t td = step_tile(a.dy.data + t * a.dy.stride * kEsz<DT>, rows, d_pitch, a.n * kEsz<DT>);
        const tile_t tx = step_tile(a.x.codes + t * a.x.code_stride, rows, x_pitch, a.k);
        const tile_t ts = step_tile(a.x.scales + t * a.x.scale_stride, rows, s_pitch, (a.k + kActBlock - 1) / kActBlock);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int q = 0; q < static_cast<int>(kEsz<DT>) / 2; ++q)
            g.d[i].v[q] = ld_step<u32x4>(td, d_from + i * 16 * d_pitch + 16 * q);
        g.c.codes = ld_step<u32x4>(tx, x_from);
        g.c.code = ld_step<uint8_t>(ts, s_from);
      }
    };
    auto store = [&](Stage& g, int buf) {
      if constexpr (!ANY) {
        if (a.n % 8)
          for (auto& d : g.d) move_down8<DT>(d, d_move);
        if (a.k % 16) move_down16(g.c.codes, x_move);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t at = (dr + 16 * i) * kPitch + 8 * dc;
        if constexpr (SUMS) {
          float f[8];
          unpack8<DT>(g.d[i], f);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] += f[e];
        }
        if constexpr (P == 1) {
          *reinterpret_cast<u32x4*>(&dys[buf][0][at]) = g.d[i].v[0];
        } else {
          float f[8];
          unpack8<DT>(g.d[i], f);
          u32x4 q[3];
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            uint32_t part[3];
            split3(f[e], f[e + 1], part);
#pragma unroll
            for (int p = 0; p < 3; ++p) q[p][e / 2] = part[p];
          }
#pragma unroll
          for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4*>(&dys[buf][p][at]) = q[p];
        }
      }
      const float scale = __uint_as_float(g.c.code << 23);
      const u32x2 q0 = decode4(g.c.codes[0], scale), q1 = decode4(g.c.codes[1], scale);
      const u32x2 q2 = decode4(g.c.codes[2], scale), q3 = decode4(g.c.codes[3], scale);
      u32x4* p = reinterpret_cast<u32x4*>(&xs[buf][xr * kPitch + 16 * xc]);
      p[0] = u32x4{q0[0], q0[1], q1[0], q1[1]};
      p[1] = u32x4{q2[0], q2[1], q3[0], q3[1]};
    };

    f32x4 acc[4][4];  // [k][n] tiles of 16: a lane holds 4 neighbours of k for one n
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    const uint32_t wk = wave % 2 * 64, wn = wave / 2 * 64;
    auto multiply = [&](int buf) {
      bf16x8 xf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) xf[i] = read_cols(xs[buf], wk + 16 * i, lane);
#pragma unroll
      for (int p = P - 1; p >= 0; --p) {  // the small parts first
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8 df = read_cols(dys[buf][p], wn + 16 * j, lane);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[i], df, acc[i][j], 0, 0, 0);
        }
      }
    };
    // The next kAhead steps' loads are on their way while one multiplies (of
    // three parts a step, one: 2048 x 1024 x 1024 fp32 33.8 us, with two 35.7;
    // 8192 x 4096 x 4096 867 and 868).
    constexpr int kAhead = ANY || P > 1 ? 1 : 3;
    Stage g[kAhead];
    if (t_end <= t_begin + kStep) {  // one step at most: nothing else is loaded
      if (t_begin < t_end) {
        load(g[0], t_begin);
        store(g[0], 0);
        __syncthreads();
        multiply(0);
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int d = 0; d < kAhead; ++d) load(g[d], t_begin + d * kStep);
      store(g[0], 0);
      load(g[0], t_begin + kAhead * kStep);
      __syncthreads();
      int buf = 0;
      for (uint64_t t0 = t_begin; t0 < t_end; t0 += kAhead * kStep) {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) {
          const uint64_t t = t0 + d * kStep;
          if (t >= t_end) break;
          multiply(buf);
          Stage& next = g[(d + 1) % kAhead];
          if (t + kStep < t_end) store(next, buf ^ 1);
          load(next, t + (1 + kAhead) * kStep);
          __syncthreads();
          buf ^= 1;
        }
      }
    }

    if constexpr (SUMS) {
#pragma unroll
      for (int e = 0; e < 8; ++e) colsum[dr][8 * dc + e] = sum[e];
      __syncthreads();
      if (tid < kTile) {
        float v = colsum[0][tid];
#pragma unroll
        for (uint32_t r = 1; r < kThreads / 16; ++r) v += colsum[r][tid];
        colsum[0][tid] = v;
        const uint64_t n = n0 + tid;
        if (k0 == 0 && n < a.n) {
          if (!w.whole) s.sums[w.split * static_cast<uint64_t>(a.n) + n] = v;
          else if (a.dbias) wgrad_write_bias(a, n, v);
        }
      }
      __syncthreads();
    }
    // out through LDS, so that a lane has eight neighbours of k; the operands'
    // last reads lie before the loop's barrier
    float* const mine = reinterpret_cast<float*>(lds) + wave * 64 * kOut;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(mine + (16 * j + lane % 16) * kOut + 16 * i + lane / 16 * 4) = acc[i][j];
    const WgradCols cols = wgrad_cols(a, k0 + wk + lane % 8 * 8, w.whole);
#pragma unroll 2
    for (uint32_t q = lane / 8; q < 64; q += 8) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = mine[q * kOut + lane % 8 * 8 + e];
      wgrad_out8(a, s, w, cols, wn + q, SUMS ? colsum[0][wn + q] : 0.0f, v);
    }
    __syncthreads();
  }
}

// ---- large products of a bf16 dY -------------------------------------------------------
// 256 x 256 of dW a block, four waves of 128 x 128, one block a CU: at 64 x 64
// a wave the LDS reads alone take as long as the products (128 B a clock;
// 512 B a 16 x 16 x 32 product's two operands against its 16 clocks, halved by
// each doubling of a wave's side).  Tokens come in steps of 32 through two LDS
// buffers; a thread's loads run two to three steps ahead in registers, and the
// operands of a half step are read while the half before it multiplies, so one
// barrier a step is all that a wave waits for.
//
// A row of 256 columns is 16 slots of 32 bytes; slot c of token r lies at
// c ^ 2 (r % 4), which spreads the four tokens that a transposing read takes
// from a column over the banks.  Of X's columns, where a thread writes 16, the
// first eight of every 16 are in the first eight slots and the others behind
// them, so that the threads' 16 bytes lie side by side (two writes 32 bytes
// apart would meet in the banks); a wave's 128 of k are therefore every other
// eight.
constexpr uint32_t kBigTile = 256;
constexpr uint32_t kBigRow = kBigTile * 2;          // bytes
constexpr uint32_t kBigBuf = kStep * kBigRow;       // bytes of one operand's step
constexpr uint32_t kBigOut = 128 + 4;               // floats from row to row on their way out
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

// Kinds of instructions, for their order.
constexpr int kValu = 0x2, kMfma = 0x8, kVmemRead = 0x20, kLdsRead = 0x100, kLdsWrite = 0x200;
// What a thread holds of a step: 4 x 8 of dY, 2 x 16 codes of X.
struct BigStage {
  u32x4 dy[4];
  u32x4 x[2];
  uint32_t scale[2];
};

// RAGGED: rows that end inside 16 bytes.
template <bool RAGGED>
__global__ __launch_bounds__(kThreads, 1) void wgrad_big_kernel(Wgrad a, WgradTiles s) {
  // dY, dY, X, X; at the end the waves' 32 rows of 128
  __shared__ __align__(256) uint8_t lds[4 * 32 * kBigOut * 4 > 4 * kBigBuf ? 4 * 32 * kBigOut * 4 : 4 * kBigBuf];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  lds_u8* const base = (lds_u8*)lds;
  // where the thread's share of a step comes from and goes to
  const uint32_t dr = tid / 32, dc = tid % 32, xr = tid / 16, xc = tid % 16;
  const uint32_t dy_pitch = static_cast<uint32_t>(a.dy.stride * 2), x_pitch = static_cast<uint32_t>(a.x.code_stride);
  const uint32_t s_pitch = static_cast<uint32_t>(a.x.scale_stride);
  const uint32_t dy_from = dr * dy_pitch + dc * 16, x_from = xr * x_pitch + xc * 16, s_from = xr * s_pitch + xc / 2;
  lds_u8* const dy_to = base + dr * kBigRow + (dc / 2 ^ dr % 4 * 2) * 32 + dc % 2 * 16;
  lds_u8* const x_to = base + 2 * kBigBuf + xr * kBigRow + (xc / 2 ^ xr % 4 * 2) * 32 + xc % 2 * 16;
  // where the wave's operands are: a lane reads column lane % 32, tokens lane / 32 * 8 and on
  const uint32_t wk = wave % 2 * 128, wn = wave / 2 * 128;
  const uint32_t x4 = lane % 16 / 4;  // token of the four that the lane's address names
  const uint32_t row = lane / 32 * 8 + x4, half = lane / 16 % 2;
  lds_u8 *x_at[4], *dy_at[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t at = row * kBigRow + (2 * (i ^ x4) + half) * 32 + lane % 4 * 8;
    x_at[i] = base + 2 * kBigBuf + at + wk * 2;
    dy_at[i] = base + at + wn * 2;
  }
  // what the tile's rows and columns have besides their products
  __shared__ __align__(16) float row_sum[kBigTile], row_last[kBigTile], col_scale[kBigTile], col_shift[kBigTile], col_last[kBigTile];
  const uint32_t items = s.full + (s.tiles - s.full) * s.splits;
  for (uint32_t b = blockIdx.x; b < items; b += gridDim.x) {
    const WgradItem w = wgrad_item(s, a.rows, b);
    const uint32_t n0 = w.n0, k0 = w.k0;
    // Where rows end inside 16 bytes, a thread reads up to 16 bytes behind them:
    // the row that follows has them.  Nothing follows the last one, whose product
    // is added at the end.  Of a step of fewer than 32 rows that reach ends inside
    // the row behind, so the threads of the rows that are not there read from
    // `kNowhere`, past any step's end (25743 x 1173 x 768: 0.8 us of 80): the
    // last row's columns must not come in a second time.
    constexpr uint32_t behind = RAGGED ? 16 : 0;
    constexpr uint32_t kNowhere = 1u << 31;
    const bool last = RAGGED && w.t_end == a.rows && a.rows > 0;
    const uint64_t t_begin = w.t_begin, t_end = last ? w.t_end - 1 : w.t_end;
    // the next step to load; nothing is left of one behind the last
    int left = static_cast<int>(t_end - t_begin);
    uint64_t dy_next = a.dy.data + (t_begin * a.dy.stride + n0) * 2;
    uint64_t x_next = a.x.codes + t_begin * a.x.code_stride + k0;
    uint64_t s_next = a.x.scales + t_begin * a.x.scale_stride + k0 / kActBlock;
    const uint32_t dy_width = (a.n - n0) * 2 + behind, x_width = a.k - k0 + behind;
    const uint32_t s_width = (a.k - k0 + kActBlock - 1) / kActBlock;
    auto load = [&](BigStage& g) {
      const int rows = left < static_cast<int>(kStep) ? left : static_cast<int>(kStep);
      const tile_t td = step_tile(dy_next, rows, dy_pitch, dy_width);
      const tile_t tx = step_tile(x_next, rows, x_pitch, x_width);
      const tile_t ts = step_tile(s_next, rows, s_pitch, s_width);
      left -= kStep;
      dy_next += static_cast<uint64_t>(dy_pitch) * kStep;
      x_next += static_cast<uint64_t>(x_pitch) * kStep;
      s_next += static_cast<uint64_t>(s_pitch) * kStep;
      const auto there = [&](uint32_t row, uint32_t from) { return !RAGGED || static_cast<int>(row) < rows ? from : kNowhere; };
#pragma unroll
      for (int i = 0; i < 4; ++i)
        g.dy[i] = ld_step<u32x4>(td, there(dr + 8 * i, dy_from + i * 8 * dy_pitch));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        g.x[i] = ld_step<u32x4>(tx, there(xr + 16 * i, x_from + i * 16 * x_pitch));
        g.scale[i] = ld_step<uint8_t>(ts, s_from + i * 16 * s_pitch);
      }
    };
    // a step's share in eight writes, a half step's operands in eight reads
    auto store = [&](const BigStage& g, uint32_t buf, int part) {
      if (part < 4) {
        *(lds_u32x4*)(dy_to + buf * kBigBuf + part * 8 * kBigRow) = g.dy[part];
        return;
      }
      const int i = part / 2 - 2, h = part % 2;
      const float scale = __uint_as_float(g.scale[i] << 23);
      const u32x2 lo = decode4(g.x[i][2 * h], scale), hi = decode4(g.x[i][2 * h + 1], scale);
      *(lds_u32x4*)(x_to + buf * kBigBuf + i * 16 * kBigRow + h * 256) = u32x4{lo[0], lo[1], hi[0], hi[1]};
    };
    bf16x8 xf[2][4], df[2][4];
    auto fetch = [&](uint32_t to, uint32_t buf, uint32_t h, int part) {
      // in the order in which the products want them
      lds_u8* const p = (part == 0 ? x_at[0] : part < 5 ? dy_at[part - 1] : x_at[part - 4]) + buf * kBigBuf + h * 16 * kBigRow;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * kBigRow));
      const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      if (part == 0) xf[to][0] = v;
      else if (part < 5) df[to][part - 1] = v;
      else xf[to][part - 4] = v;
    };
    f32x16 acc[4][4];  // [k][n] tiles of 32: a lane holds four runs of 4 of k for one n
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    auto multiply = [&](uint32_t of, int i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xf[of][i], df[of][j], acc[i][j], 0, 0, 0);
    };
    // One step, out of buffer `buf`; g holds the one behind it.  Each product
    // takes 32 clocks of the matrix core; the order below lays the other
    // instructions between them, so that neither the LDS of the CU, which the
    // four waves share, nor the wave's issue holds the products up.
    auto step = [&](BigStage& g, uint32_t buf) {
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        fetch(1, buf, 1, p);
        store(g, buf ^ 1, p);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) multiply(0, i);
      multiply(1, 0);
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kLdsRead, 2, 0);
        __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
        if (p >= 4) __builtin_amdgcn_sched_group_barrier(kValu, 5, 0);
        __builtin_amdgcn_sched_group_barrier(kLdsWrite, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(kMfma, 4, 0);
      __builtin_amdgcn_sched_barrier(0);
      __syncthreads();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = 0; p < 8; ++p) fetch(0, buf ^ 1, 0, p);
      load(g);
#pragma unroll
      for (int i = 1; i < 4; ++i) multiply(1, i);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kLdsRead, 2, 0);
        __builtin_amdgcn_sched_group_barrier(kVmemRead, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(kMfma, 4, 0);
      __builtin_amdgcn_sched_barrier(0);
    };
    BigStage g0, g1;  // the odd steps on their way, and the even ones
    load(g1);
    load(g0);
    // a wave for each, so that their loads do not wait for one another
    for (uint32_t i = lane; i < kBigTile; i += 64) {
      const uint64_t n = n0 + i, k = k0 + i;
      const bool on_n = n < a.n, on_k = k < a.k;
      if (wave == 0) {
        col_scale[i] = a.col_scale && on_k ? load_param(a.col_scale, k, a.param_dtype) : 1.0f;
      } else if (wave == 1) {
        col_shift[i] = a.col_shift && on_k ? load_param(a.col_shift, k, a.param_dtype) : 0.0f;
      } else if (wave == 2) {
        row_sum[i] = a.col_shift && on_n ? s.sums[n] : 0.0f;
        if (last) row_last[i] = on_n ? load1<kBf16>(a.dy.data + ((a.rows - 1) * a.dy.stride + n) * 2) : 0.0f;
      } else if (last) {
        const uint32_t code = on_k ? *(gc_u8*)(a.x.codes + (a.rows - 1) * a.x.code_stride + k) : 0;
        const float scale = on_k ? act_scale(load_kept_code(a.x, a.rows - 1, k / 8)) : 0.0f;
        col_last[i] = __builtin_amdgcn_cvt_f32_fp8(code, 0) * scale;
      }
    }
#pragma unroll
    for (int p = 0; p < 8; ++p) store(g1, 0, p);
    load(g1);
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 8; ++p) fetch(0, 0, 0, p);
    for (uint64_t t = t_begin; t < t_end; t += 2 * kStep) {  // a step behind the last multiplies zeros
      step(g0, 0);
      step(g1, 1);
    }
    __syncthreads();

    // out of the registers through LDS, 32 rows of dW a wave at a time, so
    // that a lane has eight neighbours of k (every other eight: see above)
    float* const mine = reinterpret_cast<float*>(lds) + wave * 32 * kBigOut;
    const uint32_t lk = lane % 16 * 16 + wk / 16;
    WgradCols cols;
    cols.k = k0 + lk;
    cols.in = static_cast<int>(a.k) - static_cast<int>(cols.k);
    float x_last[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cols.scale[e] = col_scale[lk + e];
      cols.shift[e] = col_shift[lk + e];
      x_last[e] = last ? col_last[lk + e] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const f32x4 v = {acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2], acc[i][j][4 * r + 3]};
          *reinterpret_cast<f32x4*>(mine + lane % 32 * kBigOut + 32 * i + 8 * r + lane / 32 * 4) = v;
        }
#pragma unroll 4
      for (uint32_t q = lane / 16; q < 32; q += 4) {
        const uint32_t ln = wn + 32 * j + q;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = mine[q * kBigOut + lane % 16 * 8 + e];
        if (last) {
          const float d = row_last[ln];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(d, x_last[e], v[e]);
        }
        wgrad_out8(a, s, w, cols, ln, row_sum[ln], v);
      }
    }
    __syncthreads();
  }
}

// The parts' sums with the columns' scale and shift.  SLICES threads share eight
// columns of a row of dW: each adds every SLICES-th part, then the first adds the
// others' sums, in a fixed order.  AHEAD: parts that a thread has under way.
template <uint32_t SLICES, uint32_t AHEAD>
__global__ __launch_bounds__(kThreads) void wgrad_join_kernel(Wgrad a, WgradTiles s) {
  constexpr uint32_t G = kThreads / SLICES;  // groups of eight columns a block
  __shared__ float sums[SLICES][9][G];
  const uint32_t per_row = s.tile / 8, blocks = s.tile * per_row / G;  // of a tile
  const uint32_t own = threadIdx.x % G, slice = threadIdx.x / G;
  for (uint32_t it = blockIdx.x; it < (s.tiles - s.full) * blocks; it += gridDim.x) {
    const uint32_t tile = s.full + it / blocks, in_t = it % blocks * G + own;
    const uint32_t ln = in_t / per_row, lk = in_t % per_row * 8;
    uint32_t n0, k0;
    wgrad_place(s, tile, n0, k0);
    const uint64_t n = n0 + ln;
    const int in = static_cast<int>(a.k) - static_cast<int>(k0 + lk);
    const bool on = n < a.n && in > 0;
    const bool bias = a.dbias && !s.big && k0 + lk == 0;
    float v[8] = {}, f[8], sum = 0;
    if (on) {
#pragma unroll (AHEAD)
      for (uint32_t p = slice; p < s.splits; p += SLICES) {  // a part is a whole tile, also where dW ends
        unpack8<kF32>(load8_raw<kF32>(reinterpret_cast<uint64_t>(wgrad_part(s, tile, p, ln) + lk)), f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += f[e];
      }
      if (a.col_shift || bias) {
#pragma unroll 4
        for (uint32_t p = slice; p < s.sum_parts; p += SLICES) sum += s.sums[p * static_cast<uint64_t>(a.n) + n];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[slice][e][own] = v[e];
    sums[slice][8][own] = sum;
    __syncthreads();
    if (slice == 0 && on) {
#pragma unroll
      for (uint32_t q = 1; q < SLICES; ++q) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += sums[q][e][own];
        sum += sums[q][8][own];
      }
      if (bias) wgrad_write_bias(a, n, sum);
      wgrad_write8(a, n, wgrad_cols(a, k0 + lk, true), sum, v);
    }
    __syncthreads();
  }
}

// Column sums of a bf16 dY of at least eight columns, for wgrad_big_kernel: 512
// columns and a part of the tokens a block, then the parts in order.  Loads
// without a condition, eight under way: a lane at or behind the row's end sums its
// last eight columns, as the lanes before do.  25743 x 1173: 48 us with the tail
// an element at a time and four waves a block, 12 so.
constexpr uint32_t kSumCols = 512, kSumParts = 64, kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void wgrad_sums_kernel(Wgrad a, float* parts) {
  __shared__ float sums[kSumThreads / 64][kSumCols];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t chunks = (a.n + kSumCols - 1) / kSumCols, items = chunks * kSumParts;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t c0 = it % chunks * kSumCols, p = it / chunks;
    const uint64_t t0 = a.rows * p / kSumParts, t1 = a.rows * (p + 1) / kSumParts;
    const uint64_t at = c0 + 8 * lane + 8 <= a.n ? c0 + 8 * lane : a.n - 8;
    float f[8], v[8] = {};
#pragma unroll 8
    for (uint64_t t = t0 + wave; t < t1; t += kSumThreads / 64) {
      unpack8<kBf16>(load8_raw<kBf16>(a.dy.data + (t * a.dy.stride + at) * 2), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += f[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at + e >= c0) sums[wave][at + e - c0] = v[e];  // twice, where two lanes have a column: the same sum
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kSumCols && c0 + i < a.n; i += kSumThreads) {
      float w = sums[0][i];
#pragma unroll
      for (uint32_t q = 1; q < kSumThreads / 64; ++q) w += sums[q][i];
      parts[p * a.n + c0 + i] = w;
    }
    __syncthreads();
  }
}
__global__ __launch_bounds__(64) void wgrad_sums_join_kernel(Wgrad a, const float* parts, float* sums) {
  for (uint64_t n = blockIdx.x * 64ull + threadIdx.x; n < a.n; n += gridDim.x * 64ull) {
    float v = 0;
#pragma unroll 16
    for (uint32_t p = 0; p < kSumParts; ++p) v += parts[p * static_cast<uint64_t>(a.n) + n];
    sums[n] = v;
    if (a.dbias) wgrad_write_bias(a, n, v);
  }
}

// The cut.  More parts shorten what a block takes over the tokens and cost
// their sums' way through memory.  The figures are measured (us): what a block
// of 256 columns takes beside its steps 12 (ragged 17), a step of 32 tokens 0.6,
// with every CU at work 0.85; of 128 columns 9 (behind another 4), 0.53 and, two
// a CU, 0.77, of an fp32 dY 1.2 and 1.65; a part's sums there and back 0.105 and
// 0.018, the join's launch 4 and 0.02 a part.
WgradTiles wgrad_tiles(uint64_t rows, uint64_t n, uint64_t k, bool big, bool wide, double* best_us) {
  WgradTiles s{};
  s.big = big;
  s.ragged = n % 8 != 0 || k % 16 != 0;
  s.tile = big ? kBigTile : kTile;
  s.tn = static_cast<uint32_t>((n + s.tile - 1) / s.tile);
  s.tk = static_cast<uint32_t>((k + s.tile - 1) / s.tile);
  s.tiles = s.tn * s.tk;
  const uint32_t at_once = big ? 256 : 512, rest = s.tiles % at_once;
  const uint64_t rounds = s.tiles / at_once, steps = (rows + kStep - 1) / kStep;
  const double block_us = !big ? 9.0 : s.ragged ? 17.0 : 12.0, next_us = big ? block_us : 4.0, part_us = big ? 0.105 : 0.018;
  const double one_us = big ? 0.6 : wide ? 1.2 : 0.53, all_us = big ? 0.85 : wide ? 1.65 : 0.77;
  const double whole_us = rounds ? rounds * steps * all_us + block_us + (rounds - 1) * next_us : 0.0;
  uint64_t best = 1;
  *best_us = 1e30;
  // the small kernel splits every tile or none: it takes a whole tile's column
  // sums along, and the parts of a column of tiles have to be alike
  for (uint64_t splits = 1; splits == 1 || (rest && (big || !rounds) && splits <= at_once / rest && splits <= steps);
       splits += 1 + splits / 16) {
    const double blocks = static_cast<double>(splits) * rest;
    const double fill = big ? blocks / 256 : blocks > 256 ? (blocks - 256) / 256 : 0.0;  // of the CUs; of their second places
    const double us = whole_us + (rest ? (steps + splits - 1) / splits * (one_us + (all_us - one_us) * fill) + (rounds ? next_us : block_us) : 0.0) +
                      (splits > 1 ? blocks * part_us + 4.0 + 0.02 * splits : 0.0);
    if (us < *best_us) {
      *best_us = us;
      best = splits;
    }
  }
  s.per_split = (steps + best - 1) / best * kStep;
  s.splits = steps ? static_cast<uint32_t>((rows + s.per_split - 1) / s.per_split) : 1;
  s.full = s.splits > 1 ? s.tiles - rest : s.tiles;
  s.sum_parts = big ? 1 : s.splits;
  return s;
}

// Whether 32 rows lie within 32-bit offsets.
bool wgrad_in_reach(const Wgrad& a) {
  return a.dy.stride < (1u << 24) && a.x.code_stride < (1u << 26) && a.x.scale_stride < (1u << 26);
}
// The 256-column kernel takes a bf16 dY.
bool wgrad_may_be_big(const Wgrad& a) {
  return a.dtype == kBf16 && a.n >= 8 && a.k >= 16 && wgrad_in_reach(a) && a.rows < (1u << 30);
}

uint64_t wgrad_part_bytes(const WgradTiles& s) {
  return static_cast<uint64_t>(s.tiles - s.full) * s.splits * s.tile * s.tile * 4;
}
template <int DT>
hipError_t wgrad_of(const Wgrad& a, const WgradTiles& s, uint32_t grid, bool sums, hipStream_t st) {
  if (a.n < 8 || a.k < 16 || !wgrad_in_reach(a))
    return launch_op(sums ? wgrad_kernel<DT, true, true> : wgrad_kernel<DT, false, true>, grid, kThreads, st, a, s);
  return launch_op(sums ? wgrad_kernel<DT, true, false> : wgrad_kernel<DT, false, false>, grid, kThreads, st, a, s);
}
constexpr uint64_t kJoinAlone = 98304;  // groups of eight columns from which a thread adds all parts of one
template <uint32_t SLICES, uint32_t AHEAD>
hipError_t wgrad_join(const Wgrad& a, const WgradTiles& s, hipStream_t st) {
  const uint32_t blocks = (s.tiles - s.full) * (s.tile * s.tile / 8 * SLICES / kThreads);
  return launch_op(wgrad_join_kernel<SLICES, AHEAD>, grid_for(blocks, kThreads), kThreads, st, a, s);
}
uint64_t wgrad_space(const WgradTiles& s, uint64_t n) {
  return wgrad_part_bytes(s) + (s.sum_parts + (s.big ? kSumParts : 0)) * n * 4;
}

}  // namespace

uint64_t wgrad_workspace(uint64_t rows, uint64_t n, uint64_t k) {
  // which tiles a call takes goes by its types and alignment, too
  double us;
  const uint64_t big = wgrad_space(wgrad_tiles(rows, n, k, true, false, &us), n);
  const uint64_t narrow = wgrad_space(wgrad_tiles(rows, n, k, false, false, &us), n);
  const uint64_t wide = wgrad_space(wgrad_tiles(rows, n, k, false, true, &us), n);
  return std::max(big, std::max(narrow, wide));
}

hipError_t launch_wgrad(const Wgrad& a, hipStream_t st) {
  double us, big_us;
  WgradTiles s = wgrad_tiles(a.rows, a.n, a.k, false, a.dtype == kF32, &us);
  if (wgrad_may_be_big(a)) {
    const WgradTiles big = wgrad_tiles(a.rows, a.n, a.k, true, false, &big_us);
    if (big_us <= us) s = big;
  }
  s.part = reinterpret_cast<float*>(a.ws);
  s.sums = reinterpret_cast<float*>(a.ws + wgrad_part_bytes(s));
  const bool sums = a.dbias || a.col_shift;
  const uint32_t grid = grid_for(s.full + (s.tiles - s.full) * s.splits, kThreads);
  hipError_t e;
  if (s.big) {
    if (sums) {
      float* const parts = s.sums + a.n;
      e = launch_op(wgrad_sums_kernel, grid_for((a.n + kSumCols - 1) / kSumCols * kSumParts, kSumThreads), kSumThreads, st, a, parts);
      if (e != hipSuccess) return e;
      e = launch_op(wgrad_sums_join_kernel, grid_for((a.n + 63) / 64, 64), 64, st, a, parts, s.sums);
      if (e != hipSuccess) return e;
    }
    e = launch_op(s.ragged ? wgrad_big_kernel<true> : wgrad_big_kernel<false>, grid, kThreads, st, a, s);
  } else {
    e = a.dtype == kBf16 ? wgrad_of<kBf16>(a, s, grid, sums, st) : wgrad_of<kF32>(a, s, grid, sums, st);
  }
  if (e != hipSuccess || s.splits == 1) return e;
  const uint64_t groups = static_cast<uint64_t>(s.tiles - s.full) * s.tile * s.tile / 8;
  if (s.splits <= 2) return wgrad_join<1, 2>(a, s, st);
  if (groups >= kJoinAlone) return s.splits <= 4 ? wgrad_join<1, 4>(a, s, st) : wgrad_join<1, 8>(a, s, st);
  return s.splits <= 4 ? wgrad_join<4, 1>(a, s, st) : wgrad_join<8, 4>(a, s, st);
}

}  // namespace lc
