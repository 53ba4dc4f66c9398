// Layer norm and RMS norm of rows, forward and backward.
//
//   n = (x - mean) * rstd,  rstd = 1 / sqrt(var + eps)     (RMS: mean 0, var = mean of x^2)
//   y = n * w + b
//   g = dy * w;  dx = rstd * (g - mean(g) - n * mean(g * n))     (RMS: without mean(g))
//   dw = sum over rows of dy * n;  db = sum over rows of dy
//
// Bound by memory: a row is read once and stays in registers, the variance is
// taken about the mean found before it, sums are fp32.  The forward pass may
// keep n in 8 bits, and the backward pass take it from there instead of x.  The
// sums over rows are split over blocks and joined in a fixed order.
#include "lc_ops_device.h"

namespace lc {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// TPR threads a row, NV groups of eight elements a thread.
template <int TPR>
constexpr uint32_t kNormThreads = TPR < 256 ? 256 : TPR;

// Sums of (a, b) over the TPR threads of a row, in each of them.  `red` holds
// two sets of slots used in turn: a set is written again only behind the next
// call's barrier.
template <int TPR>
__device__ __forceinline__ void row_sum2(float& a, float& b, float2 (&red)[2][kNormThreads<TPR> / 64], uint32_t& turn) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (TPR > 64) {
    constexpr uint32_t W = TPR / 64;
    const uint32_t wave = threadIdx.x >> 6, w0 = wave / W * W;
    if ((threadIdx.x & 63) == 0) red[turn][wave] = make_float2(a, b);
    __syncthreads();
    a = red[turn][w0].x;
    b = red[turn][w0].y;
#pragma unroll
    for (uint32_t w = 1; w < W; ++w) {
      a += red[turn][w0 + w].x;
      b += red[turn][w0 + w].y;
    }
    turn ^= 1;
  }
}
template <int TPR>
__device__ __forceinline__ float row_sum(float a, float2 (&red)[2][kNormThreads<TPR> / 64], uint32_t& turn) {
  float b = 0;
  row_sum2<TPR>(a, b, red, turn);
  return a;
}

template <int DT, bool LAYER, int TPR, int NV>
__global__ __launch_bounds__(kNormThreads<TPR>) void norm_fwd_kernel(NormFwd a) {
  constexpr uint32_t RPB = kNormThreads<TPR> / TPR;
  __shared__ float2 red[2][kNormThreads<TPR> / 64];
  uint32_t turn = 0;
  const uint32_t t = threadIdx.x % TPR;
  const float inv_dim = 1.0f / static_cast<float>(a.dim);
  const uint64_t items = (a.rows + RPB - 1) / RPB;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t row = row_item(it, items) * RPB + threadIdx.x / TPR;
    const bool on = row < a.rows;  // the others only take part in the barriers
    Raw8<DT> r[NV];
    float sum = 0, unused = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t g = i * TPR + t;
      r[i] = load8_row<DT, kStreams<DT>>(a.x.data + row * a.x.stride * kEsz<DT>, g, on ? in_group(a.dim, g) : 0);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) trim8_row<DT>(r[i], a.dim, in_group(a.dim, i * TPR + t));
    float v[8];
    float mean = 0;
    if constexpr (LAYER) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        unpack8<DT>(r[i], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e];
      }
      mean = row_sum<TPR>(sum, red, turn) * inv_dim;
    }
    float sq = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int n = in_group(a.dim, i * TPR + t);
      unpack8<DT>(r[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = !LAYER ? v[e] : e < n ? v[e] - mean : 0.0f;
        sq = __builtin_fmaf(d, d, sq);
      }
    }
    row_sum2<TPR>(sq, unused, red, turn);
    const float rstd = 1.0f / sqrtf(sq * inv_dim + a.eps);
    if (!on) continue;
    if (t == 0) {
      if (LAYER && a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t g = i * TPR + t;
      const int n = in_group(a.dim, g);
      float w[8], b[8], y[8];
      load_params8(a.weight, a.param_dtype, g, n, 1.0f, w);
      if constexpr (LAYER) load_params8(a.bias, a.param_dtype, g, n, 0.0f, b);
      unpack8<DT>(r[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = (LAYER ? v[e] - mean : v[e]) * rstd;
        y[e] = v[e] * w[e];
        if constexpr (LAYER) y[e] += b[e];
      }
      store8<DT, kStreams<DT>>(a.y.data + (row * a.y.stride + 8ull * g) * kEsz<DT>, y, n);
      if (a.kept.codes) {
        if (n < 8) {  // what is no element must not set its block's power: a NaN row has one here, too
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = e < n ? v[e] : 0.0f;
        }
        uint32_t code;
        const u32x2 q = act_encode8(v, code);
        store_kept8(a.kept, row, g, n, q, code);
      }
    }
  }
}

// Rows of any length (fewer than 8 columns, or beyond kNormLongest): read again
// for each of the three steps.
constexpr uint32_t kLongThreads = 1024;
template <int DT, bool LAYER>
__global__ __launch_bounds__(kLongThreads) void norm_fwd_long_kernel(NormFwd a) {
  __shared__ float2 red[2][kLongThreads / 64];
  uint32_t turn = 0;
  const float inv_dim = 1.0f / static_cast<float>(a.dim);
  const uint32_t groups = (a.dim + 31) / 32 * 4;  // whole quads, so that a block's four lanes stay together
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const uint64_t src = a.x.data + row * a.x.stride * kEsz<DT>;
    float mean = 0, sum = 0, unused = 0;
    float v[8];
    if constexpr (LAYER) {
      for (uint32_t g = threadIdx.x; g < groups; g += kLongThreads) {
        unpack8<DT>(load8_raw<DT>(src + 8ull * g * kEsz<DT>, in_group(a.dim, g)), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e];
      }
      mean = row_sum<kLongThreads>(sum, red, turn) * inv_dim;
    }
    float sq = 0;
    for (uint32_t g = threadIdx.x; g < groups; g += kLongThreads) {
      const int n = in_group(a.dim, g);
      unpack8<DT>(load8_raw<DT>(src + 8ull * g * kEsz<DT>, n), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = e < n ? v[e] - mean : 0.0f;
        sq = __builtin_fmaf(d, d, sq);
      }
    }
    row_sum2<kLongThreads>(sq, unused, red, turn);
    const float rstd = 1.0f / sqrtf(sq * inv_dim + a.eps);
    if (threadIdx.x == 0) {
      if (LAYER && a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    for (uint32_t g = threadIdx.x; g < groups; g += kLongThreads) {
      const int n = in_group(a.dim, g);
      unpack8<DT>(load8_raw<DT>(src + 8ull * g * kEsz<DT>, n), v);
      float w[8], b[8], y[8];
      load_params8(a.weight, a.param_dtype, g, n, 1.0f, w);
      load_params8(LAYER ? a.bias : 0, a.param_dtype, g, n, 0.0f, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = e < n ? (v[e] - mean) * rstd : 0.0f;
        y[e] = v[e] * w[e] + b[e];
      }
      store8<DT>(a.y.data + (row * a.y.stride + 8ull * g) * kEsz<DT>, y, n);
      if (a.kept.codes) {
        uint32_t code;
        const u32x2 q = act_encode8(v, code);
        store_kept8(a.kept, row, g, n, q, code);
      }
    }
  }
}

// ---- backward ------------------------------------------------------------------------
// Partial sums of dw and db: `parts` rows of dim each, dw's first.
struct NormParts {
  uint32_t rpb;    // rows that a block takes at once
  uint32_t parts;
};

// What a thread has of group g of a row before it is normalised.
template <int DT, bool KEPT>
struct NormIn {
  Raw8<DT> dy;
  Raw8<DT> x;
};
template <int DT>
struct NormIn<DT, true> {
  Raw8<DT> dy;
  u32x2 codes;
  uint32_t code;
};
// ANY: rows of any length, else of eight elements at least.
template <int DT, bool KEPT, bool ANY>
__device__ __forceinline__ NormIn<DT, KEPT> load_normed(const NormBwd& a, uint64_t row, uint32_t g, int n) {
  NormIn<DT, KEPT> in;
  const uint64_t dy = a.dy.data + row * a.dy.stride * kEsz<DT>;
  in.dy = ANY ? load8_raw<DT>(dy + 8ull * g * kEsz<DT>, n) : load8_row<DT, kStreams<DT>>(dy, g, n);
  if constexpr (KEPT) {
    in.code = n > 0 ? load_kept_code(a.kept, row, g) : 0;
    in.codes = ANY ? load_kept8(a.kept, row, g, n) : load_codes8_row(a.kept.codes + row * a.kept.code_stride, g, n);
  } else {
    const uint64_t x = a.x.data + row * a.x.stride * kEsz<DT>;
    in.x = ANY ? load8_raw<DT>(x + 8ull * g * kEsz<DT>, n) : load8_row<DT, kStreams<DT>>(x, g, n);
  }
  return in;
}
template <int DT, bool KEPT>
__device__ __forceinline__ void trim_normed(NormIn<DT, KEPT>& in, uint32_t dim, int n) {
  trim8_row<DT>(in.dy, dim, n);
  if constexpr (KEPT) in.codes = trim_codes8_row(in.codes, n);
  else trim8_row<DT>(in.x, dim, n);
}
// dy and n of the group; zeros behind the row's end.
template <int DT, bool KEPT>
__device__ __forceinline__ void normed8(const NormIn<DT, KEPT>& in, int n, float mean, float rstd, float (&d)[8],
                                        float (&f)[8]) {
  unpack8<DT>(in.dy, d);
  if constexpr (KEPT) {
    act_decode8(in.codes, act_scale(in.code), f);
  } else {
    unpack8<DT>(in.x, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (f[e] - mean) * rstd;
    if (n < 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = e < n ? f[e] : 0.0f;
    }
  }
}

// A block keeps its columns' weights and sums in registers and takes its turn
// at the rows.  The next row's loads in registers meanwhile, for fewer blocks a
// CU, cost more than they hide (bf16, us: 16384 x 4096 RMS norm from kept rows 75
// for 65, layer norm 71 for 69; 4096 x 16384 layer norm 92 for 79; 8192 x 8192
// 74 for 75).  dx goes through the caches, where what follows may find it.  Past
// them, of 16384 x 4096 from five sets of arrays in turn: from x 78.0 us for 74.5,
// from kept rows 66.9 for 68.5, of one set over and over 79 for 75 and 65 for 65.
template <int DT, bool LAYER, bool KEPT, int TPR, int NV>
__global__ __launch_bounds__(kNormThreads<TPR>) void norm_bwd_kernel(NormBwd a, uint32_t parts) {
  constexpr uint32_t RPB = kNormThreads<TPR> / TPR;
  __shared__ float2 red[2][kNormThreads<TPR> / 64];
  uint32_t turn = 0;
  const uint32_t t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const float inv_dim = 1.0f / static_cast<float>(a.dim);
  // The weights in LDS where registers for them would spill (128 a thread of 1024;
  // 4096 x 16384 layer norm in bf16 110 us with the spills, 79 without).
  constexpr bool kWeightsInLds = LAYER && TPR == 1024;
  __shared__ __align__(16) float w_lds[kWeightsInLds ? NV * TPR * 8 : 1];
  float w_reg[kWeightsInLds ? 1 : NV][8], dw[NV][8] = {}, db[LAYER ? NV : 1][8] = {};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const uint32_t g = i * TPR + t;
    float(&w)[8] = w_reg[kWeightsInLds ? 0 : i];
    load_params8(a.weight, a.param_dtype, g, in_group(a.dim, g), 1.0f, w);
    if constexpr (kWeightsInLds) {  // each thread reads its own again
      reinterpret_cast<f32x4*>(w_lds)[i * TPR + t] = f32x4{w[0], w[1], w[2], w[3]};
      reinterpret_cast<f32x4*>(w_lds)[(NV + i) * TPR + t] = f32x4{w[4], w[5], w[6], w[7]};
    }
  }
  auto weights = [&](int i, float(&w)[8]) {
    if constexpr (kWeightsInLds) {
      const f32x4 lo = reinterpret_cast<const f32x4*>(w_lds)[i * TPR + t], hi = reinterpret_cast<const f32x4*>(w_lds)[(NV + i) * TPR + t];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = e < 4 ? lo[e % 4] : hi[e % 4];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = w_reg[i][e];
    }
  };
  const uint64_t items = (a.rows + RPB - 1) / RPB;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t row = it * RPB + sub;
    const bool on = row < a.rows;
    const float rs = on ? a.rstd[row] : 0.0f, mu = on && LAYER && !KEPT ? a.mean[row] : 0.0f;
    NormIn<DT, KEPT> cur[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t g = i * TPR + t;
      cur[i] = load_normed<DT, KEPT, false>(a, row, g, on ? in_group(a.dim, g) : 0);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) trim_normed<DT, KEPT>(cur[i], a.dim, in_group(a.dim, i * TPR + t));
    float c1 = 0, c2 = 0;
    float d[8], n[8], w[8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t g = i * TPR + t;
      weights(i, w);
      normed8<DT, KEPT>(cur[i], on ? in_group(a.dim, g) : 0, mu, rs, d, n);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = d[e] * n[e];
        dw[i][e] += p;
        c2 = __builtin_fmaf(p, w[e], c2);
        if constexpr (LAYER) {
          db[i][e] += d[e];
          c1 = __builtin_fmaf(d[e], w[e], c1);
        }
      }
    }
    if (!a.dx.data) continue;  // uniform: every thread of the grid goes on
    row_sum2<TPR>(c1, c2, red, turn);
    c1 *= inv_dim;
    c2 *= inv_dim;
    if (!on) continue;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t g = i * TPR + t;
      const int k = in_group(a.dim, g);
      weights(i, w);
      normed8<DT, KEPT>(cur[i], k, mu, rs, d, n);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = rs * (d[e] * w[e] - c1 - n[e] * c2);
      store8<DT>(a.dx.data + (row * a.dx.stride + 8ull * g) * kEsz<DT>, d, k);
    }
  }
  if (!a.part) return;
  // the rows that the block took side by side, in order, then its part
  __shared__ float sums[RPB > 1 ? RPB : 1][RPB > 1 ? TPR * 8 : 1];
  const uint64_t out = reinterpret_cast<uint64_t>(a.part + blockIdx.x * static_cast<uint64_t>(a.dim));
  const uint64_t db_off = static_cast<uint64_t>(parts) * a.dim * 4;
  auto write = [&](float (&s)[8], uint32_t g, uint64_t to) {
    if constexpr (RPB > 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[sub][e * TPR + t] = s[e];
      __syncthreads();
      if (sub != 0) return;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (uint32_t q = 1; q < RPB; ++q) s[e] += sums[q][e * TPR + t];
    }
    store8<kF32>(to + 32ull * g, s, in_group(a.dim, g));
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    write(dw[i], i * TPR + t, out);
    if constexpr (LAYER) write(db[i], i * TPR + t, out + db_off);
  }
}

// Rows of any length, as above: a block's partial sums stay in its part of the
// workspace, each element with the thread that it belongs to.
template <int DT, bool LAYER, bool KEPT>
__global__ __launch_bounds__(kLongThreads) void norm_bwd_long_kernel(NormBwd a, uint32_t parts) {
  __shared__ float2 red[2][kLongThreads / 64];
  uint32_t turn = 0;
  const float inv_dim = 1.0f / static_cast<float>(a.dim);
  const uint32_t groups = (a.dim + 7) / 8;
  float* out = a.part ? a.part + blockIdx.x * static_cast<uint64_t>(a.dim) : nullptr;
  const uint64_t db_off = static_cast<uint64_t>(parts) * a.dim;
  bool first = true;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float rstd = a.rstd[row], mean = LAYER && !KEPT ? a.mean[row] : 0.0f;
    float c1 = 0, c2 = 0;
    float n[8], d[8], w[8];
    for (uint32_t g = threadIdx.x; g < groups; g += kLongThreads) {
      const int in = in_group(a.dim, g);
      normed8<DT, KEPT>(load_normed<DT, KEPT, true>(a, row, g, in), in, mean, rstd, d, n);
      load_params8(a.weight, a.param_dtype, g, in, 1.0f, w);
      if (out) {
        const uint64_t pw = reinterpret_cast<uint64_t>(out) + 32ull * g;
        const uint64_t pb = reinterpret_cast<uint64_t>(out + db_off) + 32ull * g;
        float s[8] = {}, r[8] = {};
        if (!first) {
          unpack8<kF32>(load8_raw<kF32>(pw, in), s);
          if constexpr (LAYER) unpack8<kF32>(load8_raw<kF32>(pb, in), r);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s[e] = __builtin_fmaf(d[e], n[e], s[e]);
          r[e] += d[e];
        }
        store8<kF32>(pw, s, in);
        if constexpr (LAYER) store8<kF32>(pb, r, in);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float gw = d[e] * w[e];
        if constexpr (LAYER) c1 += gw;
        c2 = __builtin_fmaf(gw, n[e], c2);
      }
    }
    first = false;
    if (!a.dx.data) continue;
    row_sum2<kLongThreads>(c1, c2, red, turn);
    c1 *= inv_dim;
    c2 *= inv_dim;
    for (uint32_t g = threadIdx.x; g < groups; g += kLongThreads) {
      const int in = in_group(a.dim, g);
      normed8<DT, KEPT>(load_normed<DT, KEPT, true>(a, row, g, in), in, mean, rstd, d, n);
      load_params8(a.weight, a.param_dtype, g, in, 1.0f, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = rstd * (d[e] * w[e] - c1 - n[e] * c2);
      store8<DT>(a.dx.data + (row * a.dx.stride + 8ull * g) * kEsz<DT>, d, in);
    }
  }
}

// Column sums of the parts: 32 columns a block, 32 slices of the parts, joined
// in order.  blockIdx.y: dw, db.
constexpr uint32_t kJoinCols = 32, kJoinSlices = 32;
__global__ __launch_bounds__(kJoinCols * kJoinSlices) void norm_join_kernel(NormBwd a, uint32_t parts) {
  __shared__ float sums[kJoinSlices][kJoinCols + 1];
  const uint32_t col = threadIdx.x % kJoinCols, slice = threadIdx.x / kJoinCols;
  const uint64_t dst = blockIdx.y ? a.dbias : a.dweight;
  if (!dst) return;
  const float* src = a.part + static_cast<uint64_t>(blockIdx.y) * parts * a.dim;
  for (uint64_t c0 = blockIdx.x * static_cast<uint64_t>(kJoinCols); c0 < a.dim; c0 += gridDim.x * static_cast<uint64_t>(kJoinCols)) {
    const uint64_t c = c0 + col;
    float s = 0;
    if (c < a.dim) {
#pragma unroll 16
      for (uint32_t p = slice; p < parts; p += kJoinSlices) s += src[p * static_cast<uint64_t>(a.dim) + c];
    }
    sums[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < a.dim) {
#pragma unroll
      for (uint32_t i = 1; i < kJoinSlices; ++i) s += sums[i][col];
      if (a.accumulate) s += load_param(dst, c, a.grad_dtype);
      store_param(dst, c, a.grad_dtype, s);
    }
    __syncthreads();
  }
}

// Threads a row and groups of eight a thread, the smallest shape that holds a
// row of `dim` elements; other rows take the kernels for any length.  Measured
// on 16384 x 4096 (bf16, RMS, rows kept; us forward with the rows read back /
// backward): 256 threads of 2 groups 99 / 65, 128 of 4 103 / 77, a wave of 8
// 124 / 103.
constexpr uint32_t kNormLongest = 16384;
constexpr bool norm_has_shape(uint64_t dim) { return dim >= 8 && dim <= kNormLongest; }
#define LC_NORM_SHAPES(F)          \
  if (dim <= 512) F(64, 1);        \
  else if (dim <= 1024) F(64, 2);  \
  else if (dim <= 2048) F(128, 2); \
  else if (dim <= 4096) F(256, 2); \
  else if (dim <= 6144) F(256, 3); \
  else if (dim <= 8192) F(512, 2); \
  else F(1024, 2)

// As many blocks as are resident at once, for more only add parts (16384 x
// 4096 layer norm in bf16, 12 waves a CU 69 us, 16 81; RMS norm, which holds no
// sums of db, 66 and 65).
NormParts norm_parts(uint64_t rows, uint64_t dim, bool light) {
  uint32_t tpr = kLongThreads, waves = 16;
  if (norm_has_shape(dim)) {
#define LC_NORM_SHAPE(TPR, NV) tpr = TPR, waves = NV == 1 ? 20 : NV == 2 ? (light ? 16 : 12) : light ? 12 : 8
    LC_NORM_SHAPES(LC_NORM_SHAPE);
#undef LC_NORM_SHAPE
  }
  NormParts p;
  p.rpb = tpr < 256 ? 256 / tpr : 1;
  const uint32_t block_waves = tpr < 256 ? 4 : tpr / 64;
  const uint64_t items = (rows + p.rpb - 1) / p.rpb;
  const auto blocks_of = [&](uint32_t w) -> uint64_t { return 256 * (w > block_waves ? w / block_waves : 1); };
  // up to four rows a block the parts weigh more (1024 x 4096 RMS norm in bf16, 16
  // waves a CU 18.0 us of kernels, 8 14.6)
  const uint64_t most = blocks_of(waves > 8 && items <= 4 * blocks_of(8) ? 8 : waves);
  const uint64_t turns = (items + most - 1) / most;
  // few turns are dealt out evenly: 1025 over 768 blocks as two each for 513
  uint64_t blocks = turns > 3 ? most : turns ? (items + turns - 1) / turns : 0;
  if (LC_MAX_GRID_BLOCKS > 0 && blocks > LC_MAX_GRID_BLOCKS) blocks = LC_MAX_GRID_BLOCKS;
  p.parts = static_cast<uint32_t>(blocks);
  return p;
}

template <int DT, bool LAYER, int TPR, int NV>
hipError_t norm_fwd_shape(const NormFwd& a, hipStream_t st) {
  constexpr uint32_t threads = kNormThreads<TPR>, rpb = threads / TPR;
  return launch_op(norm_fwd_kernel<DT, LAYER, TPR, NV>, grid_for((a.rows + rpb - 1) / rpb, threads), threads, st, a);
}

template <int DT, bool LAYER>
hipError_t norm_fwd_of(const NormFwd& a, hipStream_t st) {
  const uint32_t dim = a.dim;
  if (!norm_has_shape(dim))
    return launch_op(norm_fwd_long_kernel<DT, LAYER>, grid_for(a.rows, kLongThreads), kLongThreads, st, a);
#define LC_NORM_SHAPE(TPR, NV) return norm_fwd_shape<DT, LAYER, TPR, NV>(a, st)
  LC_NORM_SHAPES(LC_NORM_SHAPE);
#undef LC_NORM_SHAPE
}

template <int DT, bool LAYER, bool KEPT>
hipError_t norm_bwd_of(const NormBwd& a, const NormParts& p, hipStream_t st) {
  const uint32_t dim = a.dim;
  if (!norm_has_shape(dim))
    return launch_op(norm_bwd_long_kernel<DT, LAYER, KEPT>, p.parts, kLongThreads, st, a, p.parts);
#define LC_NORM_SHAPE(TPR, NV) \
  return launch_op(norm_bwd_kernel<DT, LAYER, KEPT, TPR, NV>, p.parts, kNormThreads<TPR>, st, a, p.parts)
  LC_NORM_SHAPES(LC_NORM_SHAPE);
#undef LC_NORM_SHAPE
}

template <int DT>
hipError_t norm_bwd_kind(const NormBwd& a, const NormParts& p, hipStream_t st) {
  const bool kept = a.kept.codes != 0;
  if (a.layer) return kept ? norm_bwd_of<DT, true, true>(a, p, st) : norm_bwd_of<DT, true, false>(a, p, st);
  return kept ? norm_bwd_of<DT, false, true>(a, p, st) : norm_bwd_of<DT, false, false>(a, p, st);
}

}  // namespace

hipError_t launch_norm_fwd(const NormFwd& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  if (a.dtype == kBf16) return a.layer ? norm_fwd_of<kBf16, true>(a, st) : norm_fwd_of<kBf16, false>(a, st);
  return a.layer ? norm_fwd_of<kF32, true>(a, st) : norm_fwd_of<kF32, false>(a, st);
}

uint64_t norm_bwd_workspace(uint64_t rows, uint64_t dim) {
  // whether a call is light goes by its kind and types
  const uint64_t a = norm_parts(rows, dim, true).parts, b = norm_parts(rows, dim, false).parts;
  return (a > b ? a : b) * 2 * dim * 4;
}

hipError_t launch_norm_bwd(const NormBwd& a, hipStream_t st) {
  const NormParts p = norm_parts(a.rows, a.dim, !a.layer && a.dtype == kBf16);
  if (a.rows > 0 && (a.part || a.dx.data)) {
    const hipError_t e = a.dtype == kBf16 ? norm_bwd_kind<kBf16>(a, p, st) : norm_bwd_kind<kF32>(a, p, st);
    if (e != hipSuccess) return e;
  }
  if (!a.dweight && !a.dbias) return hipSuccess;
  return launch_op(norm_join_kernel,
                   dim3(grid_for((a.dim + kJoinCols - 1) / kJoinCols, kJoinCols * kJoinSlices), a.dbias ? 2 : 1),
                   kJoinCols * kJoinSlices, st, a, p.parts);
}

}  // namespace lc
