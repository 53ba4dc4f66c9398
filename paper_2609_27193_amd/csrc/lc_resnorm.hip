// Layer norm and RMS norm with the residual's addition, forward and backward.
//
//   h = x + r,  n = (h - mean) * rstd,  y = n * w + b
//   g = dy * w;  dx = dr = dh + rstd * (g - mean(g) - n * mean(g * n))     (RMS: without mean(g))
//   dw = sum over rows of dy * n;  db = sum over rows of dy
//
// Bound by memory: both addends are read once, their fp32 sum stays in registers,
// is written in the residual's type and normalised as it is, before that rounding.
// y goes out as it is, in 8 bits, or both: a layer that takes its input in 8 bits
// needs no other copy (33/32 bytes an element for two).  The residual x and its
// gradient would otherwise cross memory a second time between a sum and a norm of
// their own.  Rows, sums and parts are those of the norm alone.
#include "lc_norm_device.h"

namespace lc {
namespace {

// Group g of both addends, fp32 sums; zeros behind the row's end.
template <int DT, int RT>
struct Addends {
  Raw8<DT> x;
  Raw8<RT> r;
};
template <int DT, int RT>
__device__ __forceinline__ void add8(const Addends<DT, RT>& in, float (&f)[8]) {
  float r[8];
  unpack8<DT>(in.x, f);
  unpack8<RT>(in.r, r);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] += r[e];
}
// n of the group out of h, and what the call wants of it.  f: h, overwritten.
template <int DT, bool LAYER, bool NT>
__device__ __forceinline__ void write_normed8(const ResNormFwd& a, uint64_t row, uint32_t g, int n, float mean, float rstd,
                                              float (&f)[8]) {
  float w[8], b[8], y[8];
  load_params8(a.weight, a.param_dtype, g, n, 1.0f, w);
  if constexpr (LAYER) load_params8(a.bias, a.param_dtype, g, n, 0.0f, b);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    f[e] = (LAYER ? f[e] - mean : f[e]) * rstd;
    y[e] = f[e] * w[e];
    if constexpr (LAYER) y[e] += b[e];
  }
  if (a.y.data) store8<DT, NT>(a.y.data + (row * a.y.stride + 8ull * g) * kEsz<DT>, y, n);
  if (n < 8) {  // what is no element must not set its block's power
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[e] = e < n ? f[e] : 0.0f;
      y[e] = e < n ? y[e] : 0.0f;
    }
  }
  uint32_t code;
  if (a.y8.codes) {
    const u32x2 q = act_encode8(y, code);
    store_kept8(a.y8, row, g, n, q, code);
  }
  if (a.kept.codes) {
    const u32x2 q = act_encode8(f, code);
    store_kept8(a.kept, row, g, n, q, code);
  }
}

template <int DT, int RT, bool LAYER, int TPR, int NV>
__global__ __launch_bounds__(kNormThreads<TPR>) void res_norm_fwd_kernel(ResNormFwd a) {
  constexpr uint32_t RPB = kNormThreads<TPR> / TPR;
  __shared__ float2 red[2][kNormThreads<TPR> / 64];
  uint32_t turn = 0;
  const uint32_t t = threadIdx.x % TPR;
  const float inv_dim = 1.0f / static_cast<float>(a.dim);
  const uint64_t items = (a.rows + RPB - 1) / RPB;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t row = row_item(it, items) * RPB + threadIdx.x / TPR;
    const bool on = row < a.rows;  // the others only take part in the barriers
    Addends<DT, RT> in[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t g = i * TPR + t;
      const int n = on ? in_group(a.dim, g) : 0;
      in[i].x = load8_row<DT, kStreams<DT>>(a.x.data + row * a.x.stride * kEsz<DT>, g, n);
      in[i].r = load8_row<RT, kStreams<RT>>(a.res.data + row * a.res.stride * kEsz<RT>, g, n);
    }
    float f[NV][8];
    float sum = 0, unused = 0, mean = 0, sq = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int n = in_group(a.dim, i * TPR + t);
      trim8_row<DT>(in[i].x, a.dim, n);
      trim8_row<RT>(in[i].r, a.dim, n);
      add8(in[i], f[i]);
      if (on && a.h.data)
        store8<RT, kStreams<RT>>(a.h.data + (row * a.h.stride + 8ull * (i * TPR + t)) * kEsz<RT>, f[i], n);
      if constexpr (LAYER) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += f[i][e];
      }
    }
    if constexpr (LAYER) mean = row_sum<TPR>(sum, red, turn) * inv_dim;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int n = in_group(a.dim, i * TPR + t);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = !LAYER ? f[i][e] : e < n ? f[i][e] - mean : 0.0f;
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
      write_normed8<DT, LAYER, kStreams<DT>>(a, row, g, in_group(a.dim, g), mean, rstd, f[i]);
    }
  }
}

// Rows of any length (fewer than 8 columns, or beyond kNormLongest): both addends
// are read again for each of the steps.  4096 x 20000 in bf16 137 us, layer norm 160 (96 at
// the copy's rate); 65536 x 7 520 us, for a block takes each row.
template <int DT, int RT, bool LAYER>
__global__ __launch_bounds__(kLongThreads) void res_norm_fwd_long_kernel(ResNormFwd a) {
  __shared__ float2 red[2][kLongThreads / 64];
  uint32_t turn = 0;
  const float inv_dim = 1.0f / static_cast<float>(a.dim);
  const uint32_t groups = (a.dim + 31) / 32 * 4;  // whole quads, so that a block's four lanes stay together
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float f[8];
    const auto load = [&](uint32_t g, int n) {
      Addends<DT, RT> in;
      in.x = load8_raw<DT>(a.x.data + (row * a.x.stride + 8ull * g) * kEsz<DT>, n);
      in.r = load8_raw<RT>(a.res.data + (row * a.res.stride + 8ull * g) * kEsz<RT>, n);
      add8(in, f);
    };
    float sum = 0, unused = 0, mean = 0, sq = 0;
    if constexpr (LAYER) {
      for (uint32_t g = threadIdx.x; g < groups; g += kLongThreads) {
        load(g, in_group(a.dim, g));
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += f[e];
      }
      mean = row_sum<kLongThreads>(sum, red, turn) * inv_dim;
    }
    for (uint32_t g = threadIdx.x; g < groups; g += kLongThreads) {
      const int n = in_group(a.dim, g);
      load(g, n);
      if (a.h.data) store8<RT>(a.h.data + (row * a.h.stride + 8ull * g) * kEsz<RT>, f, n);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = e < n ? f[e] - mean : 0.0f;
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
      load(g, n);
      write_normed8<DT, LAYER, false>(a, row, g, n, mean, rstd, f);
    }
  }
}

// ---- backward ------------------------------------------------------------------------
// What a thread has of group g of a row: dy, dh and h, or the normalised row's codes.
template <int DT, int RT, bool KEPT>
struct ResNormIn {
  Raw8<DT> dy;
  Raw8<RT> dh;
  Raw8<RT> h;
};
template <int DT, int RT>
struct ResNormIn<DT, RT, true> {
  Raw8<DT> dy;
  Raw8<RT> dh;
  u32x2 codes;
  uint32_t code;
};
// ANY: rows of any length, else of eight elements at least.
template <int DT, int RT, bool KEPT, bool ANY>
__device__ __forceinline__ ResNormIn<DT, RT, KEPT> load_res(const ResNormBwd& a, uint64_t row, uint32_t g, int n) {
  ResNormIn<DT, RT, KEPT> in;
  const uint64_t dy = a.dy.data + row * a.dy.stride * kEsz<DT>, dh = a.dh.data + row * a.dh.stride * kEsz<RT>;
  in.dy = ANY ? load8_raw<DT>(dy + 8ull * g * kEsz<DT>, n) : load8_row<DT, kStreams<DT>>(dy, g, n);
  if constexpr (KEPT) {
    in.code = n > 0 ? load_kept_code(a.kept, row, g) : 0;
    in.codes = ANY ? load_kept8(a.kept, row, g, n) : load_codes8_row(a.kept.codes + row * a.kept.code_stride, g, n);
  } else {
    const uint64_t h = a.x.data + row * a.x.stride * kEsz<RT>;
    in.h = ANY ? load8_raw<RT>(h + 8ull * g * kEsz<RT>, n) : load8_row<RT, kStreams<RT>>(h, g, n);
  }
  in.dh = ANY ? load8_raw<RT>(dh + 8ull * g * kEsz<RT>, n) : load8_row<RT, kStreams<RT>>(dh, g, n);
  return in;
}
template <int DT, int RT, bool KEPT>
__device__ __forceinline__ void trim_res(ResNormIn<DT, RT, KEPT>& in, uint32_t dim, int n) {
  trim8_row<DT>(in.dy, dim, n);
  trim8_row<RT>(in.dh, dim, n);
  if constexpr (KEPT) in.codes = trim_codes8_row(in.codes, n);
  else trim8_row<RT>(in.h, dim, n);
}
// dy and n of the group; zeros behind the row's end.
template <int DT, int RT, bool KEPT>
__device__ __forceinline__ void normed8(const ResNormIn<DT, RT, KEPT>& in, int n, float mean, float rstd, float (&d)[8],
                                        float (&f)[8]) {
  unpack8<DT>(in.dy, d);
  if constexpr (KEPT) {
    act_decode8(in.codes, act_scale(in.code), f);
  } else {
    unpack8<RT>(in.h, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (f[e] - mean) * rstd;
    if (n < 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = e < n ? f[e] : 0.0f;
    }
  }
}
// dx of the group, in the types that the call wants.
template <int DT, int RT>
__device__ __forceinline__ void write_dx8(const ResNormBwd& a, uint64_t row, uint32_t g, int k, const float (&d)[8]) {
  if (a.dx.data) store8<DT>(a.dx.data + (row * a.dx.stride + 8ull * g) * kEsz<DT>, d, k);
  if (a.dres.data) store8<RT>(a.dres.data + (row * a.dres.stride + 8ull * g) * kEsz<RT>, d, k);
}

// A block keeps its columns' weights and sums in registers and takes its turn at
// the rows, as the norm's gradient does.
template <int DT, int RT, bool LAYER, bool KEPT, int TPR, int NV>
__global__ __launch_bounds__(kNormThreads<TPR>) void res_norm_bwd_kernel(ResNormBwd a, uint32_t parts) {
  constexpr uint32_t RPB = kNormThreads<TPR> / TPR;
  __shared__ float2 red[2][kNormThreads<TPR> / 64];
  uint32_t turn = 0;
  const uint32_t t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const float inv_dim = 1.0f / static_cast<float>(a.dim);
  // in LDS where registers for them would spill (128 a thread of 1024)
  constexpr bool kWeightsInLds = TPR == 1024;
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
  const bool wants_dx = a.dx.data || a.dres.data;
  const uint64_t items = (a.rows + RPB - 1) / RPB;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t row = it * RPB + sub;
    const bool on = row < a.rows;
    const float rs = on ? a.rstd[row] : 0.0f, mu = on && LAYER && !KEPT ? a.mean[row] : 0.0f;
    ResNormIn<DT, RT, KEPT> cur[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t g = i * TPR + t;
      cur[i] = load_res<DT, RT, KEPT, false>(a, row, g, on ? in_group(a.dim, g) : 0);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) trim_res<DT, RT, KEPT>(cur[i], a.dim, in_group(a.dim, i * TPR + t));
    float c1 = 0, c2 = 0;
    float d[8], n[8], w[8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t g = i * TPR + t;
      weights(i, w);
      normed8<DT, RT, KEPT>(cur[i], on ? in_group(a.dim, g) : 0, mu, rs, d, n);
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
    if (!wants_dx) continue;  // uniform: every thread of the grid goes on
    row_sum2<TPR>(c1, c2, red, turn);
    c1 *= inv_dim;
    c2 *= inv_dim;
    if (!on) continue;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t g = i * TPR + t;
      const int k = in_group(a.dim, g);
      float skip[8];
      weights(i, w);
      normed8<DT, RT, KEPT>(cur[i], k, mu, rs, d, n);
      unpack8<RT>(cur[i].dh, skip);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = __builtin_fmaf(rs, d[e] * w[e] - c1 - n[e] * c2, skip[e]);
      write_dx8<DT, RT>(a, row, g, k, d);
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
// workspace, each element with the thread that it belongs to.  4096 x 20000 in bf16 254 us,
// layer norm 348 (96 at the copy's rate); 65536 x 7 873 us.
template <int DT, int RT, bool LAYER, bool KEPT>
__global__ __launch_bounds__(kLongThreads) void res_norm_bwd_long_kernel(ResNormBwd a, uint32_t parts) {
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
      normed8<DT, RT, KEPT>(load_res<DT, RT, KEPT, true>(a, row, g, in), in, mean, rstd, d, n);
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
    if (!a.dx.data && !a.dres.data) continue;
    row_sum2<kLongThreads>(c1, c2, red, turn);
    c1 *= inv_dim;
    c2 *= inv_dim;
    for (uint32_t g = threadIdx.x; g < groups; g += kLongThreads) {
      const int in = in_group(a.dim, g);
      const auto cur = load_res<DT, RT, KEPT, true>(a, row, g, in);
      float skip[8];
      normed8<DT, RT, KEPT>(cur, in, mean, rstd, d, n);
      unpack8<RT>(cur.dh, skip);
      load_params8(a.weight, a.param_dtype, g, in, 1.0f, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = __builtin_fmaf(rstd, d[e] * w[e] - c1 - n[e] * c2, skip[e]);
      write_dx8<DT, RT>(a, row, g, in, d);
    }
  }
}

template <int DT, int RT, bool LAYER, int TPR, int NV>
hipError_t res_norm_fwd_shape(const ResNormFwd& a, hipStream_t st) {
  constexpr uint32_t threads = kNormThreads<TPR>, rpb = threads / TPR;
  return launch_op(res_norm_fwd_kernel<DT, RT, LAYER, TPR, NV>, grid_for((a.rows + rpb - 1) / rpb, threads), threads, st, a);
}
template <int DT, int RT, bool LAYER>
hipError_t res_norm_fwd_of(const ResNormFwd& a, hipStream_t st) {
  const uint32_t dim = a.dim;
  if (!norm_has_shape(dim))
    return launch_op(res_norm_fwd_long_kernel<DT, RT, LAYER>, grid_for(a.rows, kLongThreads), kLongThreads, st, a);
#define LC_NORM_SHAPE(TPR, NV) return res_norm_fwd_shape<DT, RT, LAYER, TPR, NV>(a, st)
  LC_NORM_SHAPES(LC_NORM_SHAPE);
#undef LC_NORM_SHAPE
}
template <int DT, int RT>
hipError_t res_norm_fwd_kind(const ResNormFwd& a, hipStream_t st) {
  return a.layer ? res_norm_fwd_of<DT, RT, true>(a, st) : res_norm_fwd_of<DT, RT, false>(a, st);
}

// Waves a CU, by the groups of eight that a thread has: three or four streams in and
// one or two out are enough of two blocks (us at 8 / 12 / 16 waves: 16384 x 4096 in
// bf16 91 / 94 / 95, 8192 x 5120 with an fp32 stream from kept rows 101 / 115).  The
// next row's loads in registers meanwhile: 92 and 103.
constexpr NormWaves kResWaves = {16, 8, 8};  // fewer than the workspace reckons with

template <int DT, int RT, bool LAYER, bool KEPT>
hipError_t res_norm_bwd_of(const ResNormBwd& a, const NormParts& p, hipStream_t st) {
  const uint32_t dim = a.dim;
  if (!norm_has_shape(dim))
    return launch_op(res_norm_bwd_long_kernel<DT, RT, LAYER, KEPT>, p.parts, kLongThreads, st, a, p.parts);
#define LC_NORM_SHAPE(TPR, NV) \
  return launch_op(res_norm_bwd_kernel<DT, RT, LAYER, KEPT, TPR, NV>, p.parts, kNormThreads<TPR>, st, a, p.parts)
  LC_NORM_SHAPES(LC_NORM_SHAPE);
#undef LC_NORM_SHAPE
}
template <int DT, int RT>
hipError_t res_norm_bwd_kind(const ResNormBwd& a, const NormParts& p, hipStream_t st) {
  const bool kept = a.kept.codes != 0;
  if (a.layer) return kept ? res_norm_bwd_of<DT, RT, true, true>(a, p, st) : res_norm_bwd_of<DT, RT, true, false>(a, p, st);
  return kept ? res_norm_bwd_of<DT, RT, false, true>(a, p, st) : res_norm_bwd_of<DT, RT, false, false>(a, p, st);
}

}  // namespace

hipError_t launch_res_norm_fwd(const ResNormFwd& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  if (a.dtype == kF32) return res_norm_fwd_kind<kF32, kF32>(a, st);
  return a.res_dtype == kBf16 ? res_norm_fwd_kind<kBf16, kBf16>(a, st) : res_norm_fwd_kind<kBf16, kF32>(a, st);
}

hipError_t launch_res_norm_bwd(const ResNormBwd& a, hipStream_t st) {
  const NormParts p = norm_parts(a.rows, a.dim, kResWaves);
  if (a.rows > 0 && (a.part || a.dx.data || a.dres.data)) {
    const hipError_t e = a.dtype == kF32         ? res_norm_bwd_kind<kF32, kF32>(a, p, st)
                         : a.res_dtype == kBf16 ? res_norm_bwd_kind<kBf16, kBf16>(a, p, st)
                                                : res_norm_bwd_kind<kBf16, kF32>(a, p, st);
    if (e != hipSuccess) return e;
  }
  if (!a.dweight && !a.dbias) return hipSuccess;
  return norm_join(a, p.parts, st);
}

}  // namespace lc
