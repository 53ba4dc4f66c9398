// A linear layer's weight gradient from its output's gradient dY [tokens][n]
// and its input X [tokens][k] kept in 8 bits:
//
//   dW[n][k] (+)= sum over t of dY[t][n] * (X[t][k] * scale[k] + shift[k])
//             =  scale[k] * (dY^T X)[n][k] + shift[k] * s[n],   s[n] = sum over t of dY[t][n]
//   dbias[n] (+)= s[n]
//
// so the columns' scale and shift cost the main loop nothing.  Bound by the
// matrix cores: 2 n k flops a token.  A kept element is 4 significant bits
// times a power of two, so it is exact in bf16; a bf16 dY enters as it is, an
// fp32 dY as the sum of three bf16 parts (8 of its 24 bits each), which keeps
// every product exact.  Sums are fp32.
//
// Both operands lie with the tokens, over which the product sums, as rows: a
// tile goes to LDS as it lies and the transposing LDS reads give each lane the
// eight tokens of its column that the matrix instruction takes.
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

// Four bytes to four bf16, times 2^(code - 127); exact, and code 255 gives NaN.
__device__ __forceinline__ u32x2 decode4(uint32_t b, float scale) {
  const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
  const auto hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// An fp32 value as three bf16 parts of 8 bits each, whose sum it is.
__device__ __forceinline__ void split3(float v, uint32_t (&part)[3]) {
  const uint32_t u = __float_as_uint(v);
  if ((u & 0x7fffffffu) >= 0x7f800000u) {  // not finite: the first part says so alone
    part[0] = (u & 0x007fffffu ? 0x7FC0u : u >> 16);
    part[1] = part[2] = 0;
    return;
  }
  part[0] = u >> 16;
  const float r1 = v - __uint_as_float(u & 0xffff0000u);
  part[1] = __float_as_uint(r1) >> 16;
  const float r2 = r1 - __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
  part[2] = __float_as_uint(r2) >> 16;
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

struct WgradTiles {
  uint32_t tn, tk;       // tiles of n and k
  uint32_t splits;       // parts of the tokens
  uint64_t per_split;    // tokens a part, a multiple of kStep
  float* part;           // [splits][n][k], with more than one split
  float* sums;           // [splits][n]
};

template <int DT, bool SUMS>
__global__ __launch_bounds__(kThreads) void wgrad_kernel(Wgrad a, WgradTiles s) {
  constexpr int P = kPlanes<DT>;
  __shared__ __align__(16) uint16_t dys[2][P][kStep * kPitch];
  __shared__ __align__(16) uint16_t xs[2][kStep * kPitch];
  __shared__ float colsum[SUMS ? kThreads / 16 : 1][kTile];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint64_t tiles = static_cast<uint64_t>(s.tn) * s.tk * s.splits;
  for (uint64_t b = blockIdx.x; b < tiles; b += gridDim.x) {
    const uint32_t split = static_cast<uint32_t>(b % s.splits);
    const uint64_t tile = b / s.splits;
    const uint32_t n0 = static_cast<uint32_t>(tile / s.tk) * kTile, k0 = static_cast<uint32_t>(tile % s.tk) * kTile;
    const uint64_t t_begin = split * s.per_split;
    const uint64_t t_end = t_begin + s.per_split < a.rows ? t_begin + s.per_split : a.rows;

    // a thread's share of a step: two groups of eight of dY, sixteen codes of X
    const uint32_t dc = tid % 16, dr = tid / 16;
    const int d_in = static_cast<int>(a.n) - static_cast<int>(n0 + 8 * dc);
    const uint32_t xc = tid % 8, xr = tid / 8;
    const int x_in = static_cast<int>(a.k) - static_cast<int>(k0 + 16 * xc);
    Raw8<DT> d[2];
    Codes16 c;
    float sum[8] = {};
    auto load = [&](uint64_t t) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint64_t r = t + dr + 16 * i;
        d[i] = load8_raw<DT>(a.dy.data + (r * a.dy.stride + n0 + 8 * dc) * kEsz<DT>, r < t_end ? d_in : 0);
      }
      const uint64_t r = t + xr;
      c = load_codes16(a.x, r, k0 + 16 * xc, r < t_end ? x_in : 0);
    };
    auto store = [&](int buf) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t at = (dr + 16 * i) * kPitch + 8 * dc;
        if constexpr (SUMS) {
          float f[8];
          unpack8<DT>(d[i], f);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] += f[e];
        }
        if constexpr (P == 1) {
          *reinterpret_cast<u32x4*>(&dys[buf][0][at]) = d[i].v[0];
        } else {
          float f[8];
          unpack8<DT>(d[i], f);
          u32x4 q[3];
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            uint32_t lo[3], hi[3];
            split3(f[e], lo);
            split3(f[e + 1], hi);
#pragma unroll
            for (int p = 0; p < 3; ++p) q[p][e / 2] = lo[p] | hi[p] << 16;
          }
#pragma unroll
          for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4*>(&dys[buf][p][at]) = q[p];
        }
      }
      const float scale = __uint_as_float(c.code << 23);
      const u32x2 q0 = decode4(c.codes[0], scale), q1 = decode4(c.codes[1], scale);
      const u32x2 q2 = decode4(c.codes[2], scale), q3 = decode4(c.codes[3], scale);
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
    if (t_begin < t_end) {
      load(t_begin);
      store(0);
    }
    __syncthreads();
    int buf = 0;
    for (uint64_t t = t_begin; t < t_end; t += kStep) {
      const bool more = t + kStep < t_end;
      if (more) load(t + kStep);
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
      if (more) store(buf ^ 1);
      __syncthreads();
      buf ^= 1;
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
          if (s.splits > 1) {
            s.sums[split * static_cast<uint64_t>(a.n) + n] = v;
          } else if (a.dbias) {
            store_param(a.dbias, n, a.dw_dtype, v + (a.accumulate ? load_param(a.dbias, n, a.dw_dtype) : 0.0f));
          }
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t ln = wn + 16 * j + lane % 16;
      const uint64_t n = n0 + ln;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint64_t k = k0 + wk + 16 * i + lane / 16 * 4 + e;
          if (n >= a.n || k >= a.k) continue;
          float v = acc[i][j][e];
          if (s.splits > 1) {
            s.part[(split * static_cast<uint64_t>(a.n) + n) * a.k + k] = v;
            continue;
          }
          if (a.col_scale) v *= load_param(a.col_scale, k, a.param_dtype);
          if (SUMS && a.col_shift) v += colsum[0][ln] * load_param(a.col_shift, k, a.param_dtype);
          const uint64_t at = n * a.dw.stride + k;
          if (a.accumulate) v += load_param(a.dw.data, at, a.dw_dtype);
          store_param(a.dw.data, at, a.dw_dtype, v);
        }
      }
    }
    __syncthreads();
  }
}

// The splits' sums, in order, with the columns' scale and shift.
__global__ __launch_bounds__(kThreads) void wgrad_join_kernel(Wgrad a, WgradTiles s, int with_sums) {
  const uint64_t per_row = (a.k + kThreads - 1) / kThreads, items = per_row * a.n;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t n = it / per_row, k = it % per_row * kThreads + threadIdx.x;
    float sum = 0;
    if (with_sums)
      for (uint32_t p = 0; p < s.splits; ++p) sum += s.sums[p * static_cast<uint64_t>(a.n) + n];
    if (k == 0 && a.dbias)
      store_param(a.dbias, n, a.dw_dtype, sum + (a.accumulate ? load_param(a.dbias, n, a.dw_dtype) : 0.0f));
    if (k >= a.k) continue;
    float v = 0;
    for (uint32_t p = 0; p < s.splits; ++p) v += s.part[(p * static_cast<uint64_t>(a.n) + n) * a.k + k];
    if (a.col_scale) v *= load_param(a.col_scale, k, a.param_dtype);
    if (a.col_shift) v += sum * load_param(a.col_shift, k, a.param_dtype);
    const uint64_t at = n * a.dw.stride + k;
    if (a.accumulate) v += load_param(a.dw.data, at, a.dw_dtype);
    store_param(a.dw.data, at, a.dw_dtype, v);
  }
}

// Splits of the tokens: as many as fill the chip with tiles, of 128 tokens at least.
WgradTiles wgrad_tiles(uint64_t rows, uint64_t n, uint64_t k) {
  WgradTiles s{};
  s.tn = static_cast<uint32_t>((n + kTile - 1) / kTile);
  s.tk = static_cast<uint32_t>((k + kTile - 1) / kTile);
  const uint64_t tiles = static_cast<uint64_t>(s.tn) * s.tk;
  uint64_t splits = tiles >= 256 ? 1 : 512 / tiles;
  const uint64_t most = rows / 128;
  if (splits > most) splits = most;
  if (splits > 64) splits = 64;
  if (splits < 1) splits = 1;
  s.per_split = ((rows + splits - 1) / splits + kStep - 1) / kStep * kStep;
  if (s.per_split == 0) s.per_split = kStep;
  s.splits = rows ? static_cast<uint32_t>((rows + s.per_split - 1) / s.per_split) : 1;
  return s;
}

template <int DT>
void wgrad_of(const Wgrad& a, const WgradTiles& s, bool sums, hipStream_t st) {
  const uint32_t grid = grid_for(static_cast<uint64_t>(s.tn) * s.tk * s.splits, kThreads);
  if (sums) hipLaunchKernelGGL((wgrad_kernel<DT, true>), dim3(grid), dim3(kThreads), 0, st, a, s);
  else hipLaunchKernelGGL((wgrad_kernel<DT, false>), dim3(grid), dim3(kThreads), 0, st, a, s);
}

}  // namespace

uint64_t wgrad_workspace(uint64_t rows, uint64_t n, uint64_t k) {
  const WgradTiles s = wgrad_tiles(rows, n, k);
  return s.splits > 1 ? s.splits * (n * k + n) * 4 : 0;
}

hipError_t launch_wgrad(const Wgrad& a, hipStream_t st) {
  WgradTiles s = wgrad_tiles(a.rows, a.n, a.k);
  s.part = reinterpret_cast<float*>(a.ws);
  s.sums = s.part + s.splits * static_cast<uint64_t>(a.n) * a.k;
  const bool sums = a.dbias || a.col_shift;
  if (a.dtype == kBf16) wgrad_of<kBf16>(a, s, sums, st);
  else wgrad_of<kF32>(a, s, sums, st);
  if (s.splits > 1) {
    const uint64_t items = (a.k + kThreads - 1) / kThreads * static_cast<uint64_t>(a.n);
    hipLaunchKernelGGL(wgrad_join_kernel, dim3(grid_for(items, kThreads)), dim3(kThreads), 0, st, a, s, sums ? 1 : 0);
  }
  return hipGetLastError();
}

}  // namespace lc
