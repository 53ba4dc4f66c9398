// What the norms' kernels share (lc_norm.hip: the norm alone; lc_resnorm.hip: with
// the residual's addition): sums over the threads of a row, the threads that a
// row takes, and the sums over rows in parts that are joined in a fixed order.
#pragma once

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

constexpr uint32_t kLongThreads = 1024;  // of the kernels for rows of any length

// Partial sums of dw and db: `parts` rows of dim each, dw's first.
struct NormParts {
  uint32_t rpb;    // rows that a block takes at once
  uint32_t parts;
};

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
__host__ inline hipError_t norm_join(const NormBwd& a, uint32_t parts, hipStream_t st) {
  return launch_op(norm_join_kernel,
                   dim3(grid_for((a.dim + kJoinCols - 1) / kJoinCols, kJoinCols * kJoinSlices), a.dbias ? 2 : 1),
                   kJoinCols * kJoinSlices, st, a, parts);
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

// As many blocks as are resident at once, for more only add parts: waves a CU by the
// groups of eight that a thread has.
struct NormWaves {
  uint32_t of1, of2, of3;
};
// (16384 x 4096 layer norm in bf16, 12 waves a CU 69 us, 16 81; RMS norm, which holds
// no sums of db, 66 and 65.)
constexpr NormWaves kNormLight = {20, 16, 12}, kNormHeavy = {20, 12, 8};
__host__ inline NormParts norm_parts(uint64_t rows, uint64_t dim, const NormWaves& w) {
  uint32_t tpr = kLongThreads, waves = 16;
  if (norm_has_shape(dim)) {
#define LC_NORM_SHAPE(TPR, NV) tpr = TPR, waves = NV == 1 ? w.of1 : NV == 2 ? w.of2 : w.of3
    LC_NORM_SHAPES(LC_NORM_SHAPE);
#undef LC_NORM_SHAPE
  }
  NormParts p;
  p.rpb = tpr < 256 ? 256 / tpr : 1;
  const uint32_t block_waves = tpr < 256 ? 4 : tpr / 64;
  const uint64_t items = (rows + p.rpb - 1) / p.rpb;
  const auto blocks_of = [&](uint32_t n) -> uint64_t { return 256 * (n > block_waves ? n / block_waves : 1); };
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

}  // namespace
}  // namespace lc
