// Activations kept in 8 bits: written and read back.  Both are bound by memory;
// a row's groups of eight elements go to consecutive lanes, so that the four
// groups of a 32-element block lie in one quad of lanes, which finds the
// block's power of two without shared memory.
#include "lc_ops_device.h"

namespace lc {
namespace {

constexpr uint32_t kActThreads = 256;
// Groups that a thread has in flight (saved and read back, us, of one, two, four
// and eight): 8192 x 14336 bf16 126, 124, 119, 114; 8192 x 8192 fp32 100, 96, 91,
// 91; 65536 x 1024 bf16 73, 70, 76, 119.  Two: up to 2048
// columns a thread has one, and the places held for more cost waves.
constexpr int kActVecs = 2;

// `lanes` threads (a power of two, 4 at least) take a row.
template <int DT>
__global__ __launch_bounds__(kActThreads) void act_save_kernel(ActCopy a, uint32_t lanes_log2) {
  const uint32_t lanes = 1u << lanes_log2, per_block = kActThreads >> lanes_log2;
  const uint32_t groups = (a.dim + 31) / 32 * 4, lane = threadIdx.x & (lanes - 1);
  const uint64_t items = (a.rows + per_block - 1) / per_block;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t row = row_item(it, items) * per_block + (threadIdx.x >> lanes_log2);
    if (row >= a.rows) continue;
    for (uint32_t g0 = lane; g0 < groups; g0 += lanes * kActVecs) {
      Raw8<DT> r[kActVecs];
#pragma unroll
      for (int i = 0; i < kActVecs; ++i) {
        const uint32_t g = g0 + i * lanes;
        r[i] = load8_raw<DT, true>(a.x.data + (row * a.x.stride + 8ull * g) * kEsz<DT>, g < groups ? in_group(a.dim, g) : 0);
      }
#pragma unroll
      for (int i = 0; i < kActVecs; ++i) {
        const uint32_t g = g0 + i * lanes;
        if (g >= groups) break;  // whole quads
        float f[8];
        unpack8<DT>(r[i], f);
        uint32_t code;
        const u32x2 q = act_encode8(f, code);
        store_kept8(a.kept, row, g, in_group(a.dim, g), q, code);
      }
    }
  }
}

template <int DT>
__global__ __launch_bounds__(kActThreads) void act_load_kernel(ActCopy a, uint32_t lanes_log2) {
  const uint32_t lanes = 1u << lanes_log2, per_block = kActThreads >> lanes_log2;
  const uint32_t groups = (a.dim + 7) / 8, lane = threadIdx.x & (lanes - 1);
  const uint64_t items = (a.rows + per_block - 1) / per_block;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t row = row_item(it, items) * per_block + (threadIdx.x >> lanes_log2);
    if (row >= a.rows) continue;
    for (uint32_t g0 = lane; g0 < groups; g0 += lanes * kActVecs) {
      u32x2 b[kActVecs];
      uint32_t code[kActVecs];
#pragma unroll
      for (int i = 0; i < kActVecs; ++i) {
        const uint32_t g = g0 + i * lanes;
        b[i] = load_kept8(a.kept, row, g, g < groups ? in_group(a.dim, g) : 0);
        code[i] = g < groups ? load_kept_code(a.kept, row, g) : 0;
      }
#pragma unroll
      for (int i = 0; i < kActVecs; ++i) {
        const uint32_t g = g0 + i * lanes;
        if (g >= groups) break;
        float f[8];
        act_decode8(b[i], act_scale(code[i]), f);
        store8<DT, kStreams<DT>>(a.x.data + (row * a.x.stride + 8ull * g) * kEsz<DT>, f, in_group(a.dim, g));
      }
    }
  }
}

uint32_t act_lanes(uint32_t dim) {
  uint32_t lg = 2;
  while ((8u << lg) < dim && (1u << lg) < kActThreads) ++lg;
  return lg;
}

}  // namespace

hipError_t launch_act_save(const ActCopy& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const uint32_t lg = act_lanes(a.dim);
  const uint64_t per_block = kActThreads >> lg;
  const uint32_t grid = grid_for((a.rows + per_block - 1) / per_block, kActThreads);
  return launch_op(a.dtype == kBf16 ? act_save_kernel<kBf16> : act_save_kernel<kF32>, grid, kActThreads, st, a, lg);
}

hipError_t launch_act_load(const ActCopy& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const uint32_t lg = act_lanes(a.dim);
  const uint64_t per_block = kActThreads >> lg;
  const uint32_t grid = grid_for((a.rows + per_block - 1) / per_block, kActThreads);
  return launch_op(a.dtype == kBf16 ? act_load_kernel<kBf16> : act_load_kernel<kF32>, grid, kActThreads, st, a, lg);
}

}  // namespace lc
