// Activations kept in 8 bits: written and read back.  Both are bound by memory;
// a row's groups of eight elements go to consecutive lanes, so that the four
// groups of a 32-element block lie in one quad of lanes, which finds the
// block's power of two without shared memory.
#include "lc_ops_device.h"

namespace lc {
namespace {

constexpr uint32_t kActThreads = 256;

// `lanes` threads (a power of two, 4 at least) take a row.
template <int DT>
__global__ __launch_bounds__(kActThreads) void act_save_kernel(ActCopy a, uint32_t lanes_log2) {
  const uint32_t lanes = 1u << lanes_log2, per_block = kActThreads >> lanes_log2;
  const uint32_t groups = (a.dim + 31) / 32 * 4, lane = threadIdx.x & (lanes - 1);
  const uint64_t items = (a.rows + per_block - 1) / per_block;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t row = it * per_block + (threadIdx.x >> lanes_log2);
    if (row >= a.rows) continue;
    for (uint32_t g = lane; g < groups; g += lanes) {
      const int n = in_group(a.dim, g);
      float f[8];
      unpack8<DT>(load8_raw<DT>(a.x.data + (row * a.x.stride + 8ull * g) * kEsz<DT>, n), f);
      uint32_t code;
      const u32x2 q = act_encode8(f, code);
      store_kept8(a.kept, row, g, n, q, code);
    }
  }
}

template <int DT>
__global__ __launch_bounds__(kActThreads) void act_load_kernel(ActCopy a, uint32_t lanes_log2) {
  const uint32_t lanes = 1u << lanes_log2, per_block = kActThreads >> lanes_log2;
  const uint32_t groups = (a.dim + 7) / 8, lane = threadIdx.x & (lanes - 1);
  const uint64_t items = (a.rows + per_block - 1) / per_block;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t row = it * per_block + (threadIdx.x >> lanes_log2);
    if (row >= a.rows) continue;
    for (uint32_t g = lane; g < groups; g += lanes) {
      const int n = in_group(a.dim, g);
      float f[8];
      act_decode8(load_kept8(a.kept, row, g, n), act_scale(load_kept_code(a.kept, row, g)), f);
      store8<DT>(a.x.data + (row * a.x.stride + 8ull * g) * kEsz<DT>, f, n);
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
  if (a.dtype == kBf16) hipLaunchKernelGGL(act_save_kernel<kBf16>, dim3(grid), dim3(kActThreads), 0, st, a, lg);
  else hipLaunchKernelGGL(act_save_kernel<kF32>, dim3(grid), dim3(kActThreads), 0, st, a, lg);
  return hipGetLastError();
}

hipError_t launch_act_load(const ActCopy& a, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const uint32_t lg = act_lanes(a.dim);
  const uint64_t per_block = kActThreads >> lg;
  const uint32_t grid = grid_for((a.rows + per_block - 1) / per_block, kActThreads);
  if (a.dtype == kBf16) hipLaunchKernelGGL(act_load_kernel<kBf16>, dim3(grid), dim3(kActThreads), 0, st, a, lg);
  else hipLaunchKernelGGL(act_load_kernel<kF32>, dim3(grid), dim3(kActThreads), 0, st, a, lg);
  return hipGetLastError();
}

}  // namespace lc
