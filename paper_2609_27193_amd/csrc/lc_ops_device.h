// Device helpers shared by the training operators' kernels: rows in groups of
// eight elements at any element address, sums over a wave and a block, and
// the 8-bit form of a kept activation.
#pragma once

#include <type_traits>

#include "lc_device.h"
#include "lc_ops.h"

namespace lc {
namespace {

// A launch that reports its own error and leaves the program's alone.
template <typename... P>
__host__ hipError_t launch_op(void (*kernel)(P...), dim3 grid, uint32_t threads, hipStream_t st,
                              std::common_type_t<P>... args) {
  void* at[] = {&args...};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, 0, st);
  if (e != hipSuccess) (void)hipGetLastError();  // reported here
  return e;
}

constexpr int kBf16 = 1;
constexpr int kF32 = 2;
// Rows in bf16 that a kernel reads or writes once go past the caches, a lane's 16
// bytes in one access (the norm gradient's dx does not, see there).  16384 x 4096
// from five sets of arrays in turn, us through the caches and past them: norm 55.3
// and 52.6, with rows kept and read back 99.5 and 93.4, its gradient from x 83.2
// and 74.5, from kept rows 72.3 and 68.5, rows kept and read back 70.0 and 66.5.
// (Of one set over and over, what a cache still holds makes up for it: the norm
// alone takes 43 and 50.)  fp32 rows, whose 32 bytes a lane come in two halves,
// go through them (the norm 101 us, past them 107).
template <int DT>
constexpr bool kStreams = DT == kBf16;
template <int DT>
constexpr uint32_t kEsz = DT == kBf16 ? 2 : 4;

// fp32 to bf16, to nearest, halves to even; a NaN stays one.
__device__ __forceinline__ uint16_t to_bf16(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7FC0u;
  u += 0x7FFFu + ((u >> 16) & 1u);
  return static_cast<uint16_t>(u >> 16);
}

// The same for two at once, in the instruction that gfx950 has for it.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

typedef const __attribute__((address_space(1))) u32x4_any2 gc_u32x4_any2;
typedef const __attribute__((address_space(1))) u32x4_any4 gc_u32x4_any4;
typedef const __attribute__((address_space(1))) uint16_t gc_u16;
typedef const __attribute__((address_space(1))) float gc_f32;

template <int DT>
__device__ __forceinline__ float load1(uint64_t p) {
  if constexpr (DT == kBf16) return __uint_as_float(static_cast<uint32_t>(*(gc_u16*)p) << 16);
  else return *(gc_f32*)p;
}
template <int DT>
__device__ __forceinline__ void store1(uint64_t p, float v) {
  if constexpr (DT == kBf16) *(g_u16*)p = to_bf16(v);
  else *(g_f32*)p = v;
}
// One element of a small array whose type only the call knows.
// (`dtype` is the same for the whole grid: the branch costs nothing.)
__device__ __forceinline__ float load_param(uint64_t p, uint64_t i, int dtype) {
  return dtype == kBf16 ? load1<kBf16>(p + 2 * i) : load1<kF32>(p + 4 * i);
}
__device__ __forceinline__ void store_param(uint64_t p, uint64_t i, int dtype, float v) {
  if (dtype == kBf16) store1<kBf16>(p + 2 * i, v);
  else store1<kF32>(p + 4 * i, v);
}

// Eight elements as they lie in memory: 16 or 32 bytes, at any element.
template <int DT>
struct Raw8 {
  u32x4 v[DT == kBf16 ? 1 : 2];
};
// NT: non-temporal.
template <int DT, bool NT = false>
__device__ __forceinline__ Raw8<DT> load8_raw(uint64_t p) {
  Raw8<DT> r;
  if constexpr (DT == kBf16) {
    if constexpr (NT) r.v[0] = __builtin_nontemporal_load((gc_u32x4_any2*)p);
    else r.v[0] = *(gc_u32x4_any2*)p;
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (NT) r.v[i] = __builtin_nontemporal_load((gc_u32x4_any4*)(p + 16 * i));
      else r.v[i] = *(gc_u32x4_any4*)(p + 16 * i);
    }
  }
  return r;
}
// The first n of the eight, zeros behind them (a row's last group).
template <int DT, bool NT = false>
__device__ __forceinline__ Raw8<DT> load8_raw(uint64_t p, int n) {
  if (n >= 8) return load8_raw<DT, NT>(p);
  Raw8<DT> r;
  for (auto& q : r.v) q = u32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    if (i >= n) break;
    if constexpr (DT == kBf16)
      r.v[0][i / 2] |= static_cast<uint32_t>(*(gc_u16*)(p + 2 * i)) << (16 * (i & 1));
    else
      r.v[i / 4][i % 4] = __float_as_uint(*(gc_f32*)(p + 4 * i));
  }
  return r;
}
// The eight elements moved down by s, zeros behind them.
template <int DT>
__device__ __forceinline__ void move_down8(Raw8<DT>& r, uint32_t s) {
  if constexpr (DT == kBf16) {
    u32x4& v = r.v[0];
    if (s & 4) v = u32x4{v[2], v[3], 0, 0};
    if (s & 2) v = u32x4{v[1], v[2], v[3], 0};
    if (s & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  } else {
    u32x4 &a = r.v[0], &b = r.v[1];
    if (s & 4) {
      a = b;
      b = u32x4{0, 0, 0, 0};
    }
    if (s & 2) {
      a = u32x4{a[2], a[3], b[0], b[1]};
      b = u32x4{b[2], b[3], 0, 0};
    }
    if (s & 1) {
      a = u32x4{a[1], a[2], a[3], b[0]};
      b = u32x4{b[1], b[2], b[3], 0};
    }
  }
}
// Group g of a row of dim >= 8 elements at `row`, in two steps.  The last group
// of a row that is no multiple of eight is read from eight elements before the
// end and moved down by trim8_row: one load, where an element at a time takes
// seven and the registers for them.  A thread moves its groups when all their
// loads are under way, for that is where it waits for them.  n: the group's
// elements, at most 0 for a group that is not there, which reads zeros.
__device__ __forceinline__ uint32_t missing8(int n) { return n > 0 && n < 8 ? 8 - n : 0; }
template <int DT, bool NT = false>
__device__ __forceinline__ Raw8<DT> load8_row(uint64_t row, uint32_t g, int n) {
  Raw8<DT> r;
  for (auto& q : r.v) q = u32x4{0, 0, 0, 0};
  if (n > 0) r = load8_raw<DT, NT>(row + (8ull * g - missing8(n)) * kEsz<DT>);
  return r;
}
template <int DT>
__device__ __forceinline__ void trim8_row(Raw8<DT>& r, uint32_t dim, int n) {
  if (dim % 8) move_down8<DT>(r, missing8(n));  // the same for the whole grid
}
template <int DT>
__device__ __forceinline__ void unpack8(const Raw8<DT>& r, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (DT == kBf16) f[i] = i & 1 ? bf_hi(r.v[0][i / 2]) : bf_lo(r.v[0][i / 2]);
    else f[i] = __uint_as_float(r.v[i / 4][i % 4]);
  }
}
template <int DT, bool NT = false>
__device__ __forceinline__ void store8(uint64_t p, const float (&f)[8], int n) {
  if (n >= 8) {
    if constexpr (DT == kBf16) {
      const u32x4 v = {pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
      if constexpr (NT) __builtin_nontemporal_store(v, (g_u32x4_any2*)p);
      else *(g_u32x4_any2*)p = v;
    } else {
      const u32x4 a = {__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
      const u32x4 b = {__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])};
      *(g_u32x4_any4*)p = a;
      *(g_u32x4_any4*)(p + 16) = b;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < n) store1<DT>(p + kEsz<DT> * i, f[i]);
}
// Group g of a small array of `dim` elements, whose type only the call knows;
// p 0: `other` for each.
__device__ __forceinline__ void load_params8(uint64_t p, int dtype, uint32_t g, int n, float other, float (&f)[8]) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = other;
  } else if (dtype == kBf16) {
    unpack8<kBf16>(load8_raw<kBf16>(p + 16ull * g, n), f);
  } else {
    unpack8<kF32>(load8_raw<kF32>(p + 32ull * g, n), f);
  }
}
// Elements of group g of a row of `dim` that exist (at most 0 when none does).
__device__ __forceinline__ int in_group(uint32_t dim, uint32_t g) {
  return static_cast<int>(dim) - static_cast<int>(g * 8u);
}

// Item `it` of a kernel whose blocks take rows: runs of 32 items per XCD, so that
// neighbours meet in one L2 (65536 x 1024 kept in 8 bits and read back 76.0 us, in
// runs 70.4; rows of 4096, and norms, alike).  Beyond the dispatch limit, in order.
__device__ __forceinline__ uint64_t row_item(uint64_t it, uint64_t items) {
  return items <= gridDim.x ? remap_xcd_runs<32>(static_cast<uint32_t>(it), static_cast<uint32_t>(items)) : it;
}

// ---- sums over a wave and a block, fixed order ---------------------------------
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ float dpp_f32(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xF, false));
}
// Sum over the 64 lanes, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp_f32<0xB1>(v);        // lane ^ 1
  v += dpp_f32<0x4E>(v);        // lane ^ 2
  v += dpp_f32<0x141>(v);       // the other quad of each eight
  v += dpp_f32<0x140>(v);       // the other half of each row
  v += dpp_f32<0x142, 0xA>(v);  // row_bcast:15 into rows 1 and 3
  v += dpp_f32<0x143, 0xC>(v);  // row_bcast:31 into rows 2 and 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// ---- the 8-bit form --------------------------------------------------------------
// An element is a sign, 4 exponent and 3 mantissa bits (bias 7, largest value
// 448, 0x7F not a number); the 32 elements of a block share the power of two
// 2^(code - 127), the smallest that brings the largest finite one of them to
// 448 or less.  A scaled element is rounded to nearest, halves to even: at
// most 2^-4 of itself is lost, and no element saturates, except that under the
// largest power that fp32 elements reach, 2^120, the codes end at 240, for
// 256 * 2^120 would read back as an infinity.  An element that is not finite
// becomes NaN and does not count for its block's power.
constexpr uint32_t kActTopCode = 247;
__device__ __forceinline__ uint32_t act_code(uint32_t top) {  // top: bits of the largest finite magnitude
  const int c = static_cast<int>(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return static_cast<uint32_t>(c > 0 ? c : 0);
}
__device__ __forceinline__ float act_inverse(uint32_t code) { return __uint_as_float((254u - code) << 23); }
__device__ __forceinline__ float act_scale(uint32_t code) {  // 2^-127 is below the normal range; 255 stands for NaN
  return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7FC00000u : code << 23);
}
// Eight neighbours of a block whose four groups of eight lie in one quad of
// lanes: the eight bytes, and the block's code in every lane of the quad.
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, dpp_f32<0xB1>(v));
  return fmaxf(v, dpp_f32<0x4E>(v));
}
__device__ __forceinline__ u32x2 act_encode8(float (&f)[8], uint32_t& code) {
  float top = 0;  // the larger of two passes over a NaN
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[i]));
  top = quad_max(top);
  if (!(top < __builtin_inff())) {  // an infinity, or a NaN that was not quiet
    top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool finite = (__float_as_uint(f[i]) & 0x7fffffffu) < 0x7f800000u;
      f[i] = finite ? f[i] : __uint_as_float(0x7FC00000u);
      top = finite ? fmaxf(top, fabsf(f[i])) : top;
    }
    top = quad_max(top);  // the whole quad is here: `top` was the same in its lanes
  }
  code = act_code(__float_as_uint(top));
  const float inv = act_inverse(code);
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = f[i] * inv;
  if (code == kActTopCode) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = q[i] > 240.0f ? 240.0f : q[i] < -240.0f ? -240.0f : q[i];
  }
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
  return u32x2{static_cast<uint32_t>(lo), static_cast<uint32_t>(hi)};
}
__device__ __forceinline__ void act_decode8(u32x2 b, float scale, float (&f)[8]) {
  const f32x2 p0 = __builtin_amdgcn_cvt_pk_f32_fp8(b[0], false), p1 = __builtin_amdgcn_cvt_pk_f32_fp8(b[0], true);
  const f32x2 p2 = __builtin_amdgcn_cvt_pk_f32_fp8(b[1], false), p3 = __builtin_amdgcn_cvt_pk_f32_fp8(b[1], true);
  f[0] = p0[0] * scale;
  f[1] = p0[1] * scale;
  f[2] = p1[0] * scale;
  f[3] = p1[1] * scale;
  f[4] = p2[0] * scale;
  f[5] = p2[1] * scale;
  f[6] = p3[0] * scale;
  f[7] = p3[1] * scale;
}

typedef u32x2 __attribute__((aligned(1))) u32x2_any1;
typedef __attribute__((address_space(1))) u32x2_any1 g_u32x2_any1;
typedef const __attribute__((address_space(1))) u32x2_any1 gc_u32x2_any1;
typedef __attribute__((address_space(1))) uint8_t g_u8;
typedef const __attribute__((address_space(1))) uint8_t gc_u8;
__device__ __forceinline__ u32x2 load_codes8(uint64_t p, int n) {
  if (n >= 8) return *(gc_u32x2_any1*)p;
  u32x2 r = {0, 0};
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < n) r[i / 4] |= static_cast<uint32_t>(*(gc_u8*)(p + i)) << (8 * (i & 3));
  return r;
}
__device__ __forceinline__ void store_codes8(uint64_t p, u32x2 b, int n) {
  if (n >= 8) {
    __builtin_nontemporal_store(b, (g_u32x2_any1*)p);
    return;
  }
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < n) *(g_u8*)(p + i) = static_cast<uint8_t>(b[i / 4] >> (8 * (i & 3)));
}
// The same of a row of dim >= 8 codes at `row`, as load8_row and trim8_row.
__device__ __forceinline__ u32x2 load_codes8_row(uint64_t row, uint32_t g, int n) {
  u32x2 r = {0, 0};
  if (n > 0) r = *(gc_u32x2_any1*)(row + 8ull * g - missing8(n));
  return r;
}
__device__ __forceinline__ u32x2 trim_codes8_row(u32x2 b, int n) {
  return __builtin_bit_cast(u32x2, __builtin_bit_cast(uint64_t, b) >> (8 * missing8(n)));
}
// Group g of row r of a kept activation, and its block's scale.
__device__ __forceinline__ u32x2 load_kept8(const Kept& k, uint64_t row, uint32_t g, int n) {
  return load_codes8(k.codes + row * k.code_stride + 8ull * g, n);
}
__device__ __forceinline__ uint32_t load_kept_code(const Kept& k, uint64_t row, uint32_t g) {
  return *(gc_u8*)(k.scales + row * k.scale_stride + g / 4);
}
__device__ __forceinline__ void store_kept8(const Kept& k, uint64_t row, uint32_t g, int n, u32x2 b, uint32_t code) {
  if (n <= 0) return;
  store_codes8(k.codes + row * k.code_stride + 8ull * g, b, n);
  if (g % 4 == 0) *(g_u8*)(k.scales + row * k.scale_stride + g / 4) = static_cast<uint8_t>(code);
}

}  // namespace
}  // namespace lc
