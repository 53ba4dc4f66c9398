// Momentum and Newton-Schulz steps for matrices of one shape:
//
//   buf <- g + mu buf,  u = g + mu buf (Nesterov) or buf,  X = u / (|u| + eps)
//   a step:  A = X X^T,  B = b A + c A A,  X <- a X + B X
//
// on the shorter side (a tall matrix is transposed on its way in and out), m rows
// of n.  Bound by the matrix cores: 4 m^2 n + 2 m^3 flops a step, of which the
// halves of A and A A below the diagonal are written from those above.
//
// X, A and B are held in fp16, times a power of two that keeps their largest
// possible element, which is bounded by the largest singular value that the steps'
// polynomials allow, at 2^15 or less: 11 bits of every element, where bf16 at the
// same rate keeps 8.  X is the sum of two such planes, 22 bits.  A result in fp32, and
// any of few rows (kOnePlane), takes A and B as two planes as well and a product as
// three (the fourth is below the last bit); the others hold one plane of A and B and
// multiply the first planes alone, and X's second enters through a X.
//
// An error of X itself lies in all singular directions, and a X carries it on: the
// steps raise the small ones by up to `a` each, a^5 = 480 in five.  An error E of A or
// B stands to the left of X, (a + B + E) X: it turns and stretches what X holds, by
// |E| over the least |a + b s^2 + c s^4| (0.64 with the default coefficients), and adds nothing
// to directions that X has little of; nor does what B misses of X's second plane, as
// B is s^2 there.  So the error does not depend on how far the singular values are
// apart.  Five steps of 3.4445, -4.775, 2.0315, bf16 results, off by of their norm: 512 x 1024
// of normal elements 2.3e-3, of rank 64 1.8e-3, of rank 4 1.7e-3, of which the
// result's own rounding is 1.7e-3 (with X in one plane 2.1e-3, 2.2e-2 and 7.2e-2).  Where
// all singular values are alike, a rounding falls the same way on each and comes out
// as a common factor, 4.5e-3 in all of 384 x 384.  X's second plane costs memory: 4096 x 4096
// 1311 -> 1367 us, two of 14336 x 4096 7.02 -> 7.36 ms, two of 400 x 20000 338 -> 410 us.
// Sums, norms and the momentum are fp32 or wider.
//
// Inside, sides are padded to multiples of 64 with zeros, which stay zeros, and a
// plane lies in panels of 32 columns: a row's 64 bytes of a panel, the next row's
// behind it.  What a step of a product takes of either operand is then whole
// kilobytes of neighbours (4096^3 with tiles of 256, X in one plane, in rows as they
// are 124 us, in panels 114, with both of its planes 124; its upper half with tiles of
// 192 100 and 78).
#include <algorithm>
#include <cmath>

#include "lc_ops_device.h"

namespace lc {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef const __attribute__((address_space(3))) f16x8 lds_f16x8;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) float lds_f32;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;

constexpr uint32_t kThreads = 256;  // four waves
constexpr uint32_t kPad = 64;       // of both sides
constexpr uint32_t kStep = 32;      // of the sum, in LDS at a time
constexpr uint32_t kPanel = 32;     // columns
constexpr uint32_t kNormBlocks = 1024;  // of one matrix, at most: every block of the next kernel adds their sums

// ---- the update and its norm -----------------------------------------------------------
// Matrix z of the group: where its gradient and momentum are.
struct OrthoIn {
  uint64_t g[kOrthoMost], g_stride[kOrthoMost];
  uint64_t buf[kOrthoMost], buf_stride[kOrthoMost];  // buf[0] 0: no momentum
  uint32_t rows, cols;
  float mu;
  int nesterov;
};
// Eight elements of u from column c on, out of the gradient and the momentum as
// it is (OLD) or already is.  The new momentum is left in b.
template <int DT, bool OLD>
__device__ __forceinline__ void update8(const OrthoIn& a, uint32_t z, uint32_t row, uint32_t c, int n, float (&u)[8],
                                        float (&b)[8]) {
  unpack8<DT>(load8_raw<DT>(a.g[z] + (row * a.g_stride[z] + c) * kEsz<DT>, n), u);
  if (!a.buf[0]) return;
  unpack8<kF32>(load8_raw<kF32>(a.buf[z] + (row * a.buf_stride[z] + c) * 4, n), b);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (OLD) b[e] = __builtin_fmaf(a.mu, b[e], u[e]);
    u[e] = a.nesterov ? __builtin_fmaf(a.mu, b[e], u[e]) : b[e];
  }
}

__device__ __forceinline__ double block_sum(double v, double (&red)[kThreads / 64]) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (uint32_t w = 1; w < kThreads / 64; ++w) v += red[w];
  return v;
}

// The new momentum, and the squares of u summed in 64 bits: a gradient's elements
// may be as small as their squares are no fp32 numbers.  Bound by memory: 4096 x 4096
// of bf16 and its momentum 33 us at 1024 blocks, 5.1 TB/s, 41 at 512 and 63 at 256;
// twice 4096 x 14336 222, 209 and 232.
template <int DT>
__global__ __launch_bounds__(kThreads) void ortho_norm_kernel(OrthoIn a, double* sums) {
  __shared__ double red[kThreads / 64];
  const uint32_t z = blockIdx.y, groups = (a.cols + 7) / 8;
  const uint32_t items = a.rows * groups;  // 2^29 at most
  double s = 0;
  for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < items; i += gridDim.x * kThreads) {
    const uint32_t row = i / groups, c = i % groups * 8;
    const int n = static_cast<int>(a.cols - c);
    float u[8], b[8];
    update8<DT, true>(a, z, row, c, n, u, b);
    if (a.buf[0]) store8<kF32>(a.buf[z] + (row * a.buf_stride[z] + c) * 4, b, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += e < n ? static_cast<double>(u[e]) * u[e] : 0.0;
  }
  s = block_sum(s, red);
  if (threadIdx.x == 0) sums[z * gridDim.x + blockIdx.x] = s;
}

// fp16 planes of eight neighbours: the value's, and of two the rest's times 2^11.
constexpr float kRestUp = 2048.0f;
template <int PLANES>
__device__ __forceinline__ void store_planes8(uint64_t p, uint64_t plane, const float (&v)[8]) {
  u32x4 hi, lo;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const f16x2 h = {static_cast<_Float16>(v[e]), static_cast<_Float16>(v[e + 1])};
    hi[e / 2] = __builtin_bit_cast(uint32_t, h);
    if constexpr (PLANES == 2) {
      const f16x2 l = {static_cast<_Float16>((v[e] - static_cast<float>(h[0])) * kRestUp),
                       static_cast<_Float16>((v[e + 1] - static_cast<float>(h[1])) * kRestUp)};
      lo[e / 2] = __builtin_bit_cast(uint32_t, l);
    }
  }
  *(g_u32x4*)p = hi;
  if constexpr (PLANES == 2) *(g_u32x4*)(p + plane) = lo;
}
typedef const __attribute__((address_space(1))) u32x4 gc_u32x4;
template <int PLANES>
struct Planes8 {
  u32x4 v[PLANES];
};
template <int PLANES>
__device__ __forceinline__ Planes8<PLANES> load_planes(uint64_t p, uint64_t plane) {
  Planes8<PLANES> x;
  x.v[0] = *(gc_u32x4*)p;
  if constexpr (PLANES == 2) x.v[1] = *(gc_u32x4*)(p + plane);
  return x;
}
// Two elements of a plane to fp32.
__device__ __forceinline__ f32x2 halves(uint32_t w) {
  const f16x2 h = __builtin_bit_cast(f16x2, w);
  return f32x2{static_cast<float>(h[0]), static_cast<float>(h[1])};
}
template <int PLANES>
__device__ __forceinline__ void unpack_planes(const Planes8<PLANES>& x, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const f32x2 h = halves(x.v[0][e / 2]);
    v[e] = h[0];
    v[e + 1] = h[1];
    if constexpr (PLANES == 2) {
      const f32x2 l = halves(x.v[1][e / 2]);
      v[e] = __builtin_fmaf(l[0], 1.0f / kRestUp, v[e]);
      v[e + 1] = __builtin_fmaf(l[1], 1.0f / kRestUp, v[e + 1]);
    }
  }
}

// Element (row, col) of a plane whose panels are `panel` bytes apart.
__device__ __forceinline__ uint64_t in_panels(uint64_t row, uint32_t col, uint64_t panel) {
  return col / kPanel * panel + row * (kPanel * 2) + col % kPanel * 2;
}

// X of the group: u over its norm, m x n, padded.
struct OrthoX {
  uint64_t x, plane, next;  // the first matrix's first plane; bytes to the second plane, to the next matrix
  uint32_t m, n;            // padded
  double eps, power;        // what X is held times
};
// Blocks of 64 x 64 of a matrix: a tall one goes through LDS.
template <int DT, bool TALL>
__global__ __launch_bounds__(kThreads) void ortho_load_kernel(OrthoIn a, OrthoX o, const double* sums, uint32_t n_sums) {
  __shared__ double red[kThreads / 64];
  __shared__ float tile[TALL ? 64 : 1][65];
  const uint32_t z = blockIdx.y;
  double s = 0;
  for (uint32_t i = threadIdx.x; i < n_sums; i += kThreads) s += sums[z * n_sums + i];
  const double norm = sqrt(block_sum(s, red));
  // a matrix of zeros stays one; of what is not finite, the whole becomes NaN
  const double by = norm < __builtin_inf() ? (norm > 0 ? o.power / (norm + o.eps) : 0.0) : __builtin_nan("");
  const uint32_t across = (TALL ? o.m : o.n) / 64;  // of the gradient's columns
  const uint32_t tiles = (o.m / 64) * (o.n / 64);
  const uint64_t base = o.x + z * o.next;
  for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const uint32_t r0 = t / across * 64, c0 = t % across * 64;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t lr = threadIdx.x / 8 + 32 * h, lc = threadIdx.x % 8 * 8, row = r0 + lr, c = c0 + lc;
      const int n = row < a.rows ? static_cast<int>(a.cols) - static_cast<int>(c) : 0;
      float u[8] = {}, b[8];
      if (n > 0) update8<DT, false>(a, z, row, c, n, u, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = e < n ? static_cast<float>(u[e] * by) : 0.0f;
      if constexpr (TALL) {
#pragma unroll
        for (int e = 0; e < 8; ++e) tile[lr][lc + e] = u[e];
      } else {
        store_planes8<2>(base + in_panels(row, c, o.m * (kPanel * 2)), o.plane, u);
      }
    }
    if constexpr (TALL) {
      __syncthreads();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t lc = threadIdx.x / 8 + 32 * h, lr = threadIdx.x % 8 * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[lr + e][lc];
        store_planes8<2>(base + in_panels(c0 + lc, r0 + lr, o.m * (kPanel * 2)), o.plane, v);
      }
      __syncthreads();
    }
  }
}

// ---- the products --------------------------------------------------------------------------
// D[i][j] = f_acc * sum over k of L[i][k] R'[k][j] + f_aux * aux[i][j], of planes of
// fp16.  A symmetric one (SYM) takes R' = R^T, with R's rows along the sum as L's, and
// computes the tiles on and above the diagonal; else R' = R.
struct OrthoProduct {
  uint64_t left, right, aux, out;              // of the group's first matrix
  uint64_t left_plane, right_plane, out_plane; // bytes to the second plane (aux: as out); of one plane not looked at
  uint64_t left_next, right_next, out_next;    // bytes to the next matrix (aux: as out)
  uint32_t left_panel, right_panel, out_panel; // bytes from panel to panel (aux: as out)
  uint32_t rows, cols, k;                      // multiples of 64
  uint32_t ti, tj, tiles, count;               // tiles down, across and of a matrix; matrices
  uint32_t splits, split_k;                    // parts of the sum and its steps a part
  float f_acc, f_aux;
  float* part;                                 // [count * tiles][splits][T][T], splits > 1
};
// Where a group's last products go: the caller's matrices.
struct OrthoOut {
  uint64_t data[kOrthoMost], stride[kOrthoMost];
  uint32_t m, n;  // of X, without its padding
  int tall, dtype;
};

__device__ __forceinline__ void ortho_place(const OrthoProduct& p, bool sym, uint32_t t, uint32_t& i, uint32_t& j) {
  if (sym) {  // columns of the upper triangle
    j = static_cast<uint32_t>((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while ((j + 1) * (j + 2) / 2 <= t) ++j;
    while (j * (j + 1) / 2 > t) --j;
    i = t - j * (j + 1) / 2;
  } else {  // eight tiles down by all across
    const uint32_t group = t / (8 * p.tj), in_g = t - group * 8 * p.tj;
    const uint32_t high = p.ti - group * 8 < 8 ? p.ti - group * 8 : 8;
    j = in_g / high;
    i = group * 8 + in_g % high;
  }
  // the same for the whole block, which the square root hides
  i = __builtin_amdgcn_readfirstlane(i);
  j = __builtin_amdgcn_readfirstlane(j);
}

constexpr int kMfma = 0x8, kVmemRead = 0x20, kLdsRead = 0x100;  // kinds of instructions, for their order

// A barrier behind which all waves have what they read from LDS and all but the
// newest N loads to LDS of each have landed.  A fence would wait for every load.
template <uint32_t N>
__device__ __forceinline__ void barrier_lds() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);  // vmcnt(N) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// A lane's 16 bytes to LDS, the wave's 64 after each other: descriptor, place, bytes,
// offset, scalar offset and two more.  The whole offset is in the operand that the
// bounds check covers.
#define LC_BUFFER_LOAD_LDS __builtin_amdgcn_raw_ptr_buffer_load_lds
__device__ __forceinline__ void load_lds(tile_t t, uint8_t* to, uint32_t off) {
  LC_BUFFER_LOAD_LDS(t, (lds_void*)to, 16, off, 0, 0, 0);
}

// Eight neighbours of row i of D from column j on, in the result's type.
template <int PLANES>
__device__ __forceinline__ void ortho_out8(const OrthoOut& o, uint32_t z, uint64_t row, uint32_t col, int n, const float (&v)[8]) {
  if (n <= 0) return;
  const uint64_t at = row * o.stride[z] + col;
  if (PLANES == 1 || o.dtype == kBf16) store8<kBf16>(o.data[z] + at * 2, v, n);
  else store8<kF32>(o.data[z] + at * 4, v, n);
}

constexpr int kSym = 0, kMid = 1, kLast = 2;

// T x T of D a block, four waves of T/2 x T/2.  A step of the sum is 32; the loads
// write LDS by themselves, four steps on their way in turn, for one wave a SIMD has
// nothing else to hide the way from HBM with (4096^3: with two steps of 64 160 us).
//
// LDS: T rows of an operand's step (L, and R of SYM), of 64 bytes along the sum, whose
// 16-byte pieces lie at c ^ row / 4 % 4, so that the 16 rows of a quarter read are in
// different banks; of R as it lies, T / 32 panels of 32 rows of 64 bytes, of which half
// a transposing read takes four rows, 256 bytes.
// PLANES: of each operand; where the result is X, it and aux have two in any case.
// GROUPS: 3 gives each of two planes' products four waves and LDS of their own, for few tiles, whose steps wait for their loads (five steps in
// fp32, all of 1024^3 232 us with one group and 190 with three, 512^3 152 and 137, six of
// 1027 x 509 232 and 208; 1500^3, where the larger tiles fill the chip, 423 and 506).
template <int MODE, int T, int PLANES, int GROUPS>
__global__ __launch_bounds__(kThreads * GROUPS, GROUPS > 1 ? GROUPS : T >= 192 ? 1 : 2) void ortho_product_kernel(OrthoProduct p, OrthoOut o) {
  static_assert(GROUPS == 1 || (GROUPS == 3 && PLANES == 2 && T == 64), "a group's sums lie in its buffers on their way");
  constexpr bool SYM = MODE == kSym;
  constexpr int HELD = SYM ? PLANES : 2;      // planes of aux and of the result
  constexpr uint32_t NF = T / 64;             // 32-wide pieces of a wave's side
  constexpr uint32_t kOperand = T * kStep * 2;  // bytes
  constexpr uint32_t kLoads = T / 64;         // of an operand, a thread
  constexpr uint32_t kOut = T / 2 + 4;        // floats from row to row on their way out
  static_assert(32 * kOut * 4 <= 2 * kOperand, "a wave's rows on their way out lie in one buffer");
  __shared__ __align__(1024) uint8_t all0[GROUPS * 2 * kOperand];
  __shared__ __align__(1024) uint8_t all1[GROUPS * 2 * kOperand];
  __shared__ __align__(1024) uint8_t all2[GROUPS * 2 * kOperand];
  __shared__ __align__(1024) uint8_t all3[GROUPS * 2 * kOperand];
  const uint32_t group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  uint8_t* const stage0 = all0 + group * 2 * kOperand;
  uint8_t* const stage1 = all1 + group * 2 * kOperand;
  uint8_t* const stage2 = all2 + group * 2 * kOperand;
  uint8_t* const stage3 = all3 + group * 2 * kOperand;
  const uint32_t tid = threadIdx.x % kThreads, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t items = p.count * p.tiles * p.splits;
  for (uint32_t b = blockIdx.x; b < items; b += gridDim.x) {
    const uint32_t item = items <= gridDim.x ? remap_xcd(b, items) : b;
    const uint32_t split = item % p.splits, tile = item / p.splits, z = tile / p.tiles;
    uint32_t ti, tj;
    ortho_place(p, SYM, tile % p.tiles, ti, tj);
    const uint32_t i0 = ti * T, j0 = tj * T;
    // the steps of this part
    const uint32_t k_begin = split * p.split_k, k_all = p.k / kStep;  // split_k is even, as k_all is
    const uint32_t k_end = k_begin + p.split_k < k_all ? k_begin + p.split_k : k_all;
    const uint64_t left = p.left + z * p.left_next + i0 * (kPanel * 2ull);
    const uint64_t right = p.right + z * p.right_next + (SYM ? j0 * (kPanel * 2ull) : static_cast<uint64_t>(j0 / kPanel) * p.right_panel);
    const uint32_t left_rows = p.rows - i0 < T ? p.rows - i0 : T, right_rows = p.cols - j0 < T ? p.cols - j0 : T;
    // a load takes 16 rows of a panel
    const uint32_t rows16 = wave * 1024 + lane / 4 * 64 + (lane % 4 ^ lane / 16) * 16;
    const uint32_t right_at = SYM ? rows16 : wave / 2 * p.right_panel + wave % 2 * 1024 + lane * 16;
    const uint32_t right_by = SYM ? 4096 : 2 * p.right_panel;  // to the thread's next load
    // Nothing is read behind an operand: rows and columns that are not there are
    // not stored, whatever LDS holds for them.
    const int left_bytes = static_cast<int>(left_rows * (kPanel * 2));
    const int right_bytes = static_cast<int>(SYM ? right_rows * (kPanel * 2) : right_rows / kPanel * p.right_panel);
    const uint64_t left_step = p.left_panel, right_step = SYM ? p.right_panel : kStep * (kPanel * 2);
    // `next` says where the next step comes from, a half step ahead of its loads: the
    // scalar unit's work would hold up the products behind a barrier.
    tile_t from_left, from_right;
    uint64_t left_next = 0, right_next = 0;
    int todo = 0, turn = 0;  // steps not yet under way; how many of them are left where the planes change
    auto next = [&] {
      from_left = make_tile(reinterpret_cast<const void*>(left_next), todo > 0 ? left_bytes : 0);
      from_right = make_tile(reinterpret_cast<const void*>(right_next), todo > 0 ? right_bytes : 0);
      left_next += left_step;
      right_next += right_step;
      --todo;
      if (PLANES == 2 && todo == turn) {
        left_next = left + k_begin * left_step;
        right_next = right + p.right_plane + k_begin * right_step;
      }
    };
    auto load_left = [&](uint8_t* stage) {
#pragma unroll
      for (uint32_t q = 0; q < kLoads; ++q)
        load_lds(from_left, stage + (q * 4 + wave) * 1024, rows16 + q * 4096);
    };
    auto load_right = [&](uint8_t* stage) {
#pragma unroll
      for (uint32_t q = 0; q < kLoads; ++q) load_lds(from_right, stage + kOperand + (q * 4 + wave) * 1024, right_at + q * right_by);
    };
    // operands of 16 of the sum
    const uint32_t wi = wave % 2 * (T / 2), wj = wave / 2 * (T / 2);
    f16x8 lf[2][NF], rf[2][NF];
    // of R as it lies: column lane % 32 of a panel, rows lane / 32 * 8 and on
    const uint32_t tr_at = kOperand + wj * (kStep * 2) + (lane / 32 * 8 + lane % 16 / 4) * 64 + lane / 16 % 2 * 32 + lane % 4 * 8;
    auto fetch = [&](uint8_t* stage, uint32_t to, uint32_t sub) {
      const uint32_t piece = ((2 * sub + lane / 32) ^ (lane / 4 % 4)) * 16;
      const auto right_of = [&](uint32_t f) {
        if constexpr (SYM) {
          rf[to][f] = *(lds_f16x8*)(stage + kOperand + (wj + 32 * f + lane % 32) * 64 + piece);
        } else {
          uint8_t* const at = stage + tr_at + f * (kPanel * kStep * 2) + sub * 1024;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 256));
          rf[to][f] = __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
      };
      right_of(0);  // in the order in which the products want them
#pragma unroll
      for (uint32_t f = 0; f < NF; ++f) lf[to][f] = *(lds_f16x8*)(stage + (wi + 32 * f + lane % 32) * 64 + piece);
#pragma unroll
      for (uint32_t f = 1; f < NF; ++f) right_of(f);
    };
    f32x16 acc[NF][NF];  // [j][i] pieces of 32: a lane holds four runs of 4 of j for one i
#pragma unroll
    for (uint32_t j = 0; j < NF; ++j)
#pragma unroll
      for (uint32_t i = 0; i < NF; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[j][i][e] = 0;
    auto multiply = [&](uint32_t of) {
#pragma unroll
      for (uint32_t j = 0; j < NF; ++j)
#pragma unroll
        for (uint32_t i = 0; i < NF; ++i) acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(rf[of][j], lf[of][i], acc[j][i], 0, 0, 0);
    };
    // One step out of `cur`: the operands of each half are read while the half before
    // it multiplies.  When all waves have the step in registers, the loads of the
    // fourth behind it go into `cur`, L's in this step's second half, R's in the next
    // one's first (into `old`): each takes the CU's address unit 16 clocks, and those
    // of four waves in a row hold up the products behind them.
    // The order lays reads and loads between the products, or the compiler reads an
    // operand right before it waits for it.
    constexpr int kProducts = NF * NF, kReads = (SYM ? 2 : 3) * NF, kPer = (kReads + kProducts - 1) / kProducts;
    constexpr int kEvery = kProducts / static_cast<int>(kLoads);
    auto order = [] {
#pragma unroll
      for (int t = 0; t < kProducts; ++t) {
        __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
        if (t * kPer < kReads) __builtin_amdgcn_sched_group_barrier(kLdsRead, kPer, 0);
        if (t % kEvery == kEvery - 1) __builtin_amdgcn_sched_group_barrier(kVmemRead, 1, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    auto step = [&](uint8_t* old, uint8_t* cur, uint8_t* nxt) {
      __builtin_amdgcn_sched_barrier(0);
      fetch(cur, 1, 1);
      load_right(old);
      next();
      multiply(0);
      order();
      barrier_lds<4 * kLoads>();  // the next step is there, the two behind it on their way
      fetch(nxt, 0, 0);
      load_left(cur);
      multiply(1);
      order();
    };
    // first the products of a second plane, of either side, then those of the first
#pragma unroll 1
    for (uint32_t big = PLANES == 2 && GROUPS == 1 ? 0 : 1; big < 2; ++big) {
      const uint32_t steps = (k_end - k_begin) * (big ? 1 : 2);  // even
      todo = static_cast<int>(steps);
      turn = big ? -1 - todo : todo / 2;  // never, with the first planes
      left_next = left + ((GROUPS == 1 ? big : group) == 0 && PLANES == 2 ? p.left_plane : 0) + k_begin * left_step;
      right_next = right + (GROUPS > 1 && group == 1 ? p.right_plane : 0) + k_begin * right_step;
      for (uint8_t* const stage : {stage0, stage1, stage2}) {
        next();
        load_left(stage);
        load_right(stage);
      }
      next();
      load_left(stage3);
      barrier_lds<5 * kLoads>();
      fetch(stage0, 0, 0);
      for (uint32_t s = 0; s < steps / 4; ++s) {
        step(stage3, stage0, stage1);
        step(stage0, stage1, stage2);
        step(stage1, stage2, stage3);
        step(stage2, stage3, stage0);
      }
      if (steps % 4) {
        step(stage3, stage0, stage1);
        step(stage0, stage1, stage2);
      }
      if (PLANES == 2 && !big) {
        barrier_lds<0>();
#pragma unroll
        for (uint32_t j = 0; j < NF; ++j)
#pragma unroll
          for (uint32_t i = 0; i < NF; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[j][i][e] *= 1.0f / kRestUp;
      }
    }

    // out through LDS, 32 rows a wave at a time; the next rows of aux are on their way
    // meanwhile, clamped to what is there: what is not is not stored
    constexpr uint32_t kRounds = T / 32;  // of 16 rows of a panel
    const uint32_t row0 = i0 + wi, col0 = j0 + wj;
    const uint64_t out = p.out + z * p.out_next, aux = p.aux + z * p.out_next;
    const bool has_aux = p.aux && p.splits == 1 && group == GROUPS - 1;
    Planes8<HELD> x[2][kRounds];
    auto load_aux = [&](uint32_t f) {
#pragma unroll
      for (uint32_t r = 0; r < kRounds; ++r) {
        const uint32_t row = row0 + 32 * f + r % 2 * 16 + lane / 4, col = col0 + r / 2 * kPanel + lane % 4 * 8;
        const uint64_t at = in_panels(row < p.rows ? row : p.rows - 1, col < p.cols ? col : p.cols - 8, p.out_panel);
        x[f % 2][r] = load_planes<HELD>(aux + at, p.out_plane);
      }
    };
    if (has_aux) {
      load_aux(0);
      barrier_lds<kRounds * HELD>();
    } else {
      barrier_lds<0>();
    }
    if constexpr (GROUPS > 1) {  // the last group adds the others' sums
      constexpr uint32_t kTheirs = 2 * kOperand;
      if (group < GROUPS - 1) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(lds_f32x4*)((q < 2 ? (q == 0 ? stage0 : stage1) : q == 2 ? stage2 : stage3) + tid * 16) =
              f32x4{acc[0][0][4 * q], acc[0][0][4 * q + 1], acc[0][0][4 * q + 2], acc[0][0][4 * q + 3]};
        barrier_lds<0>();
        __syncthreads();  // with the last group, behind the item
        continue;
      }
      barrier_lds<kRounds * HELD>();
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint8_t* const at = (q < 2 ? (q == 0 ? all0 : all1) : q == 2 ? all2 : all3) + tid * 16;
        const f32x4 u = *(lds_f32x4*)at, v = *(lds_f32x4*)(at + kTheirs);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[0][0][4 * q + e] = __builtin_fmaf(u[e] + v[e], 1.0f / kRestUp, acc[0][0][4 * q + e]);
      }
    }
    lds_f32* const mine = (lds_f32*)(wave < 2 ? (wave == 0 ? stage0 : stage1) : wave == 2 ? stage2 : stage3);
    const bool turned = SYM ? ti != tj : MODE == kLast;
#pragma unroll
    for (uint32_t f = 0; f < NF; ++f) {
      if (has_aux && f + 1 < NF) load_aux(f + 1);
#pragma unroll
      for (uint32_t j = 0; j < NF; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *(lds_f32x4*)(mine + lane % 32 * kOut + 32 * j + 8 * r + lane / 32 * 4) =
              f32x4{acc[j][f][4 * r], acc[j][f][4 * r + 1], acc[j][f][4 * r + 2], acc[j][f][4 * r + 3]};
      if (p.splits > 1) {
        float* const to = p.part + (static_cast<uint64_t>(tile) * p.splits + split) * (T * T) + (wi + 32 * f) * T + wj;
#pragma unroll
        for (uint32_t r = 0; r < kRounds; ++r) {
          const uint32_t q = r % 2 * 16 + lane / 4, c = r / 2 * kPanel + lane % 4 * 8;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            *(f32x4*)(to + q * T + c + 4 * h) = *(lds_f32x4*)(mine + q * kOut + c + 4 * h);
        }
        continue;
      }
#pragma unroll
      for (uint32_t r = 0; r < kRounds; ++r) {
        const uint32_t q = r % 2 * 16 + lane / 4, c = r / 2 * kPanel + lane % 4 * 8, row = row0 + 32 * f + q, col = col0 + c;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = mine[q * kOut + c + e] * p.f_acc;
        if (has_aux) {
          float y[8];
          unpack_planes<HELD>(x[f % 2][r], y);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(p.f_aux, y[e], v[e]);
        }
        if (MODE != kLast && row < p.rows && col < p.cols)
          store_planes8<HELD>(out + in_panels(row, col, p.out_panel), p.out_plane, v);
        if (turned) {
#pragma unroll
          for (int e = 0; e < 8; ++e) mine[q * kOut + c + e] = v[e];
        }
      }
      if (!turned) continue;
      // the caller's rows, or the other side of the diagonal: four lanes take 32 neighbours of a column of these rows
#pragma unroll 2
      for (uint32_t r = 0; r < kRounds; ++r) {
        constexpr uint32_t kGroups = T / 16;  // of eight columns in a wave's row
        const uint32_t g = lane + 64 * r;
        float v[8];
        if (MODE == kLast && !o.tall) {
          const uint32_t q = g / kGroups, c = g % kGroups * 8, row = row0 + 32 * f + q, col = col0 + c;
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = mine[q * kOut + c + e];
          if (row < o.m) ortho_out8<PLANES>(o, z, row, col, static_cast<int>(o.n) - static_cast<int>(col), v);
          continue;
        }
        const uint32_t j = g / 4, c = g % 4 * 8, row = col0 + j, col = row0 + 32 * f + c;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = mine[(c + e) * kOut + j];
        if (MODE == kLast) {
          if (row < o.n) ortho_out8<PLANES>(o, z, row, col, static_cast<int>(o.m) - static_cast<int>(col), v);
        } else if (row < p.cols && col < p.rows) {
          store_planes8<HELD>(out + in_panels(row, col, p.out_panel), p.out_plane, v);
        }
      }
    }
    __syncthreads();
  }
}

// The parts' sums of a symmetric product, to both sides of the diagonal.  A block
// takes 8 rows of a panel: 32 groups of eight columns, whose parts eight slices of
// threads add in turn; the slices' sums are added in order.
constexpr uint32_t kSlices = 8, kJoinRows = kThreads / kSlices / 4;
template <int PLANES>
__global__ __launch_bounds__(kThreads) void ortho_join_kernel(OrthoProduct p, uint32_t side) {
  __shared__ float sums[kSlices][8][kThreads / kSlices];
  __shared__ float out_rows[kJoinRows][kPanel + 1];
  const uint32_t across = side / kPanel, per_tile = across * (side / kJoinRows);
  const uint32_t items = p.count * p.tiles * per_tile;
  const uint32_t own = threadIdx.x % (kThreads / kSlices), slice = threadIdx.x / (kThreads / kSlices);
  for (uint32_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint32_t tile = it / per_tile, z = tile / p.tiles, sub = it % per_tile;
    const uint32_t si = sub / across * kJoinRows, sj = sub % across * kPanel;
    uint32_t ti, tj;
    ortho_place(p, true, tile % p.tiles, ti, tj);
    const uint32_t i0 = ti * side + si, j0 = tj * side + sj;
    const bool on = i0 < p.rows && j0 < p.cols;  // the same for the block
    const uint64_t out = p.out + z * p.out_next, aux = p.aux + z * p.out_next;
    const uint32_t q = own / 4, c = own % 4 * 8;
    float v[8] = {}, x[8];
    if (on) {
      const float* const part = p.part + (static_cast<uint64_t>(tile) * p.splits * side + si + q) * side + sj + c;
#pragma unroll 4
      for (uint32_t s = slice; s < p.splits; s += kSlices) {
        unpack8<kF32>(load8_raw<kF32>(reinterpret_cast<uint64_t>(part + static_cast<uint64_t>(s) * side * side)), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += x[e];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[slice][e][own] = v[e];
    __syncthreads();
    if (on && slice == 0) {
#pragma unroll
      for (uint32_t s = 1; s < kSlices; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += sums[s][e][own];
      const uint64_t at = in_panels(i0 + q, j0 + c, p.out_panel);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= p.f_acc;
      if (p.aux) {
        unpack_planes<PLANES>(load_planes<PLANES>(aux + at, p.out_plane), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(p.f_aux, x[e], v[e]);
      }
      store_planes8<PLANES>(out + at, p.out_plane, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) out_rows[q][c + e] = v[e];
    }
    __syncthreads();
    if (on && slice == 0 && ti != tj) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = out_rows[e][own];
      store_planes8<PLANES>(out + in_panels(j0 + own, i0, p.out_panel), p.out_plane, v);
    }
    __syncthreads();
  }
}

// ---- the plan ------------------------------------------------------------------------------
uint64_t padded(uint64_t x) { return (x + kPad - 1) / kPad * kPad; }

// How the products of a shape are cut.
struct OrthoCut {
  uint32_t side, groups, ti, tj, tiles, splits, split_k;
};
// What a block of a side takes, measured (us): beside its steps, and a step of 32, of
// 1 to per_cu blocks a CU; `lone`, a step of one on the whole chip.  A step of three
// groups is one of each.  The upper half and the whole of n^3 (without X's second plane,
// which any side writes alike), tiles of 64 / 128 / 192 / 256: n = 1024 8, 11, 18, 29 and 8, 10, 16, 25; 2048 20, 19, 29, 45 and 28, 21, 29, 43;
// 3000 58, 43, 42, 64 and 88, 65, 51, 65; 4096 154, 90, 68, 88 and 222, 125, 127, 112.
struct OrthoCost {
  uint32_t side, groups, per_cu;
  double lone, base[4], step[4];
};
constexpr OrthoCost kOrthoCosts[] = {{64, 1, 4, 0.114, {4.0, 4.5, 4.5, 5.5}, {0.125, 0.15, 0.26, 0.35}},
                                     {64, 3, 1, 0.2, {5.0}, {0.19}},
                                     {128, 1, 2, 0.144, {6.0, 9.6}, {0.21, 0.43}},
                                     {192, 1, 1, 0.25, {9.0}, {0.46}},
                                     {256, 1, 1, 0.44, {13.0}, {0.76}}};
double ortho_us(const OrthoCost& c, uint64_t blocks, uint32_t steps) {
  const uint64_t rounds = blocks / (256 * c.per_cu), rest = blocks % (256 * c.per_cu);
  double us = rounds * (c.base[c.per_cu - 1] + steps * c.step[c.per_cu - 1]);
  if (rest) {
    const uint32_t b = static_cast<uint32_t>((rest + 255) / 256) - 1;
    const double step = b == 0 ? c.lone + (c.step[0] - c.lone) * (rest / 256.0) : c.step[b];
    us += (c.base[b] + steps * step) * (rounds && c.per_cu == 4 ? 0.6 : 1.0);  // small blocks begin beside the round before
  }
  return us;
}
constexpr uint64_t kMostPartBytes = 256ull * 256 * 256 * 4;  // of a round of blocks
constexpr bool within_most_parts() {
  for (const OrthoCost& c : kOrthoCosts)
    if (256ull * c.per_cu * c.side * c.side * 4 > kMostPartBytes) return false;
  return true;
}
static_assert(within_most_parts(), "parts are of one round at most");
// A symmetric product may be split over its sum, whose parts then go through memory
// (4 TB/s there and back) and a join.
OrthoCut ortho_cut(uint64_t rows, uint64_t cols, uint64_t k, uint32_t count, bool sym, int planes) {
  const uint32_t pairs = static_cast<uint32_t>(k / (2 * kStep));  // of steps
  OrthoCut best{};
  double best_us = 1e30;
  for (const OrthoCost& cost : kOrthoCosts) {
    if (planes == 1 && cost.groups > 1) continue;
    if (planes == 2 && cost.side == 256) continue;  // its sums leave no registers for a second plane's way
    OrthoCut c{};
    c.side = cost.side;
    c.groups = cost.groups;
    c.ti = static_cast<uint32_t>((rows + c.side - 1) / c.side);
    c.tj = static_cast<uint32_t>((cols + c.side - 1) / c.side);
    c.tiles = sym ? c.ti * (c.ti + 1) / 2 : c.ti * c.tj;
    const uint64_t tiles = static_cast<uint64_t>(c.tiles) * count;
    for (uint32_t splits = 1; splits == 1 || (sym && splits <= pairs && tiles * splits <= 256 * cost.per_cu); splits += 1 + splits / 16) {
      c.split_k = (pairs + splits - 1) / splits * 2;
      c.splits = (2 * pairs + c.split_k - 1) / c.split_k;
      const double us = ortho_us(cost, tiles * c.splits, c.split_k * (planes == 2 && c.groups == 1 ? 3 : 1)) +
                        (c.splits > 1 ? 4.5 + tiles * c.splits * c.side * c.side * 8 / 4e6 : 0.0);
      if (us < best_us) {
        best_us = us;
        best = c;
      }
    }
  }
  return best;
}
uint64_t ortho_part_bytes(const OrthoCut& c, uint32_t count) {
  return c.splits > 1 ? static_cast<uint64_t>(c.tiles) * count * c.splits * c.side * c.side * 4 : 0;
}

// A bf16 result of a shorter side of this and more takes A, B and the products from
// one plane and is off by 2.0e-3 (4096) to 2.7e-3 (384 x 16000) of its norm for normal elements,
// 1.7e-3 of it its own rounding.  Below, one plane would give 2.3e-3 (128 x 1024) to 3.1e-3
// (16 x 16) and save launches' time above all, 98 us for 134 (256 x 1024), 86 for 116
// (four of 256 x 256), at most 528 for 809 (four of 383 x 16000); two give 1.7e-3.  Above, the
// products are the time, and two planes take three times as many (2048 x 2048 668 us
// for 296, 4096 x 4096 3808 for 1358).
constexpr uint64_t kOnePlane = 384;

// Of X, A and B of the matrices at once, more than which only a single one takes.  Of
// such long ones fewer keep the chip at work as well: 64 of 256 x 65536 (bf16, five
// steps) in three turns 26.2 ms, in one, of 8 GiB, 26.6; 24 of 512 x 65536 (fp32, three) in two
// 19.0 and in one 19.0; eight of 4096 x 65536 (bf16, two) each alone 53.8, four at once 56.8.
// Even turns: 17 of 2048 x 2048 3.62 ms, as 16 and 1 3.79.
constexpr uint64_t kOrthoSpace = 4ull << 30;

// Matrices at once and their place in the workspace.
struct OrthoPlan {
  uint64_t m, n;  // padded
  bool tall;
  uint32_t planes, group;
  uint64_t x_bytes, a_bytes;  // of one matrix, all planes; X has two
  uint64_t sums, x0, x1, a, b, part, bytes;  // offsets, and the whole
  OrthoCut gram, poly, mid;
};
OrthoPlan ortho_plan(uint32_t count, uint64_t rows, uint64_t cols, int out_dtype) {
  OrthoPlan p{};
  p.tall = rows > cols;
  p.m = padded(p.tall ? cols : rows);
  p.n = padded(p.tall ? rows : cols);
  p.planes = out_dtype == kF32 || std::min(rows, cols) < kOnePlane ? 2 : 1;
  p.x_bytes = p.m * p.n * 4;
  p.a_bytes = p.m * p.m * 2 * p.planes;
  // as many as keep the chip at work, a round of 256 tiles four times, unless they are so
  // long that fewer do and more would only take memory
  const uint64_t tiles = ((p.m + 255) / 256) * ((p.m + 255) / 256);
  const uint64_t most = std::max<uint64_t>(1, std::min(1024 / tiles, kOrthoSpace / (2 * (p.x_bytes + p.a_bytes))));
  const uint32_t places = static_cast<uint32_t>(std::min<uint64_t>(count, most));
  const uint32_t turns = (count + places - 1) / places;
  p.group = (count + turns - 1) / turns;  // 17 as 9 and 8, not as 16 and 1
  p.gram = ortho_cut(p.m, p.m, p.n, p.group, true, p.planes);
  p.poly = ortho_cut(p.m, p.m, p.m, p.group, true, p.planes);
  p.mid = ortho_cut(p.m, p.n, p.m, p.group, false, p.planes);
  p.sums = 0;
  p.x0 = kOrthoMost * kNormBlocks * 8;
  p.x1 = p.x0 + places * p.x_bytes;
  p.a = p.x1 + places * p.x_bytes;
  p.b = p.a + places * p.a_bytes;
  p.part = p.b + places * p.a_bytes;
  // of several turns room for any parts, lest 17 need less than 16
  p.bytes = p.part + (turns > 1 ? kMostPartBytes : std::max(ortho_part_bytes(p.gram, p.group), ortho_part_bytes(p.poly, p.group)));
  return p;
}

// The power of two that brings `bound` to 2^14 .. 2^15.
int exponent_for(double bound) {
  if (!(bound > 0)) return 0;
  int e;
  std::frexp(bound, &e);  // bound < 2^e
  return 15 - e;
}
double largest(double x, double a, double b, double c) { return std::fabs(x * (a + x * x * (b + x * x * c))); }
// The largest |a s + b s^3 + c s^5| of s in [0, top].
double ortho_bound(double top, const double* k) {
  double best = largest(top, k[0], k[1], k[2]);
  const double m = std::max({std::fabs(k[0]), std::fabs(k[1]), std::fabs(k[2])});
  if (m == 0) return 0;
  // its slope is a + 3 b q + 5 c q^2, q = s^2, over m, lest d overflows.  -b and the root of
  // d are added where both have one sign: their difference would lose the smaller
  // root, which the other gives as it divides c / a.
  const double a = 5 * (k[2] / m), b = 3 * (k[1] / m), c = k[0] / m, d = b * b - 4 * a * c;
  double roots[2];
  int n = 0;
  if (d >= 0) {
    const double t = -0.5 * (b + std::copysign(std::sqrt(d), b));
    if (a != 0) roots[n++] = t / a;
    if (t != 0) roots[n++] = c / t;
  }
  for (int i = 0; i < n; ++i)
    if (roots[i] > 0 && roots[i] < top * top) best = std::max(best, largest(std::sqrt(roots[i]), k[0], k[1], k[2]));
  return best;
}
// The same of |b q + c q^2|, q in [0, top].
double ortho_bound_b(double top, double b, double c) {
  double best = std::fabs(top * (b + top * c));
  if (c != 0) {
    const double q = -b / (2 * c);
    if (q > 0 && q < top) best = std::max(best, std::fabs(q * (b + q * c)));
  }
  return best;
}
// What the roundings of a step may add to a bound: they move singular values by some
// 0.1 % a step (one plane; 0.4 % in five where all are alike).  fp16 itself holds twice what X,
// A and B are brought to.  More would refuse steps whose polynomial turns upwards right
// behind the range that the one before leaves: with 2 % a step (8.2, -22.9, 16.5), (4.07, -2.87,
// 0.522), (3.92, -2.83, 0.53), (3.29, -2.42, 0.49), ... go from 2.03 to 2.29, 8.63, 2e4 and on.
constexpr double kSlack = 1.005;

template <int MODE, int T, int PLANES, int GROUPS = 1>
hipError_t product_as(const OrthoProduct& p, const OrthoOut& o, hipStream_t st) {
  const uint64_t items = static_cast<uint64_t>(p.count) * p.tiles * p.splits;
  return launch_op(ortho_product_kernel<MODE, T, PLANES, GROUPS>, grid_for(items, kThreads * GROUPS), kThreads * GROUPS, st, p, o);
}
template <int MODE, int PLANES>
hipError_t product_of(const OrthoProduct& p, const OrthoOut& o, const OrthoCut& c, hipStream_t st) {
  if constexpr (PLANES == 1)
    if (c.side == 256) return product_as<MODE, 256, PLANES>(p, o, st);
  if constexpr (PLANES == 2)
    if (c.groups == 3) return product_as<MODE, 64, PLANES, 3>(p, o, st);
  if (c.side == 192) return product_as<MODE, 192, PLANES>(p, o, st);
  if (c.side == 128) return product_as<MODE, 128, PLANES>(p, o, st);
  return product_as<MODE, 64, PLANES>(p, o, st);
}
template <int MODE>
hipError_t product(OrthoProduct& p, const OrthoOut& o, const OrthoCut& c, uint32_t planes, hipStream_t st) {
  p.ti = c.ti;
  p.tj = c.tj;
  p.tiles = c.tiles;
  p.splits = c.splits;
  p.split_k = c.split_k;
  const hipError_t e = planes == 2 ? product_of<MODE, 2>(p, o, c, st) : product_of<MODE, 1>(p, o, c, st);
  if (e != hipSuccess || p.splits == 1) return e;
  const uint64_t items = static_cast<uint64_t>(p.count) * p.tiles * (c.side / kPanel) * (c.side / kJoinRows);
  return launch_op(planes == 2 ? ortho_join_kernel<2> : ortho_join_kernel<1>, grid_for(items, kThreads), kThreads, st, p, c.side);
}

template <int DT>
hipError_t load_x(const OrthoIn& in, const OrthoX& x, bool tall, dim3 grid, const double* sums, uint32_t n_sums, hipStream_t st) {
  return launch_op(tall ? ortho_load_kernel<DT, true> : ortho_load_kernel<DT, false>, grid, kThreads, st, in, x, sums, n_sums);
}

}  // namespace

bool ortho_in_range(uint32_t steps, const double* coefs) {
  double x = 1.0;
  for (uint32_t s = 0; s < steps; ++s) {
    const double* const k = coefs + 3 * s;
    const double q = x * x * kSlack;
    x = ortho_bound(x, k) * kSlack;
    if (x != 0 && x < 1.0 / kOrthoLargest) return false;
    if (!(x < kOrthoLargest) || !(ortho_bound_b(q, k[1], k[2]) < kOrthoLargest) || !(q < kOrthoLargest)) return false;
  }
  return true;
}

uint64_t ortho_workspace(uint32_t count, uint64_t rows, uint64_t cols, int out_dtype) {
  return ortho_plan(count, rows, cols, out_dtype).bytes;
}

hipError_t launch_ortho(const Ortho& a, hipStream_t st) {
  const OrthoPlan plan = ortho_plan(a.count, a.rows, a.cols, a.out_dtype);
  const uint64_t ws = reinterpret_cast<uint64_t>(a.ws);
  double* const sums = reinterpret_cast<double*>(ws + plan.sums);
  float* const part = reinterpret_cast<float*>(ws + plan.part);
  const uint32_t panel = static_cast<uint32_t>(plan.m * (kPanel * 2));  // of X and of A and B: all have m rows
  const uint64_t x_plane = plan.m * plan.n * 2, a_plane = plan.m * plan.m * 2;
  for (uint32_t z0 = 0; z0 < a.count; z0 += plan.group) {
    const uint32_t count = std::min(plan.group, a.count - z0);
    OrthoIn in{};
    OrthoOut out{};
    for (uint32_t z = 0; z < count; ++z) {
      in.g[z] = a.grads[z0 + z].data;
      in.g_stride[z] = a.grads[z0 + z].stride;
      in.buf[z] = a.momenta ? a.momenta[z0 + z].data : 0;
      in.buf_stride[z] = a.momenta ? a.momenta[z0 + z].stride : 0;
      out.data[z] = a.outs[z0 + z].data;
      out.stride[z] = a.outs[z0 + z].stride;
    }
    in.rows = static_cast<uint32_t>(a.rows);
    in.cols = static_cast<uint32_t>(a.cols);
    in.mu = static_cast<float>(a.momentum);
    in.nesterov = a.nesterov;
    out.m = static_cast<uint32_t>(std::min(a.rows, a.cols));
    out.n = static_cast<uint32_t>(std::max(a.rows, a.cols));
    out.tall = plan.tall;
    out.dtype = a.out_dtype;
    const uint64_t groups = a.rows * ((a.cols + 7) / 8);
    uint32_t blocks = static_cast<uint32_t>(std::min<uint64_t>(kNormBlocks, (groups + kThreads - 1) / kThreads));
    if (LC_MAX_GRID_BLOCKS > 0 && blocks > LC_MAX_GRID_BLOCKS) blocks = LC_MAX_GRID_BLOCKS;
    hipError_t e = launch_op(a.dtype == kBf16 ? ortho_norm_kernel<kBf16> : ortho_norm_kernel<kF32>, dim3(blocks, count), kThreads, st, in, sums);
    if (e != hipSuccess) return e;
    double bound = 1.0;
    int ex = exponent_for(bound * kSlack);
    uint64_t x = ws + plan.x0, other = ws + plan.x1;
    const OrthoX ox{x, x_plane, plan.x_bytes, static_cast<uint32_t>(plan.m), static_cast<uint32_t>(plan.n), a.eps, std::ldexp(1.0, ex)};
    const dim3 load_grid(grid_for((plan.m / 64) * (plan.n / 64), kThreads), count);
    e = a.dtype == kBf16 ? load_x<kBf16>(in, ox, plan.tall, load_grid, sums, blocks, st) : load_x<kF32>(in, ox, plan.tall, load_grid, sums, blocks, st);
    if (e != hipSuccess) return e;
    for (uint32_t s = 0; s < a.steps; ++s) {
      const double* const k = a.coefs + 3 * s;
      const double bound_a = bound * bound * kSlack;
      const int ea = exponent_for(bound_a);
      OrthoProduct p{};  // A = X X^T
      p.left = p.right = x;
      p.left_plane = p.right_plane = x_plane;
      p.left_next = p.right_next = plan.x_bytes;
      p.left_panel = p.right_panel = p.out_panel = panel;
      p.out = ws + plan.a;
      p.out_plane = a_plane;
      p.out_next = plan.a_bytes;
      p.rows = p.cols = static_cast<uint32_t>(plan.m);
      p.k = static_cast<uint32_t>(plan.n);
      p.count = count;
      p.part = part;
      p.f_acc = static_cast<float>(std::ldexp(1.0, ea - 2 * ex));
      if ((e = product<kSym>(p, out, plan.gram, plan.planes, st)) != hipSuccess) return e;
      uint64_t left = p.out;
      int el = ea;
      double by = k[1];  // of A X; B = b A needs no product of its own
      if (k[2] != 0) {   // B = b A + c A A
        const int eb = exponent_for(ortho_bound_b(bound_a, k[1], k[2]) * kSlack);
        p.left = p.right = p.aux = ws + plan.a;
        p.left_plane = p.right_plane = a_plane;
        p.left_next = p.right_next = plan.a_bytes;
        p.out = ws + plan.b;
        p.k = static_cast<uint32_t>(plan.m);
        p.f_acc = static_cast<float>(std::ldexp(k[2], eb - 2 * ea));
        p.f_aux = static_cast<float>(std::ldexp(k[1], eb - ea));
        if ((e = product<kSym>(p, out, plan.poly, plan.planes, st)) != hipSuccess) return e;
        left = p.out;
        el = eb;
        by = 1.0;
      }
      bound = ortho_bound(bound, k) * kSlack;
      const bool last = s + 1 == a.steps;
      const int eo = last ? 0 : exponent_for(bound);
      const double scale = last ? a.scale : 1.0;
      p.left = left;  // X <- a X + B X
      p.left_plane = a_plane;
      p.left_next = plan.a_bytes;
      p.right = p.aux = x;
      p.right_plane = x_plane;
      p.right_next = plan.x_bytes;
      p.out = other;
      p.out_plane = x_plane;
      p.out_next = plan.x_bytes;
      p.cols = static_cast<uint32_t>(plan.n);
      p.k = static_cast<uint32_t>(plan.m);
      p.f_acc = static_cast<float>(std::ldexp(by * scale, eo - el - ex));
      p.f_aux = static_cast<float>(std::ldexp(k[0] * scale, eo - ex));
      e = last ? product<kLast>(p, out, plan.mid, plan.planes, st) : product<kMid>(p, out, plan.mid, plan.planes, st);
      if (e != hipSuccess) return e;
      std::swap(x, other);
      ex = eo;
    }
  }
  return hipSuccess;
}

}  // namespace lc
