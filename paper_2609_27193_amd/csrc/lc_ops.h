// Arguments and launchers of the training operators (embedding, norm, kept
// activations, linear weight gradient), shared by their entry points
// (lc_ops.cpp) and their kernels (lc_embed.hip, lc_norm.hip, lc_wgrad.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lc {

constexpr uint32_t kActBlock = 32;  // elements of a row that share a power of two

// Rows of elements in device memory; `stride` elements from one row to the next.
struct Rows {
  uint64_t data;
  uint64_t stride;
};

// A kept activation: one byte an element, one byte a block of kActBlock.
struct Kept {
  uint64_t codes;
  uint64_t scales;
  uint64_t code_stride;   // bytes from row to row
  uint64_t scale_stride;
};

struct EmbedFwd {
  Rows w, out;
  uint64_t tokens;
  uint64_t n;      // tokens
  int64_t first;   // token of the table's first row
  uint64_t vocab;  // rows of the table
  uint32_t dim;
  float scale;
  int w_dtype, out_dtype, token64;
};
hipError_t launch_embed_fwd(const EmbedFwd& a, hipStream_t st);

struct EmbedBwd {
  Rows dout, dw;
  uint64_t tokens;
  uint64_t n;
  int64_t first;
  uint64_t vocab;
  uint32_t dim;
  float scale;
  int dout_dtype, dw_dtype, token64, accumulate;
  uint8_t* ws;
};
uint64_t embed_bwd_workspace(uint64_t n, uint64_t dim);
hipError_t launch_embed_bwd(const EmbedBwd& a, hipStream_t st);

struct NormFwd {
  Rows x, y;
  Kept kept;        // codes 0: nothing is kept
  uint64_t weight;  // 0: ones
  uint64_t bias;    // 0: zeros
  float* mean;      // null: not written
  float* rstd;
  uint64_t rows;
  uint32_t dim;
  float eps;
  int dtype, param_dtype, layer;  // layer: subtract the mean
};
hipError_t launch_norm_fwd(const NormFwd& a, hipStream_t st);

struct NormBwd {
  Rows dy, x, dx;   // x.data 0: the normalised rows come from `kept`; dx.data 0: no dx
  Kept kept;
  uint64_t weight;
  const float* mean;
  const float* rstd;
  float* part;      // partial sums, null: neither dweight nor dbias
  uint64_t rows;
  uint32_t dim;
  int dtype, param_dtype, layer;
  uint64_t dweight, dbias;
  int grad_dtype, accumulate;
};
uint64_t norm_bwd_workspace(uint64_t rows, uint64_t dim);
hipError_t launch_norm_bwd(const NormBwd& a, hipStream_t st);

struct ActCopy {
  Rows x;  // the activation, read or written
  Kept kept;
  uint64_t rows;
  uint32_t dim;
  int dtype;
};
hipError_t launch_act_save(const ActCopy& a, hipStream_t st);
hipError_t launch_act_load(const ActCopy& a, hipStream_t st);

struct Wgrad {
  Rows dy, dw;
  Kept x;
  uint64_t col_scale, col_shift;  // 0: none
  uint64_t dbias;                 // 0: none
  uint64_t rows;                  // tokens
  uint32_t n, k;                  // columns of dy, of x
  int dtype, param_dtype, dw_dtype, accumulate;
  uint8_t* ws;
};
uint64_t wgrad_workspace(uint64_t rows, uint64_t n, uint64_t k);
hipError_t launch_wgrad(const Wgrad& a, hipStream_t st);

}  // namespace lc
