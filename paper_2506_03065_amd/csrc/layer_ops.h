// Launch interface of the operators around the attention of a layer: residual update and norms, rotary positions,
// block-scaled FP8 products.  Arguments are validated by the entry points (layer_api.cpp); strides are in elements.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "layer_index.h"
#include "sparse_vdit.h"

namespace svd {

struct RowsView {
  void* data;   // nullptr: absent
  int64_t stride_b, stride_l;
};

// ---- residual update and norms ----

struct NormLaunch {
  RowChunks ch;
  int B, C;
  int stream_type, norm, post_norm;
  float eps;
  int64_t mod_stride_b, mod_stride_g;
  svd_norm_vectors vec;
  RowsView x, y, x_out, h;   // backward: x_out is read
  uint8_t* h_scales;         // not nullptr: h is E4M3
  int64_t h_scale_stride;
  RowsView dh, dx_out, dx, dy;
  svd_norm_grads grads;
  float* partial;            // backward: [B * per_entry][3][C]
  float* sums;               // [B * groups][3][C], where several groups add to a weight's gradient
};
hipError_t launch_norm_forward(const NormLaunch& p, hipStream_t stream);
hipError_t launch_norm_backward(const NormLaunch& p, hipStream_t stream);

// ---- rotary positions ----

struct RopeTensor {
  const __bf16* x;      // backward: may be nullptr without a norm
  const __bf16* dout;   // backward
  __bf16* out;          // backward: dx
  int H;
  int64_t x_b, x_h, x_l, d_b, d_h, d_l, o_b, o_h, o_l;
  const float *weight, *bias;
  float *dweight, *dbias;
};
struct RopeLaunch {
  svd_rope_desc r;
  const float* table;
  int norm;
  float eps;
  int B, L, D, n;
  RopeTensor t[2];
  float* partial;   // [n][work-groups][2][D]
};
hipError_t launch_rope_table(const svd_rope_desc& r, double base, const double start[3], const double step[3], float* table,
                             hipStream_t stream);
hipError_t launch_rope_forward(const RopeLaunch& p, hipStream_t stream);
hipError_t launch_rope_backward(const RopeLaunch& p, hipStream_t stream);

// ---- block-scaled FP8 products ----

struct QuantLaunch {
  const void* src;
  int src_type, R, C;
  int64_t src_stride;
  uint8_t* dst;
  int64_t dst_stride;
  uint8_t* scales;
  int64_t scale_stride;
};
hipError_t launch_quantise_rows(const QuantLaunch& p, hipStream_t stream);
hipError_t launch_quantise_columns(const QuantLaunch& p, hipStream_t stream);

struct MatmulLaunch {
  svd_blockscale_desc d;
  const uint8_t *a, *a_scales, *b, *b_scales;
  const float* bias;
  __bf16* out;
};
hipError_t launch_blockscale_matmul(const MatmulLaunch& p, hipStream_t stream);

}  // namespace svd
