// Host-side launchers of the MXFP4 kernels (mx_quant.hip, mx_linear.hip,
// mx_sparse.hip) and of norm.hip, as si_launch.h: arguments are validated by the
// caller (mx_api.hip).
#pragma once

#include "si_launch.h"

namespace si {

hipError_t launch_quantize_mx(const void* w, int dtype, size_t rows, int n, size_t ldw, uint8_t* q, uint8_t* scale,
                              hipStream_t s);
hipError_t launch_dequantize_mx(const uint8_t* q, const uint8_t* scale, size_t rows, int n, void* w, int dtype,
                                hipStream_t s);
hipError_t launch_pack_signs_mx(const uint8_t* q_gate, int k, int d, uint32_t* signs, hipStream_t s);

// Products with MXFP4 weights: y [m][rows] from the activations and W [rows][n]
// (codes q, scales s), or ReLU(x W^T) * (x W_up^T) with q_up, s_up set.  The
// activations are fp16 or bf16 (x) or MXFP4 (xq, xs).
struct MxLinear {
  const void* x = nullptr;  // [m][ldx], x_dtype
  int x_dtype = 0;
  size_t ldx = 0;
  const uint8_t* xq = nullptr;
  const uint8_t* xs = nullptr;
  const uint8_t* q = nullptr;
  const uint8_t* s = nullptr;
  const uint8_t* q_up = nullptr;
  const uint8_t* s_up = nullptr;
  int m = 0, rows = 0, n = 0;
  void* y = nullptr;  // [m][rows], y_dtype
  int y_dtype = 0;
  bool relu = false;  // one matrix: max(y, 0)
  void* ws = nullptr;
};
// Scratch of a call: a padded copy of activations that cannot be read in whole
// 16-byte pieces, and the partial sums of products whose n is split.
size_t mx_linear_workspace(const MxLinear& c);
// Place of the call's tile in its list; -1 for the kernel of a few tokens and rows.
int mx_linear_tile(const MxLinear& c);
// Whether the call's grids stay within what a launch can hold.
bool mx_linear_fits(const MxLinear& c);
hipError_t launch_mx_linear(const MxLinear& c, hipStream_t s);

struct NormArgs {
  const void* h;
  const void* b;
  void* h_out;
  void* x;
  const float* post_w;
  const float* gate;
  const float* pre_w;
  size_t tokens, rows_per_gate;
  size_t ldh, ldb, ldo, ldx;  // row strides in elements
  int d;
  int h_dtype, b_dtype, x_dtype;
  float scale, eps;
};
hipError_t launch_norm_residual(const NormArgs& a, hipStream_t s);

// The sparse MLP with MXFP4 weights (rows from the packed signs, or from
// mask_in when signs is NULL).
struct MxMlpCall {
  const uint32_t* signs = nullptr;
  const uint8_t* q_gate = nullptr;
  const uint8_t* s_gate = nullptr;
  const uint8_t* q_up = nullptr;
  const uint8_t* s_up = nullptr;
  const uint8_t* q_down_t = nullptr;
  const uint8_t* s_down_t = nullptr;
  const uint16_t* x = nullptr;
  const uint8_t* mask_in = nullptr;
  int k = 0, d = 0, b = 1, T = 0, margin = 0;
  uint32_t flags = 0;
  uint8_t* mask = nullptr;
  int32_t* idx = nullptr;
  int32_t* n_out = nullptr;
  float* y = nullptr;
  void* ws = nullptr;
  int32_t* counters = nullptr;
};
hipError_t launch_mx_mlp(const MxMlpCall& c, hipStream_t s);

}  // namespace si
