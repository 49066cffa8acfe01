// The dense products' arguments and tiles, shared by their kernels (dense_tile.h),
// the choice among them (dense.hip) and the C ABI (dense_api.hip).
#pragma once

#include "mx.h"
#include "si_launch.h"

namespace si {

// C[n][m] = sum over the segments of sum_k A(m, k) B(n, k); see dense_tile.h.
struct DenseArgs {
  const void* a[2];  // W and W_up of a gated product; or by segment of k, or by batch
  const void* b[2];  // by segment of k, or by batch
  size_t lda, ldb;   // bytes from row to row
  int M, N, K;       // K: of a segment
  int segs;          // 1, or 2: the sum goes on over a[1], b[1]
  void* c[2];        // [N][M] of c_dtype, by batch
  int c_dtype;
  int relu;          // one matrix: max(C, 0)
  float* g;          // gated: the two sums themselves, or NULL
  float* u;
  // The product is dh, the gradient of h = relu(gate) * up (both float32) or, up NULL, of
  // h = relu(..) (gate is h, of c_dtype): c[0] is written with dg and du with du, rows of
  // ldc values (a multiple of 8), zeros behind the M-th.
  const void* gate;
  const float* up;
  void* du;
  int ldc;
  float* part;       // partial sums [split][parts_of][N][M], or NULL
  int split, parts_of;
  const float* sa[2];  // e4m3: scales of A's blocks [M / 128][blocks] ...
  const float* sb;     // ... and of B's rows [N][blocks]
  int blocks;
  int m_tiles, n_tiles;
};

// Tiles by size: values along m (both matrices of a gated product) and n, planes of
// a stage.  The first two are for few rows of B, which then lie along k.
struct DenseShape {
  int bm, bn, wk, threads, st;  // st: stages in LDS
  int resident;                 // blocks a compute unit
  // Weights of a stage, and of what a round of blocks takes besides, in the estimate that
  // ranks tiles and splits (plan_of).  They are fitted to the ranking: a measured stage
  // takes 1.3 to 2.1 times as long.
  float stage_us, round_us;
};
constexpr DenseShape kDenseTiles[] = {{64, 16, 4, 512, 3, 1, 0.69f, 0.7f},  {64, 32, 4, 512, 3, 1, 0.93f, 0.9f},
                                      {64, 64, 2, 512, 3, 1, 0.59f, 2.0f},  {128, 128, 1, 512, 2, 2, 0.76f, 2.0f},
                                      {128, 256, 1, 512, 3, 1, 0.71f, 2.4f}, {256, 256, 1, 512, 2, 1, 1.03f, 6.0f}};
constexpr int kDenseTileCount = 6;
constexpr int kDenseFew = 100;  // in place of a tile: the kernel for up to kFewTokens rows of B (dense_few.hip)
constexpr int kFewTokens = 4;

// Instances (dense_*.hip): value type, layouts of A and B, matrices.
hipError_t dense_rr(int type, const DenseArgs& a, int tile, hipStream_t s);                 // x W^T
hipError_t dense_gated(int type, const DenseArgs& a, int tile, hipStream_t s);              // x W_gate^T, x W_up^T
hipError_t dense_cr(int type, const DenseArgs& a, int tile, hipStream_t s);                 // dy W
hipError_t dense_dh(int type, const DenseArgs& a, int tile, hipStream_t s);                 // the same, to dg and du
hipError_t dense_cc(int type, const DenseArgs& a, int tile, int batches, hipStream_t s);    // dy^T x
hipError_t dense_fp8(const DenseArgs& a, int mats, int tile, hipStream_t s);
hipError_t dense_few(int type, int mats, const DenseArgs& a, hipStream_t s);                // x W^T, a few tokens; type 2: e4m3

// dg and du of one value: the gradient is 0 where the gate is <= 0; a NaN gate lets it
// pass.
__device__ inline void gated_grad(float dh, float gate, float up, float& dg, float& du) {
  dg = gate <= 0.f ? 0.f : dh * up;
  du = dh * (gate <= 0.f ? 0.f : gate);
}

// What dg and du of four values, row n from m on (a multiple of 4), ask for.  UP: both
// sums are kept; else gate is h.  WHOLE: M is a multiple of 4.  Zeros behind the M-th.
struct GatedPiece {
  f32x4 g, u;
};
template <bool UP, bool WHOLE>
__device__ inline GatedPiece gated_piece(const DenseArgs& a, int n, int m) {
  const size_t at = (size_t)n * a.M + m;
  GatedPiece p = {{0.f, 0.f, 0.f, 0.f}, {1.f, 1.f, 1.f, 1.f}};
  if constexpr (WHOLE) {
    if (m >= a.M) return p;
    if constexpr (UP) {
      p.g = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.gate) + at);
      p.u = *reinterpret_cast<const f32x4*>(a.up + at);
    } else {
      const u32x2 h = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(a.gate) + at);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t v = h[e >> 1] >> (16 * (e & 1));
        p.g[e] = a.c_dtype == kBF16 ? bf16_lo(v) : (float)__builtin_bit_cast(_Float16, (uint16_t)v);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (m + e < a.M) {
        p.g[e] = load_one(a.gate, at + e, UP ? kF32 : a.c_dtype);
        if constexpr (UP) p.u[e] = a.up[at + e];
      }
  }
  return p;
}

// dg (x, y) and du (z, w) of four values from m on, rounded; zeros behind the M-th.
__device__ inline u32x4 gated_grads(const DenseArgs& a, int m, f32x4 dh, const GatedPiece& p) {
  float x[4], y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    gated_grad(dh[e], p.g[e], p.u[e], x[e], y[e]);
    if (m + e >= a.M) x[e] = y[e] = 0.f;
  }
  auto pack = [&](float v, float w) { return a.c_dtype == kBF16 ? pack_bf2(v, w) : pack_f2(v, w); };
  return u32x4{pack(x[0], x[1]), pack(x[2], x[3]), pack(y[0], y[1]), pack(y[2], y[3])};
}

// They in their place.
template <bool UP>
__device__ inline void put_gated_grad(const DenseArgs& a, int n, int m, f32x4 dh, const GatedPiece& p) {
  const size_t at = (size_t)n * a.ldc + m;
  const u32x4 v = gated_grads(a, m, dh, p);
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.c[0]) + at) = u32x2{v.x, v.y};
  if constexpr (UP) *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.du) + at) = u32x2{v.z, v.w};
}

// ---- calls (dense.hip), arguments validated by the caller ----------------------

// A matrix of a call: rows of n values of type dtype, ld elements apart.
struct DenseMat {
  const void* p = nullptr;
  int dtype = 0;
  size_t ld = 0;
};

// y = x W^T, relu'd or gated: W [rows][n], or [n][rows] when transposed.
struct DenseLinear {
  DenseMat x, w, w_up;
  int type = 0;  // kF16 or kBF16: the type of the products
  bool transposed = false, relu = false;
  int m = 0, rows = 0, n = 0;
  void* y = nullptr;
  int y_dtype = 0;
  float* g = nullptr;
  float* u = nullptr;
  void* ws = nullptr;
};
size_t dense_linear_workspace(const DenseLinear& c);
int dense_linear_tile(const DenseLinear& c);  // place of its tile; -1: more than one launch can hold
hipError_t launch_dense_linear(const DenseLinear& c, hipStream_t s);

// Gradients of DenseLinear.  gate NULL: of y = x W^T (dy); else of the ReLU'd or
// gated product, whose sums (one matrix: outputs) were kept.  down given: of the whole
// MLP, whose hidden values h were kept; dy is then that of y = h W_down^T, [m][n].
struct DenseGrad {
  DenseMat dy, x, w, w_up;
  DenseMat gate, up;
  DenseMat down, h;  // W_down [n][rows], h [m][rows]
  int type = 0;
  bool transposed = false;
  int m = 0, rows = 0, n = 0;
  void* dx = nullptr;
  void* dw = nullptr;
  void* dw_up = nullptr;
  void* dw_down = nullptr;
  void* ws = nullptr;
};
size_t dense_grad_workspace(const DenseGrad& c);
int dense_dx_tile(const DenseGrad& c);
int dense_dh_tile(const DenseGrad& c);
int dense_dw_down_tile(const DenseGrad& c);
int dense_dw_tile(const DenseGrad& c);
hipError_t launch_dense_grad(const DenseGrad& c, hipStream_t s);

// Products of e4m3 values with block scales.
struct DenseFp8 {
  const uint8_t* xq = nullptr;
  const float* xs = nullptr;
  const uint8_t* q = nullptr;
  const float* s = nullptr;
  const uint8_t* q_up = nullptr;
  const float* s_up = nullptr;
  int m = 0, rows = 0, n = 0;
  void* y = nullptr;
  int y_dtype = 0;
  bool relu = false;
  void* ws = nullptr;
};
size_t dense_fp8_workspace(const DenseFp8& c);
int dense_fp8_tile(const DenseFp8& c);
hipError_t launch_dense_fp8(const DenseFp8& c, hipStream_t s);
__host__ __device__ inline int fp8_padded(int n) { return (n + 15) / 16 * 16; }
__host__ __device__ inline int fp8_blocks(int n) { return (n + 127) / 128; }

// ---- e4m3 rows and blocks (fp8.hip) ------------------------------------------------
hipError_t launch_quantize_rows_fp8(const void* x, int dtype, size_t ld, size_t rows, int n, uint8_t* q, float* scale,
                                    hipStream_t s);
hipError_t launch_quantize_blocks_fp8(const void* w, int dtype, size_t ld, int rows, int n, uint8_t* q, float* scale,
                                      hipStream_t s);
hipError_t launch_dequantize_fp8(const uint8_t* q, const float* scale, int rows_per_scale, size_t rows, int n, void* w,
                                 int dtype, hipStream_t s);

// ---- LayerNorm and RMSNorm (norm_train.hip) ------------------------------------------
struct LayerNormArgs {
  const void* x;
  size_t ldx;
  int dtype;          // of x, y, dy and dx
  const void* w;
  const void* b;
  int w_dtype;        // of w, b and their gradients
  void* y;            // [tokens][d]
  float* mean;        // [tokens], or NULL
  float* rstd;
  size_t tokens;
  int d, center;      // center: LayerNorm
  float eps;
};
hipError_t launch_layer_norm(const LayerNormArgs& a, hipStream_t s);
struct LayerNormGrad {
  const void* dy;
  size_t ldy;
  const void* x;
  size_t ldx;
  int dtype;
  const void* w;
  int w_dtype;
  const float* mean;
  const float* rstd;
  void* dx;           // [tokens][d], or NULL
  void* dw;           // [d], or NULL
  void* db;
  size_t tokens;
  int d, center;
  float* part;        // workspace
};
size_t layer_norm_grad_workspace(size_t tokens, int d);
hipError_t launch_layer_norm_grad(const LayerNormGrad& a, hipStream_t s);

}  // namespace si
