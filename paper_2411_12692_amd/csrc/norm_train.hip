// LayerNorm and RMSNorm with their gradients.  For a row x of d values:
//     c = x - mean(x) (LayerNorm) or x,  r = 1 / sqrt(mean(c^2) + eps),  n = c r
//     y = n w + b
// and for a gradient dy, with e = dy w:
//     dx = r (e - mean(e) - n mean(e n))     (mean(e) for LayerNorm alone)
//     dw = sum over rows of dy n,  db = sum over rows of dy
// all in float32; the mean and r of each row are kept between the two passes.
//
// Bound by memory.  A row is read once and stays in registers between its sums (the
// variance is taken of c, after the mean).  In the backward pass a thread owns the
// same columns of every row of its block, so the columns' sums stay in registers
// over the block's rows and are written once a block; k_norm_columns adds the
// blocks' sums in their order, so that the gradients are the same bits in every run.
// Measured at 4096 x 5120, bf16: forward 19.6 us (4.3 TB/s), backward 38 to 40 (3.7 TB/s,
// 21 MB of blocks' sums among its bytes; 256, 768 and 1024 blocks: 37.5, 42, 44 us, and
// 15.2, 14, 15.4 where 512 take 13.4, at 1999 x 4096 without a bias) and 4.3 for the
// columns; a token of 4096 2.7.
#include <algorithm>

#include "dense.h"
#include "norm_rows.h"

namespace si {

constexpr int kLnThreads = 512;

// gt threads take a row, U pieces of 8 values each: a wave (four rows a block), or
// the block.
template <bool VEC, bool WAVE, int U>
__global__ __launch_bounds__(WAVE ? 256 : kLnThreads) void k_layer_norm(LayerNormArgs a) {
  __shared__ float part[kLnThreads / kWave];
  const int gt = WAVE ? kWave : (int)blockDim.x;
  const int t = WAVE ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const size_t row = WAVE ? (size_t)blockIdx.x * 4 + threadIdx.x / kWave : blockIdx.x;
  if (WAVE && row >= a.tokens) return;  // whole waves, which meet no barrier
  const int d = a.d;
  Raw8 xr[U];
#pragma unroll
  for (int u = 0; u < U; ++u) xr[u] = load_raw<VEC>(a.x, row * a.ldx, a.dtype, t, gt, u, d);
  float x[U][8], mean = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) to_floats(xr[u], a.dtype, x[u]);
  if (a.center) {
    float s = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += x[u][e];
    mean = row_sum<WAVE>(s, part) / (float)d;
  }
  float ss = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[u][e] -= mean;
      if (index_of<VEC>(t, gt, u, e) < d) ss = fmaf(x[u][e], x[u][e], ss);
    }
  const float r = 1.0f / sqrtf(row_sum<WAVE>(ss, part) / (float)d + a.eps);
  if (t == 0 && a.rstd) {
    if (a.center) a.mean[row] = mean;
    a.rstd[row] = r;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float w[8], b[8];
    to_floats(load_raw<VEC>(a.w, 0, a.w_dtype, t, gt, u, d), a.w_dtype, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[u][e] = x[u][e] * r * w[e];
    if (a.b) {
      to_floats(load_raw<VEC>(a.b, 0, a.w_dtype, t, gt, u, d), a.w_dtype, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] += b[e];
    }
    store8<VEC>(a.y, row * (size_t)d, a.dtype, t, gt, u, d, x[u]);
  }
}

// Sums of N values over the threads of a row.
template <bool WAVE, int N>
__device__ inline void row_sums(float (&v)[N], float (*part)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_total(v[i]);
  if constexpr (!WAVE) {
    __syncthreads();  // the last sums' readers are done
    if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) part[threadIdx.x / kWave][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    for (int w = 0; w < (int)(blockDim.x / kWave); ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += part[w][i];
  }
}

// A row at a time, the requests of the block's next row in flight meanwhile.  (Two rows
// ahead, or two at a time with shared barriers: no faster.)
template <bool VEC, bool WAVE, int U>
__global__ __launch_bounds__(WAVE ? 256 : kLnThreads) void k_layer_norm_grad(LayerNormGrad a) {
  __shared__ float part[kLnThreads / kWave][2];
  __shared__ float cols[WAVE ? 4 : 1][2][WAVE ? 512 : 1];
  const int gt = WAVE ? kWave : (int)blockDim.x;
  const int t = WAVE ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const int d = a.d;
  const size_t first = WAVE ? (size_t)blockIdx.x * 4 + threadIdx.x / kWave : blockIdx.x;
  const size_t stride = WAVE ? (size_t)gridDim.x * 4 : gridDim.x;
  float w[U][8], dw[U][8], db[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    to_floats(load_raw<VEC>(a.w, 0, a.w_dtype, t, gt, u, d), a.w_dtype, w[u]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[u][e] = db[u][e] = 0.f;
  }
  struct Row {
    Raw8 x[U], g[U];
    float mean, r;
  };
  auto load = [&](size_t row, Row& q) {
    if (row >= a.tokens) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      q.x[u] = load_raw<VEC>(a.x, row * a.ldx, a.dtype, t, gt, u, d);
      q.g[u] = load_raw<VEC>(a.dy, row * a.ldy, a.dtype, t, gt, u, d);
    }
    q.mean = a.center ? a.mean[row] : 0.f;
    q.r = a.rstd[row];
  };
  auto take = [&](size_t row, Row& q) {
    float n[U][8], g[U][8], sums[2] = {0.f, 0.f};
    const float mean = q.mean, r = q.r;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      to_floats(q.x[u], a.dtype, n[u]);
      to_floats(q.g[u], a.dtype, g[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[u][e] = (n[u][e] - mean) * r;
        dw[u][e] = fmaf(g[u][e], n[u][e], dw[u][e]);
        db[u][e] += g[u][e];
        g[u][e] *= w[u][e];
        if (index_of<VEC>(t, gt, u, e) < d) {
          sums[0] += g[u][e];
          sums[1] = fmaf(g[u][e], n[u][e], sums[1]);
        }
      }
    }
    load(row + stride, q);
    if (!a.dx) return;
    row_sums<WAVE>(sums, part);
    const float me = a.center ? sums[0] / (float)d : 0.f, mn = sums[1] / (float)d;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[u][e] = (g[u][e] - me - n[u][e] * mn) * r;
      store8<VEC>(a.dx, row * (size_t)d, a.dtype, t, gt, u, d, g[u]);
    }
  };
  Row q;
  load(first, q);
  for (size_t row = first; row < a.tokens; row += stride) take(row, q);
  if (!a.part) return;
  // [block][dw, db][d]
  float* out = a.part + (size_t)blockIdx.x * 2 * d;
  if constexpr (WAVE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = index_of<VEC>(t, gt, 0, e);
      cols[threadIdx.x / kWave][0][i] = dw[0][e];
      cols[threadIdx.x / kWave][1][i] = db[0][e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (a.db ? 2 : 1) * d; i += 256) {
      const int k = i >= d, c = i - k * d;
      out[i] = (cols[0][k][c] + cols[1][k][c]) + (cols[2][k][c] + cols[3][k][c]);
    }
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      store8<VEC>(out, 0, kF32, t, gt, u, d, dw[u]);
      if (a.db) store8<VEC>(out, (size_t)d, kF32, t, gt, u, d, db[u]);
    }
  }
}

// The blocks' column sums, added in a fixed order: 64 columns a block, its 16 waves
// take every 16th block's sums each.
__global__ __launch_bounds__(1024) void k_norm_columns(const float* __restrict__ part, int blocks, int d,
                                                       void* __restrict__ dw, void* __restrict__ db, int dt) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, k = blockIdx.y;
  void* out = k ? db : dw;
  if (!out) return;
  const int c = blockIdx.x * 64 + lane;
  float v = 0.f;
  if (c < d) {
    const float* p = part + (size_t)k * d + c;
    int b = wv;
    for (; b + 7 * 16 < blocks; b += 8 * 16) {  // eight requests at once
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = p[(size_t)(b + 16 * e) * 2 * d];
#pragma unroll
      for (int e = 0; e < 8; ++e) v += f[e];
    }
    for (; b < blocks; b += 16) v += p[(size_t)b * 2 * d];
  }
  s[wv][lane] = v;
  __syncthreads();
  if (wv == 0 && c < d) {
#pragma unroll
    for (int w = 1; w < 16; ++w) v += s[w][lane];
    store_one(out, c, dt, v);
  }
}

namespace {

struct Shape {
  bool wave;
  int u;
  unsigned threads;
};
// a wave a row up to 512 values; else as many pieces a thread as 512 threads need,
// then no more threads than that takes
Shape shape_of(int d) {
  const int pieces = (d + 7) / 8;
  if (pieces <= kWave) return {true, 1, 256};
  const int u = (pieces + kLnThreads - 1) / kLnThreads, per = u <= 1 ? 1 : u <= 2 ? 2 : 4;
  return {false, per, (unsigned)((pieces + per - 1) / per + kWave - 1) / kWave * kWave};
}

bool whole(const void* p, size_t ld, int dt) {
  return !p || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * dtype_bytes(dt) % 16 == 0);
}

// Blocks of the backward pass: two a compute unit, so that the blocks' sums, 8 d
// bytes each, stay few (4096 x 5120 bf16, both kernels: 45 us with 512 blocks, 49 with
// 768, 54 with 1024); no more than rows.
unsigned grad_blocks(size_t tokens, int d) {
  const size_t rows = shape_of(d).wave ? 4 : 1;
  return (unsigned)std::min<size_t>((tokens + rows - 1) / rows, 512);
}

}  // namespace

#define SI_LN(KERNEL, ...)                                                       \
  do {                                                                           \
    if (sh.wave) KERNEL<V, true, 1><<<__VA_ARGS__, sh.threads, 0, s>>>(a);       \
    else if (sh.u == 1) KERNEL<V, false, 1><<<__VA_ARGS__, sh.threads, 0, s>>>(a); \
    else if (sh.u == 2) KERNEL<V, false, 2><<<__VA_ARGS__, sh.threads, 0, s>>>(a); \
    else KERNEL<V, false, 4><<<__VA_ARGS__, sh.threads, 0, s>>>(a);              \
  } while (0)

template <bool V>
static hipError_t forward(const LayerNormArgs& a, const Shape& sh, hipStream_t s) {
  const unsigned grid = (unsigned)(sh.wave ? (a.tokens + 3) / 4 : a.tokens);
  SI_LN(k_layer_norm, grid);
  return hipGetLastError();
}

hipError_t launch_layer_norm(const LayerNormArgs& a, hipStream_t s) {
  const bool vec = a.d % 8 == 0 && whole(a.x, a.ldx, a.dtype) && whole(a.y, a.d, a.dtype) && whole(a.w, 0, a.w_dtype) &&
                   whole(a.b, 0, a.w_dtype);
  return vec ? forward<true>(a, shape_of(a.d), s) : forward<false>(a, shape_of(a.d), s);
}

size_t layer_norm_grad_workspace(size_t tokens, int d) { return (size_t)grad_blocks(tokens, d) * 2 * d * sizeof(float); }

template <bool V>
static hipError_t backward(const LayerNormGrad& a, const Shape& sh, unsigned grid, hipStream_t s) {
  SI_LN(k_layer_norm_grad, grid);
  return hipGetLastError();
}

hipError_t launch_layer_norm_grad(const LayerNormGrad& a, hipStream_t s) {
  const unsigned blocks = grad_blocks(a.tokens, a.d);
  if (blocks > 0) {
    const bool vec = a.d % 8 == 0 && whole(a.x, a.ldx, a.dtype) && whole(a.dy, a.ldy, a.dtype) &&
                     whole(a.dx, a.d, a.dtype) && whole(a.w, 0, a.w_dtype);
    const hipError_t e = vec ? backward<true>(a, shape_of(a.d), blocks, s) : backward<false>(a, shape_of(a.d), blocks, s);
    if (e != hipSuccess) return e;
  }
  if (!a.dw && !a.db) return hipSuccess;
  k_norm_columns<<<dim3((unsigned)(a.d + 63) / 64, a.db ? 2 : 1), 1024, 0, s>>>(a.part, (int)blocks, a.d, a.dw, a.db,
                                                                                a.w_dtype);
  return hipGetLastError();
}

}  // namespace si
