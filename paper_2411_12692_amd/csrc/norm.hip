// What stands between the products of two decoder blocks, in one pass:
//     h' = h + s * g (.) P(b)      P(b) = RMSNorm(b) * post_w, or b itself
//     x  = RMSNorm(h') * pre_w     RMSNorm(v) = v / sqrt(mean(v^2) + eps)
// b is a block's output (the MLP's y), g a gate by channel, shared by runs of
// tokens or one for each, s the residual scale; every part but h is optional.
//
// Bound by memory: h and b are read once and stay in registers as float between
// the two reductions, h' and x are written once; x is formed from the unrounded
// h'.  A row's requests are all in flight before the first sum.
// (4096 x 5120 bf16 with both norms and a gate: 39 us, 168 MB = 4.3 TB/s; with 512
// threads a row, a third of them idle, 4 us more.  Rows that do not start on 16
// bytes go value by value: 4096 x 5119, 91 us.  One token of 4096: 3.3 us.)
#include "mx_launch.h"
#include "norm_rows.h"

namespace si {

constexpr int kNormThreads = 512;

// gt threads take a row, U pieces of 8 values each: a wave (four rows a block), or
// the block.
template <bool VEC, bool WAVE, int U>
__global__ __launch_bounds__(WAVE ? 256 : kNormThreads) void k_norm_residual(NormArgs a) {
  __shared__ float part[kNormThreads / kWave];
  const int gt = WAVE ? kWave : (int)blockDim.x;
  const int t = WAVE ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const size_t row = WAVE ? (size_t)blockIdx.x * 4 + threadIdx.x / kWave : blockIdx.x;
  if (WAVE && row >= a.tokens) return;  // whole waves, which meet no barrier
  const int d = a.d;
  Raw8 hr[U], br[U];
#pragma unroll
  for (int u = 0; u < U; ++u) hr[u] = load_raw<VEC>(a.h, row * a.ldh, a.h_dtype, t, gt, u, d);
  float h[U][8];
  if (a.b) {
#pragma unroll
    for (int u = 0; u < U; ++u) br[u] = load_raw<VEC>(a.b, row * a.ldb, a.b_dtype, t, gt, u, d);
    float rs = 1.f;
    if (a.post_w) {
      float ss = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float f[8];
        to_floats(br[u], a.b_dtype, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
      }
      rs = 1.0f / sqrtf(row_sum<WAVE>(ss, part) / (float)d + a.eps);
    }
    const size_t grow = a.gate ? row / a.rows_per_gate : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[8], m[8];
      to_floats(br[u], a.b_dtype, f);
      if (a.post_w) {
        to_floats(load_raw<VEC>(a.post_w, 0, kF32, t, gt, u, d), kF32, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = f[e] * rs * m[e];
      }
      if (a.gate) {
        to_floats(load_raw<VEC>(a.gate, grow * (size_t)d, kF32, t, gt, u, d), kF32, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= m[e];
      }
      to_floats(hr[u], a.h_dtype, h[u]);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[u][e] = fmaf(a.scale, f[e], h[u][e]);
    }
    if (a.h_out) {
#pragma unroll
      for (int u = 0; u < U; ++u) store8<VEC>(a.h_out, row * a.ldo, a.h_dtype, t, gt, u, d, h[u]);
    }
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u) to_floats(hr[u], a.h_dtype, h[u]);
  }
  if (!a.x) return;
  float ss = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (index_of<VEC>(t, gt, u, e) < d) ss = fmaf(h[u][e], h[u][e], ss);
  const float rs = 1.0f / sqrtf(row_sum<WAVE>(ss, part) / (float)d + a.eps);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float m[8];
    to_floats(load_raw<VEC>(a.pre_w, 0, kF32, t, gt, u, d), kF32, m);
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] *= h[u][e] * rs;
    store8<VEC>(a.x, row * a.ldx, a.x_dtype, t, gt, u, d, m);
  }
}

template <bool VEC>
static hipError_t norm_shape(const NormArgs& a, hipStream_t s) {
  const int pieces = (a.d + 7) / 8;
  if (pieces <= kWave) {
    k_norm_residual<VEC, true, 1><<<(unsigned)((a.tokens + 3) / 4), 256, 0, s>>>(a);
    return hipGetLastError();
  }
  // as many pieces a thread as 512 threads need, then no more threads than that
  // takes (5120 values: 320 threads of 2 pieces)
  const int u = (pieces + kNormThreads - 1) / kNormThreads;
  const int per = u <= 1 ? 1 : u <= 2 ? 2 : 4;
  const unsigned threads = (unsigned)((pieces + per - 1) / per + kWave - 1) / kWave * kWave;
  const unsigned grid = (unsigned)a.tokens;
  if (per == 1)
    k_norm_residual<VEC, false, 1><<<grid, threads, 0, s>>>(a);
  else if (per == 2)
    k_norm_residual<VEC, false, 2><<<grid, threads, 0, s>>>(a);
  else
    k_norm_residual<VEC, false, 4><<<grid, threads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_norm_residual(const NormArgs& a, hipStream_t s) {
  // whole 16-byte pieces: rows of a multiple of 8 values that start on 16 bytes
  bool vec = a.d % 8 == 0;
  auto check = [&](const void* p, size_t ld, int dt) {
    if (p) vec = vec && (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * dtype_bytes(dt) % 16 == 0;
  };
  check(a.h, a.ldh, a.h_dtype);
  check(a.b, a.ldb, a.b_dtype);
  check(a.h_out, a.ldo, a.h_dtype);
  check(a.x, a.ldx, a.x_dtype);
  check(a.post_w, 0, kF32);
  check(a.gate, 0, kF32);
  check(a.pre_w, 0, kF32);
  return vec ? norm_shape<true>(a, s) : norm_shape<false>(a, s);
}

}  // namespace si
