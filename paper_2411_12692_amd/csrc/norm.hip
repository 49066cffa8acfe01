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
#include "layer_common.h"
#include "mx.h"
#include "mx_launch.h"

namespace si {

// 8 values as they lie in memory (the second half used by float alone): the
// loads of h and b are issued before either is converted.
struct Raw8 {
  u32x4 a, b;
};

// VEC: piece p of a row is its values 8 p .. 8 p + 7, whole (d, strides and
// addresses allow 16-byte requests).  Otherwise value e of a thread's piece u is
// row value i = t + gt (8 u + e), so that neighbouring lanes read neighbouring
// values of rows that start anywhere.
template <bool VEC>
__device__ inline int index_of(int t, int gt, int u, int e) {
  return VEC ? (t + gt * u) * 8 + e : t + gt * (8 * u + e);
}

template <bool VEC>
__device__ inline Raw8 load_raw(const void* p, size_t base, int dt, int t, int gt, int u, int d) {
  Raw8 r = {u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
  if constexpr (VEC) {
    const int i = (t + gt * u) * 8;
    if (i < d) {
      if (dt == kF32) {
        const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + base + i);
        r.a = q[0];
        r.b = q[1];
      } else {
        r.a = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + base + i);
      }
    }
  } else {
    if (dt == kF32) {
      const float* q = static_cast<const float*>(p) + base;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = index_of<VEC>(t, gt, u, e), j = index_of<VEC>(t, gt, u, 4 + e);
        if (i < d) r.a[e] = __float_as_uint(q[i]);
        if (j < d) r.b[e] = __float_as_uint(q[j]);
      }
    } else {
      const uint16_t* q = static_cast<const uint16_t*>(p) + base;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = index_of<VEC>(t, gt, u, 2 * e), j = index_of<VEC>(t, gt, u, 2 * e + 1);
        uint32_t v = i < d ? q[i] : 0u;
        if (j < d) v |= (uint32_t)q[j] << 16;
        r.a[e] = v;
      }
    }
  }
  return r;
}

__device__ inline void to_floats(const Raw8& r, int dt, float (&f)[8]) {
  if (dt == kF32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[e] = __uint_as_float(r.a[e]);
      f[4 + e] = __uint_as_float(r.b[e]);
    }
  } else if (dt == kBF16) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = bf16_lo(r.a[e]);
      f[2 * e + 1] = bf16_hi(r.a[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = (float)as_h2(r.a[e]).x;
      f[2 * e + 1] = (float)as_h2(r.a[e]).y;
    }
  }
}

template <bool VEC>
__device__ inline void store8(void* p, size_t base, int dt, int t, int gt, int u, int d, const float (&f)[8]) {
  if constexpr (VEC) {
    const int i = (t + gt * u) * 8;
    if (i >= d) return;
    if (dt == kF32) {
      f32x4* q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + base + i);
      q[0] = f32x4{f[0], f[1], f[2], f[3]};
      q[1] = f32x4{f[4], f[5], f[6], f[7]};
    } else if (dt == kBF16) {
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + base + i) =
          u32x4{pack_bf2(f[0], f[1]), pack_bf2(f[2], f[3]), pack_bf2(f[4], f[5]), pack_bf2(f[6], f[7])};
    } else {
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + base + i) =
          u32x4{pack_f2(f[0], f[1]), pack_f2(f[2], f[3]), pack_f2(f[4], f[5]), pack_f2(f[6], f[7])};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = index_of<VEC>(t, gt, u, e);
      if (i < d) store_one(p, base + i, dt, f[e]);
    }
  }
}

// Sum over the threads of a row: one wave (WAVE) or the block.
template <bool WAVE>
__device__ inline float row_sum(float v, float* part) {
  v = wave_total(v);
  if constexpr (!WAVE) {
    __syncthreads();  // the last sum's readers are done
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < (int)(blockDim.x / kWave); ++w) v += part[w];
  }
  return v;
}

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
