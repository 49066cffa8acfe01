// Rows held in registers by the threads that share them, for the kernels that
// normalise rows (norm.hip, norm_train.hip): loads, stores and sums.
#pragma once

#include "layer_common.h"
#include "mx.h"

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

}  // namespace si
