// Rows and blocks of 8-bit floating point values (e4m3: 4 bits of exponent, 3 of
// fraction, largest value 448, no infinities) with float32 scales:
//     scale = max |v| * (1 / 448) over a block,  code = the nearest e4m3 of v / scale
// with 1 / 448, the product and the quotient rounded to float32 each, ties to the even
// code (the product, as PyTorch divides a tensor by a number on the GPU: a scale that is
// one step off puts values at the border between two codes on the other side).  Tokens have a
// scale for each 128 values of a row, weights one for each 128 x 128 block.  Rows
// are stored as n rounded up to 16 codes (zeros behind the n-th), so that a row's
// codes are whole 16-byte pieces.  A block of zeros has scale 0 and codes 0; one
// with an infinity or a NaN scale NaN and codes 0, so that it reads back as NaN.
//
// Bound by memory: values are read once and held until their block's scale is known
// (tokens, 4096 x 5120 bf16: 17.3 to 19.3 us, 3.5 TB/s, one request of 16 bytes a thread; one
// token a launch, 2.8; weights, 11008 x 4096 fp16: 34.8 us, 3.9 TB/s; back to fp16 21.7).
#include "dense.h"
#include "layer_common.h"

namespace si {

// 8 values of a row from value c on, as float; zeros behind the n-th.
__device__ inline void load8(const void* p, size_t base, int dt, int c, int n, bool vec, float (&f)[8]) {
  if (vec && c + 8 <= n) {
    if (dt == kF32) {
      const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + base + c);
      const u32x4 a = q[0], b = q[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = __uint_as_float(a[e]);
        f[4 + e] = __uint_as_float(b[e]);
      }
    } else {
      const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + base + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[2 * e] = dt == kF16 ? (float)as_h2(v[e]).x : bf16_lo(v[e]);
        f[2 * e + 1] = dt == kF16 ? (float)as_h2(v[e]).y : bf16_hi(v[e]);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = c + e < n ? load_one(p, base + c + e, dt) : 0.f;
  }
}

// The bits of |v| are ordered as |v| is, infinities and then NaN above all.
__device__ inline uint32_t top_bits(const float (&f)[8], uint32_t top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
  return top;
}

__device__ inline float scale_of(uint32_t top) {
  return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float(top) * (1.f / 448.f);
}

__device__ inline u32x2 codes_of(const float (&f)[8], float scale) {
  uint32_t c[2] = {0, 0};
  if (scale > 0.f) {
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = fminf(fmaxf(__fdiv_rn(f[e], scale), -448.f), 448.f);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h], q[4 * h + 1], 0, false);
      v = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h + 2], q[4 * h + 3], v, true);
      c[h] = (uint32_t)v;
    }
  }
  return u32x2{c[0], c[1]};
}

// 16 threads a block of 128 values.
__global__ __launch_bounds__(256) void k_quantize_rows_fp8(const void* __restrict__ x, int dt, size_t ld, size_t rows,
                                                           int n, bool vec, uint8_t* __restrict__ q,
                                                           float* __restrict__ scale) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int blocks = fp8_blocks(n), np = fp8_padded(n);
  const size_t blk = i / 16;
  if (blk >= rows * (size_t)blocks) return;  // whole groups of 16 lanes
  const size_t r = blk / blocks;
  const int b = (int)(blk - r * blocks), c = b * 128 + (int)(i & 15) * 8;
  float f[8];
  load8(x, r * ld, dt, c, n, vec, f);
  uint32_t top = top_bits(f, 0u);
#pragma unroll
  for (int m = 8; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m, 16));
  const float s = scale_of(top);
  if (c < np) *reinterpret_cast<u32x2*>(q + r * np + c) = codes_of(f, s);
  if ((i & 15) == 0) scale[blk] = s;
}

// A block of 256 threads a block of 128 x 128: thread (row, piece) has 8 values of
// every 16th row.
__global__ __launch_bounds__(256) void k_quantize_blocks_fp8(const void* __restrict__ w, int dt, size_t ld, int rows,
                                                             int n, bool vec, uint8_t* __restrict__ q,
                                                             float* __restrict__ scale) {
  __shared__ uint32_t tops[4];
  const int blocks = fp8_blocks(n), np = fp8_padded(n);
  const int rb = blockIdx.x / blocks, b = blockIdx.x - rb * blocks;
  const int c = b * 128 + (threadIdx.x & 15) * 8, r0 = rb * 128 + (threadIdx.x >> 4);
  float f[8][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    load8(w, (size_t)min(r, rows - 1) * ld, dt, c, r < rows ? n : 0, vec, f[i]);
    top = top_bits(f[i], top);
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m, kWave));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  const float s = scale_of(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (r < rows && c < np) *reinterpret_cast<u32x2*>(q + (size_t)r * np + c) = codes_of(f[i], s);
  }
  if (threadIdx.x == 0) scale[blockIdx.x] = s;
}

// 8 values a thread; a scale serves `per` rows.
__global__ __launch_bounds__(256) void k_dequantize_fp8(const uint8_t* __restrict__ q, const float* __restrict__ scale,
                                                        int per, size_t rows, int n, void* __restrict__ w, int dt) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int np = fp8_padded(n), pieces = np / 8;
  if (i >= rows * (size_t)pieces) return;
  const size_t r = i / pieces;
  const int c = (int)(i - r * pieces) * 8;
  if (c >= n) return;  // a row's codes behind its values
  const u32x2 v = *reinterpret_cast<const u32x2*>(q + r * np + c);
  const float s = scale[r / per * fp8_blocks(n) + c / 128];
  float f[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[h], true);
    f[4 * h] = lo.x * s;
    f[4 * h + 1] = lo.y * s;
    f[4 * h + 2] = hi.x * s;
    f[4 * h + 3] = hi.y * s;
  }
  const size_t at = r * n + c;
  if (n % 8 == 0 && dt != kF32) {
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = dt == kF16 ? pack_f2(f[2 * e], f[2 * e + 1]) : pack_bf2(f[2 * e], f[2 * e + 1]);
    *reinterpret_cast<u32x4_e2*>(static_cast<uint16_t*>(w) + at) = o;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < n) store_one(w, at + e, dt, f[e]);
  }
}

static bool whole(const void* p, size_t ld, int dt) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * dtype_bytes(dt) % 16 == 0;
}

hipError_t launch_quantize_rows_fp8(const void* x, int dtype, size_t ld, size_t rows, int n, uint8_t* q, float* scale,
                                    hipStream_t s) {
  const size_t threads = rows * fp8_blocks(n) * 16;
  k_quantize_rows_fp8<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(x, dtype, ld, rows, n, whole(x, ld, dtype), q, scale);
  return hipGetLastError();
}

hipError_t launch_quantize_blocks_fp8(const void* w, int dtype, size_t ld, int rows, int n, uint8_t* q, float* scale,
                                      hipStream_t s) {
  const size_t blocks = (size_t)((rows + 127) / 128) * fp8_blocks(n);
  k_quantize_blocks_fp8<<<(unsigned)blocks, 256, 0, s>>>(w, dtype, ld, rows, n, whole(w, ld, dtype), q, scale);
  return hipGetLastError();
}

hipError_t launch_dequantize_fp8(const uint8_t* q, const float* scale, int rows_per_scale, size_t rows, int n, void* w,
                                 int dtype, hipStream_t s) {
  const size_t threads = rows * (fp8_padded(n) / 8);
  k_dequantize_fp8<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(q, scale, rows_per_scale, rows, n, w, dtype);
  return hipGetLastError();
}

}  // namespace si
