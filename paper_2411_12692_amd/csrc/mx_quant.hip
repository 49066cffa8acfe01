// Rows to MXFP4 and back, and the sign words of MXFP4 gate rows for the
// predictor (Section IV-A needs a weight's sign alone, whatever its format).
//
// A block of 32 values v with the largest magnitude m > 0 gets the scale 2^X,
// X = floor(log2 m) - 2 (m's leading bit lands on the largest code's, 4), at
// least -127, and each value the nearest code of v / 2^X, ties to the even code,
// 6 above 6; the quotient by a power of two is exact and the conversion
// instruction rounds it once, so the codes are those of the definition bit for
// bit.  A block of zeros gets the scale byte 0, one with an infinity or a NaN
// the byte 255 (every value of it reads back as NaN).  Signs are kept, those of
// zeros too.
//
// Both directions are bound by memory: nothing is read or written twice.  A
// lane takes 8 values (16 or 32 bytes of input, 4 bytes of codes), a quad of
// lanes a block, whose maximum takes two exchanges inside the quad; a thread
// takes kUnits such pieces, a block's width apart, so that all its requests are
// in flight together.  Loads are non-temporal: with cached ones 11008 x 4100 bf16
// there and back took 51.7 us instead of 44.9 (26.7 us = 4.3 TB/s to MXFP4, 18.8 us =
// 6.1 TB/s back; 2048 x 4096 fp16 7.0 and 6.1 us, where the launch counts).
#include "mx.h"
#include "mx_launch.h"

namespace si {

constexpr int kQT = 256;  // threads of a block
constexpr int kUnits = 4;  // pieces of 8 values a thread

// Where a piece of the padded rows lies: row and piece in the row.
struct Piece {
  size_t row;
  int c;
};

// The pieces of a block: blockIdx.x covers kQT * kUnits consecutive pieces of
// the padded rows, `per` of them a row.  One wide division a block (uniform),
// the rest in 32 bits.
__device__ inline Piece piece_of(uint32_t off, uint32_t per, size_t row0, uint32_t c0) {
  uint32_t c = c0 + off;  // < 2^24 / 8 + 128 + 1024
  size_t row = row0;
  if (c >= per) {
    const uint32_t q = c / per;
    row += q;
    c -= q * per;
  }
  return {row, (int)c};
}

template <int CTRL>
__device__ inline uint32_t quad_max(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true));
}

// 8 values of a row from element c8, as floats (0 past the row's end).
template <int DT>
__device__ inline void load8(const void* w, size_t base, int c8, int n, float (&f)[8]) {
  if (c8 + 8 <= n) {
    if constexpr (DT == kF32) {
      const float* p = static_cast<const float*>(w) + base + c8;
      const u32x4 a = __builtin_nontemporal_load(reinterpret_cast<const u32x4_e4*>(p));
      const u32x4 b = __builtin_nontemporal_load(reinterpret_cast<const u32x4_e4*>(p + 4));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[i] = __uint_as_float(a[i]);
        f[4 + i] = __uint_as_float(b[i]);
      }
    } else {
      const u32x4 a = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4_e2*>(static_cast<const uint16_t*>(w) + base + c8));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (DT == kBF16) {
          f[2 * i] = bf16_lo(a[i]);
          f[2 * i + 1] = bf16_hi(a[i]);
        } else {
          f[2 * i] = (float)as_h2(a[i]).x;
          f[2 * i + 1] = (float)as_h2(a[i]).y;
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = c8 + i < n ? load_one(w, base + c8 + i, DT) : 0.f;
  }
}

template <int DT>
__global__ __launch_bounds__(kQT) void k_quantize_mx(const void* __restrict__ w, size_t rows, int n, size_t ldw,
                                                     uint32_t* __restrict__ q, uint8_t* __restrict__ scale) {
  const uint32_t per = (uint32_t)mx_padded(n) / 8;
  const size_t first = (size_t)blockIdx.x * (kQT * kUnits);
  const size_t row0 = first / per;
  const uint32_t c0 = (uint32_t)(first - row0 * per);
  float f[kUnits][8];
  Piece p[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    p[u] = piece_of(threadIdx.x + kQT * u, per, row0, c0);
    if (p[u].row < rows) load8<DT>(w, p[u].row * ldw, p[u].c * 8, n, f[u]);
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    // a quad's pieces lie in one row (16 pieces to a stretch of 128 values), so
    // its four lanes leave together
    if (p[u].row >= rows) continue;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[u][i]) & 0x7fffffffu);
    m = quad_max<0xB1>(m);  // quad_perm(1,0,3,2)
    m = quad_max<0x4E>(m);  // quad_perm(2,3,0,1)
    const uint32_t e = m >> 23;  // floor(log2 m) + 127 for a normal number; 255 for inf and NaN
    const uint32_t byte = e == 255u ? 255u : e > 2u ? e - 2u : 0u;
    const float s = mx_scale(e == 255u ? 254u : byte);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[u][0], f[u][1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[u][2], f[u][3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[u][4], f[u][5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[u][6], f[u][7], s, 3);
    if (e == 255u) c &= 0x88888888u;  // a block without numbers: signs alone
    q[p[u].row * per + p[u].c] = c;
    if ((threadIdx.x & 3) == 0) scale[p[u].row * (per / 4) + (p[u].c >> 2)] = (uint8_t)byte;
  }
}

template <int DT>
__global__ __launch_bounds__(kQT) void k_dequantize_mx(const uint32_t* __restrict__ q,
                                                       const uint8_t* __restrict__ scale, size_t rows, int n,
                                                       void* __restrict__ w) {
  const uint32_t per = (uint32_t)mx_padded(n) / 8;
  const size_t first = (size_t)blockIdx.x * (kQT * kUnits);
  const size_t row0 = first / per;
  const uint32_t c0 = (uint32_t)(first - row0 * per);
  uint32_t c[kUnits], b[kUnits];
  Piece p[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    p[u] = piece_of(threadIdx.x + kQT * u, per, row0, c0);
    if (p[u].row < rows) {
      c[u] = __builtin_nontemporal_load(q + p[u].row * per + p[u].c);
      b[u] = scale[p[u].row * (per / 4) + (p[u].c >> 2)];
    }
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (p[u].row >= rows) continue;
    const float s = mx_scale(b[u]);
    const int c8 = p[u].c * 8;
    const size_t at = p[u].row * (size_t)n + c8;
    if (c8 + 8 <= n) {
      if constexpr (DT == kF32) {
        const f32x2 v0 = mx_f32x2<0>(c[u], s), v1 = mx_f32x2<1>(c[u], s), v2 = mx_f32x2<2>(c[u], s),
                    v3 = mx_f32x2<3>(c[u], s);
        float* o = static_cast<float*>(w) + at;
        const u32x4 a = {__float_as_uint(v0.x), __float_as_uint(v0.y), __float_as_uint(v1.x), __float_as_uint(v1.y)};
        const u32x4 d = {__float_as_uint(v2.x), __float_as_uint(v2.y), __float_as_uint(v3.x), __float_as_uint(v3.y)};
        *reinterpret_cast<u32x4_e4*>(o) = a;
        *reinterpret_cast<u32x4_e4*>(o + 4) = d;
      } else {
        *reinterpret_cast<u32x4_e2*>(static_cast<uint16_t*>(w) + at) = mx_half8<DT == kBF16>(c[u], s);
      }
    } else {
      // the piece that the row ends in: one value at a time, moved down in the
      // word so that the conversion's lowest byte holds it
      uint32_t r = c[u];
      for (int i = c8; i < n; ++i, r >>= 4) {
        if constexpr (DT == kF32)
          static_cast<float*>(w)[at + (i - c8)] = mx_f32x2<0>(r, s).x;
        else
          static_cast<uint16_t*>(w)[at + (i - c8)] = (uint16_t)mx_half8<DT == kBF16>(r, s).x;
      }
    }
  }
}

// The MXFP4 form of k_pack_signs (pack.hip has the layout): one thread per
// (row, word), 16 bytes of codes each; bit j is the sign bit of code j.
// (11008 x 4096, at load only: 7.6 us for 28 MB, 5.5 of a copy's rate; a thread has
// one request in flight.)
__global__ __launch_bounds__(256) void k_pack_signs_mx(const u32x4* __restrict__ q, int k, int d,
                                                       uint32_t* __restrict__ signs) {
  const int W = d >> 5;
  const int kpad = (k + kRowGroup - 1) / kRowGroup * kRowGroup;
  const size_t t = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (t >= (size_t)kpad * W) return;
  const int i = (int)(t / W), wd = (int)(t % W);
  uint32_t word = 0;
  if (i < k) {
    const u32x4 v = q[(size_t)i * W + wd];
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int j = 0; j < 8; ++j) word |= ((v[h] >> (4 * j + 3)) & 1u) << (8 * h + j);
  }
  signs[((size_t)(wd >> 2) * kpad + i) * 4 + (wd & 3)] = word;
}

static size_t mx_blocks(size_t rows, int n) {
  return (rows * (size_t)(mx_padded(n) / 8) + kQT * kUnits - 1) / (kQT * kUnits);
}

hipError_t launch_quantize_mx(const void* w, int dtype, size_t rows, int n, size_t ldw, uint8_t* q, uint8_t* scale,
                              hipStream_t s) {
  const unsigned grid = (unsigned)mx_blocks(rows, n);
  uint32_t* q4 = reinterpret_cast<uint32_t*>(q);
  if (dtype == kF16)
    k_quantize_mx<kF16><<<grid, kQT, 0, s>>>(w, rows, n, ldw, q4, scale);
  else if (dtype == kBF16)
    k_quantize_mx<kBF16><<<grid, kQT, 0, s>>>(w, rows, n, ldw, q4, scale);
  else
    k_quantize_mx<kF32><<<grid, kQT, 0, s>>>(w, rows, n, ldw, q4, scale);
  return hipGetLastError();
}

hipError_t launch_dequantize_mx(const uint8_t* q, const uint8_t* scale, size_t rows, int n, void* w, int dtype,
                                hipStream_t s) {
  const unsigned grid = (unsigned)mx_blocks(rows, n);
  const uint32_t* q4 = reinterpret_cast<const uint32_t*>(q);
  if (dtype == kF16)
    k_dequantize_mx<kF16><<<grid, kQT, 0, s>>>(q4, scale, rows, n, w);
  else if (dtype == kBF16)
    k_dequantize_mx<kBF16><<<grid, kQT, 0, s>>>(q4, scale, rows, n, w);
  else
    k_dequantize_mx<kF32><<<grid, kQT, 0, s>>>(q4, scale, rows, n, w);
  return hipGetLastError();
}

hipError_t launch_pack_signs_mx(const uint8_t* q_gate, int k, int d, uint32_t* signs, hipStream_t s) {
  const int kpad = (k + kRowGroup - 1) / kRowGroup * kRowGroup;
  const size_t threads = (size_t)kpad * (d >> 5);
  k_pack_signs_mx<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(reinterpret_cast<const u32x4*>(q_gate), k, d, signs);
  return hipGetLastError();
}

}  // namespace si
