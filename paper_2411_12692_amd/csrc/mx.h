// MXFP4 on gfx950: 32 consecutive values of a row share a power-of-two scale
// (one byte X + 127; 255 is NaN), a value is a 4-bit e2m1 code, two codes a byte
// with the first in the low half.  Rows are padded with zeros to a multiple of
// kMxPad values, so that a row's codes are whole 64-byte pieces, its scales
// whole 4-byte words and its products whole K = 128 matrix instructions.
#pragma once

#include "si_device.h"

namespace si {

constexpr int kMxBlock = 32;  // values that share a scale
constexpr int kMxPad = 128;   // a row's stored length is a multiple of this

__host__ __device__ inline int mx_padded(int n) { return (n + kMxPad - 1) / kMxPad * kMxPad; }

// Element types of the calls that take more than one (si_dtype).
enum : int { kF16 = 0, kBF16 = 1, kF32 = 2 };
__host__ __device__ inline int dtype_bytes(int t) { return t == kF32 ? 4 : 2; }

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
// 16 bytes at any element boundary (rows of an odd length start anywhere)
typedef u32x4 u32x4_e2 __attribute__((aligned(2)));
typedef u32x4 u32x4_e4 __attribute__((aligned(4)));
typedef u32x4 u32x4_e8 __attribute__((aligned(8)));

// A scale byte as the float whose exponent field it is: the operand of the
// conversion instructions, which read that field alone (0 is 2^-127, 255 NaN).
__device__ inline float mx_scale(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// A scale byte as a factor of a float product (0 and 255 are not what their bits
// would be as a float: zero and infinity).
__device__ inline float mx_factor(uint32_t byte) {
  const uint32_t bits = byte == 0u ? 0x00400000u : byte << 23;
  return __builtin_bit_cast(float, byte == 255u ? 0x7fc00000u : bits);
}

// Two codes (byte SEL of `codes`) times the scale.
template <int SEL>
__device__ inline uint32_t mx_f16x2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL));
}
template <int SEL>
__device__ inline uint32_t mx_bf16x2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
template <int SEL>
__device__ inline f32x2 mx_f32x2(uint32_t codes, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, SEL);
}

// Eight codes (32 bits) times the scale, as 16 bytes of fp16 or bf16.
template <bool BF>
__device__ inline u32x4 mx_half8(uint32_t codes, float scale) {
  if constexpr (BF)
    return u32x4{mx_bf16x2<0>(codes, scale), mx_bf16x2<1>(codes, scale), mx_bf16x2<2>(codes, scale),
                 mx_bf16x2<3>(codes, scale)};
  else
    return u32x4{mx_f16x2<0>(codes, scale), mx_f16x2<1>(codes, scale), mx_f16x2<2>(codes, scale),
                 mx_f16x2<3>(codes, scale)};
}

__device__ inline float bf16_lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ inline float bf16_hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }

// float -> bf16 bits, to nearest even (the hardware conversion)
__device__ inline uint32_t pack_bf2(float lo, float hi) {
  const bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ inline uint32_t pack_f2(float lo, float hi) {
  const f16x2 v = {(_Float16)lo, (_Float16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

__device__ inline float load_one(const void* p, size_t i, int t) {
  if (t == kF32) return static_cast<const float*>(p)[i];
  const uint16_t v = static_cast<const uint16_t*>(p)[i];
  return t == kF16 ? (float)__builtin_bit_cast(_Float16, v) : __builtin_bit_cast(float, (uint32_t)v << 16);
}
__device__ inline void store_one(void* p, size_t i, int t, float v) {
  if (t == kF32)
    static_cast<float*>(p)[i] = v;
  else
    static_cast<uint16_t*>(p)[i] = (uint16_t)(t == kF16 ? pack_f2(v, 0.f) : pack_bf2(v, 0.f));
}

}  // namespace si
