// x W^T for up to 4 tokens, W's rows read once straight into registers: what decoding
// takes of the dense products.  A wave takes RW rows of W (of both matrices), 16 bytes a
// lane at a time, U pieces of each row in a round, the next round's pieces in flight
// while one is multiplied; the tokens' values come from the caches.  Sums stay with the
// lanes until the row ends.
//
// Bound by W's bytes: at one token 2 flops for each value read.  7B gate and up (180 MB):
// 27.2 us with the same W in every call, part of it in the last-level cache, 29.6 us, 6.1
// TB/s, with others in turn; e4m3, 4096 x 11008 (45 MB): 10.3 and 13.3 us (3.4 TB/s), a
// launch and two round trips of memory; gate and up of 11008 x 4096 (90 MB) 15.7 and 17.5.
#include "dense.h"
#include "layer_common.h"

namespace si {

namespace {

// Values of a 16-byte piece as floats: 8 of 16 bits or 16 of 8.
template <int T>
__device__ inline void piece_values(u32x4 v, float (&f)[T == 2 ? 16 : 8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (T == 2) {
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[e], true);
      f[4 * e] = lo.x;
      f[4 * e + 1] = lo.y;
      f[4 * e + 2] = hi.x;
      f[4 * e + 3] = hi.y;
    } else if constexpr (T == 1) {
      f[2 * e] = bf16_lo(v[e]);
      f[2 * e + 1] = bf16_hi(v[e]);
    } else {
      f[2 * e] = (float)as_h2(v[e]).x;
      f[2 * e + 1] = (float)as_h2(v[e]).y;
    }
  }
}

}  // namespace

// T: 0 fp16, 1 bf16, 2 e4m3; MT tokens at most.
template <int T, int MATS, int MT, int RW, int U>
__global__ __launch_bounds__(256) void k_dense_few(DenseArgs a) {
  constexpr int PV = T == 2 ? 16 : 8;  // values of a piece
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
  const int row0 = (blockIdx.x * 4 + wv) * RW;
  if (row0 >= a.M) return;  // whole waves, which meet no barrier
  const int pieces = (a.K + PV - 1) / PV;
  const uint8_t* w[MATS][RW];
#pragma unroll
  for (int q = 0; q < MATS; ++q)
#pragma unroll
    for (int i = 0; i < RW; ++i)
      w[q][i] = static_cast<const uint8_t*>(a.a[q]) + (size_t)min(row0 + i, a.M - 1) * a.lda;
  const uint8_t* x[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) x[t] = static_cast<const uint8_t*>(a.b[0]) + (size_t)min(t, a.N - 1) * a.ldb;
  float acc[MATS][RW][MT];
#pragma unroll
  for (int q = 0; q < MATS; ++q)
#pragma unroll
    for (int i = 0; i < RW; ++i)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[q][i][t] = 0.f;

  struct Round {
    u32x4 w[U][MATS][RW];
  };
  auto load = [&](int p0, Round& r) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const size_t at = (size_t)min(p0 + lane + kWave * j, pieces - 1) * 16;
#pragma unroll
      for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int i = 0; i < RW; ++i) r.w[j][q][i] = load_nt(reinterpret_cast<const u32x4*>(w[q][i] + at));
    }
  };
  auto multiply = [&](int p0, const Round& r) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int p = p0 + lane + kWave * j;
      const bool on = p < pieces;
      const int pc = min(p, pieces - 1);
      u32x4 xv[MT];
      float sx[MT], sw[MATS];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        xv[t] = *reinterpret_cast<const u32x4*>(x[t] + (size_t)pc * 16);
        if constexpr (T == 2) sx[t] = a.sb[(size_t)min(t, a.N - 1) * a.blocks + pc / 8];
      }
      if constexpr (T == 2) {
#pragma unroll
        for (int q = 0; q < MATS; ++q) sw[q] = a.sa[q][(size_t)(row0 / 128) * a.blocks + pc / 8];
      }
      float xf[MT][PV];
#pragma unroll
      for (int t = 0; t < MT; ++t) piece_values<T>(xv[t], xf[t]);
#pragma unroll
      for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int i = 0; i < RW; ++i) {
          float wf[PV];
          piece_values<T>(r.w[j][q][i], wf);
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            float s = T == 2 ? 0.f : acc[q][i][t];
#pragma unroll
            for (int e = 0; e < PV; ++e) s = fmaf(wf[e], xf[t][e], s);
            if constexpr (T == 2) s = fmaf(s, sw[q] * sx[t], acc[q][i][t]);
            acc[q][i][t] = on ? s : acc[q][i][t];  // past the row's end: its last piece again
          }
        }
    }
  };
  Round r[2];
  constexpr int kStep = kWave * U;
  load(0, r[0]);
  for (int p0 = 0; p0 < pieces; p0 += 2 * kStep) {
    if (p0 + kStep < pieces) load(p0 + kStep, r[1]);
    multiply(p0, r[0]);
    if (p0 + kStep >= pieces) break;
    if (p0 + 2 * kStep < pieces) load(p0 + 2 * kStep, r[0]);
    multiply(p0 + kStep, r[1]);
  }
#pragma unroll
  for (int q = 0; q < MATS; ++q)
#pragma unroll
    for (int i = 0; i < RW; ++i)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[q][i][t] = wave_total(acc[q][i][t]);
  if (lane != 0) return;
#pragma unroll
  for (int i = 0; i < RW; ++i)
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      if (row0 + i >= a.M || t >= a.N) continue;
      const size_t at = (size_t)t * a.M + row0 + i;
      float v = acc[0][i][t];
      if constexpr (MATS == 2) {
        if (a.g) {
          a.g[at] = v;
          a.u[at] = acc[MATS - 1][i][t];
        }
        v = (v > 0.f || v != v ? v : 0.f) * acc[MATS - 1][i][t];
      } else if (a.relu) {
        v = v > 0.f || v != v ? v : 0.f;
      }
      store_one(a.c[0], at, a.c_dtype, v);
    }
}

template <int T, int MATS, int MT>
static hipError_t few_tokens(const DenseArgs& a, hipStream_t s) {
  constexpr int RW = MATS == 2 ? 1 : 2, U = 4;
  k_dense_few<T, MATS, MT, RW, U><<<(unsigned)((a.M + 4 * RW - 1) / (4 * RW)), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int T, int MATS>
static hipError_t few_mats(const DenseArgs& a, hipStream_t s) {
  return a.N == 1 ? few_tokens<T, MATS, 1>(a, s) : a.N == 2 ? few_tokens<T, MATS, 2>(a, s) : few_tokens<T, MATS, 4>(a, s);
}

template <int T>
static hipError_t few_type(int mats, const DenseArgs& a, hipStream_t s) {
  return mats == 2 ? few_mats<T, 2>(a, s) : few_mats<T, 1>(a, s);
}

hipError_t dense_few(int type, int mats, const DenseArgs& a, hipStream_t s) {
  if (a.M < 1 || a.N < 1 || a.N > kFewTokens || a.K < 1) return hipErrorInvalidValue;
  return type == 2 ? few_type<2>(mats, a, s) : type == 1 ? few_type<1>(mats, a, s) : few_type<0>(mats, a, s);
}

}  // namespace si
