// Products with MXFP4 weights on the matrix cores: y = x W^T, and with a second
// matrix ReLU(x W^T) * (x W_up^T) (Eq. (1) steps 1-3 of a prompt).
//
// The weights are the A operand (16 rows of W), the tokens the B operand (16
// tokens), so a lane ends with 4 consecutive values of one token's y.  The sum
// over n is taken 128 at a time: lane group g of 16 lanes holds block g (32
// values, 16 bytes of codes, one scale) of its row.
//  * fp16 / bf16 activations: the codes become fp16 or bf16 in registers, scaled
//    (in fp16 exactly where the weight has an fp16 value, in bf16 always), and
//    go through four K = 32 instructions, the j-th with the values 8 j .. 8 j + 7
//    of each group's block: the order inside a sum is free as long as both
//    operands agree.
//  * MXFP4 activations: one K = 128 instruction takes both codes and both scales.
//
// Two shapes of kernel:
//  * k_mx_skinny, up to 16 tokens, bound by the bytes of W: a block owns 16 rows,
//    its waves split n and every wave streams straight into registers.
//  * k_mx_tile: tiles of W and x pass through LDS, double-buffered, written there
//    by the loads themselves.  Where the tiles are fewer than the compute units,
//    n is split over blocks as well and k_mx_join adds the parts in order.
#include "layer_common.h"
#include "mx.h"
#include "mx_launch.h"

namespace si {

enum : int { kActF16 = 0, kActBF16 = 1, kActMx = 2 };

struct LinArgs {
  const uint8_t* q[2];  // codes of W and W_up
  const uint8_t* s[2];
  const void* x;        // fp16 / bf16 rows or codes
  const uint8_t* xs;    // scales of MXFP4 activations
  size_t ldx;           // bytes from row to row of x
  int m, rows, steps;   // steps: 128 values each
  void* y;
  int y_dtype;
  float* part;          // [split][mats][m][rows], or NULL
  int split;
  int relu;             // one matrix: max(y, 0)
  int row_tiles, tok_tiles;
};

__device__ inline f32x4 mfma_half(bool bf, u32x4 a, u32x4 b, f32x4 c) {
  if (bf)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                0);
}
template <int SA, int SB>
__device__ inline f32x4 mfma_mx(u32x4 a, u32x4 b, f32x4 c, uint32_t sa, uint32_t sb) {
  const i32x8 av = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  const i32x8 bv = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, c, 4, 4, SA, (int)sa, SB, (int)sb);
}

// max(g, 0) where a NaN stays one
__device__ inline float relu(float g) { return g > 0.f || g != g ? g : 0.f; }

// ---- up to 16 tokens ---------------------------------------------------------

constexpr int kSW = 8;       // waves of a block: each takes every 8th step
constexpr int kSAhead = 4;   // steps of a wave in flight

template <int ACT, int MATS>
__global__ __launch_bounds__(kSW * kWave) void k_mx_skinny(LinArgs a) {
  constexpr int XV = ACT == kActMx ? 1 : 4;  // 16-byte pieces of x a lane and step
  __shared__ f32x4 red[kSW][MATS][kWave];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int row0 = blockIdx.x * 16;
  const size_t pitch_q = (size_t)a.steps * 64, pitch_s = (size_t)a.steps * 4;
  const int row = min(row0 + r, a.rows - 1), tok = min(r, a.m - 1);
  const uint8_t* xp = static_cast<const uint8_t*>(a.x) + (size_t)tok * a.ldx + g * (ACT == kActMx ? 16 : 64);
  const uint8_t* xsp = ACT == kActMx ? a.xs + (size_t)tok * pitch_s + g : nullptr;
  const uint8_t* qp[MATS];
  const uint8_t* sp[MATS];
  f32x4 acc[MATS];
#pragma unroll
  for (int w = 0; w < MATS; ++w) {
    qp[w] = a.q[w] + (size_t)row * pitch_q + g * 16;
    sp[w] = a.s[w] + (size_t)row * pitch_s + g;
    acc[w] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  for (int k0 = wv; k0 < a.steps; k0 += kSW * kSAhead) {
    u32x4 c[kSAhead][MATS], x[kSAhead][XV];
    uint32_t sc[kSAhead][MATS], sx[kSAhead];
#pragma unroll
    for (int i = 0; i < kSAhead; ++i) {
      const int k = min(k0 + kSW * i, a.steps - 1);
#pragma unroll
      for (int w = 0; w < MATS; ++w) {
        c[i][w] = load_nt(reinterpret_cast<const u32x4*>(qp[w] + (size_t)k * 64));
        sc[i][w] = sp[w][k * 4];
      }
#pragma unroll
      for (int j = 0; j < XV; ++j)
        x[i][j] = *reinterpret_cast<const u32x4*>(xp + (size_t)k * (ACT == kActMx ? 64 : 256) + j * 16);
      sx[i] = ACT == kActMx ? xsp[k * 4] : 0u;
    }
#pragma unroll
    for (int i = 0; i < kSAhead; ++i) {
      if (k0 + kSW * i < a.steps) {
#pragma unroll
        for (int w = 0; w < MATS; ++w) {
          if constexpr (ACT == kActMx) {
            acc[w] = mfma_mx<0, 0>(c[i][w], x[i][0], acc[w], sc[i][w], sx[i]);
          } else {
            const float s = mx_scale(sc[i][w]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              acc[w] = mfma_half(ACT == kActBF16, mx_half8<ACT == kActBF16>(c[i][w][j], s), x[i][j], acc[w]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int w = 0; w < MATS; ++w) red[wv][w][lane] = acc[w];
  __syncthreads();
  if (tid < 256) {
    const int orow = tid & 15, otok = tid >> 4;
    float v[MATS];
#pragma unroll
    for (int w = 0; w < MATS; ++w) {
      v[w] = 0.f;
#pragma unroll
      for (int p = 0; p < kSW; ++p) v[w] += red[p][w][(orow >> 2) * 16 + otok][orow & 3];
    }
    if (row0 + orow < a.rows && otok < a.m)
      store_one(a.y, (size_t)otok * a.rows + row0 + orow, a.y_dtype,
                MATS == 2 ? relu(v[0]) * v[MATS - 1] : a.relu ? relu(v[0]) : v[0]);
  }
}

// ---- tiles ---------------------------------------------------------------------

// A tile: BR rows of W (BR / MATS of each matrix) by BT tokens, WR x WT waves, KB
// steps of 128 values a stage.
template <int ACT, int MATS, int BR, int BT, int WR, int WT>
struct Tile {
  static constexpr int NW = WR * WT;
  static constexpr int KB = ACT == kActMx ? 2 : 1;
  static constexpr int R = BR / WR / 16, T = BT / WT / 16;  // 16-row and 16-token pieces of a wave
  static constexpr int WRow = 64 * KB;                      // bytes of a row's codes in a stage
  static constexpr int XRow = ACT == kActMx ? 64 * KB : 256;
  static constexpr int SRow = 4 * KB;                       // bytes of a row's scales
  static constexpr int WBytes = BR * WRow, XBytes = BT * XRow;
  static constexpr int WsBytes = BR * SRow, XsBytes = ACT == kActMx ? BT * SRow : 0;
  static constexpr int Bytes = WBytes + XBytes + WsBytes + XsBytes;
  // wave requests of a stage: 1 KB of codes or activations, 256 bytes of scales
  static constexpr int IW = WBytes / 1024, IX = XBytes / 1024, IWs = WsBytes / 256, IXs = XsBytes / 256;
  static_assert(R % MATS == 0 && IW % NW == 0 && IX % NW == 0, "whole requests a wave");
};

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef const __attribute__((address_space(1))) uint8_t glb_u8;

// Where 16-byte piece p of row r of a stage lies in its row: rows that share
// banks hold their pieces in different places.
template <int ROW>
__device__ inline int swizzle(int r, int p) {
  if constexpr (ROW == 64)
    return p ^ ((r >> 1) & 3);
  else if constexpr (ROW == 128)
    return p ^ (r & 7);
  else
    return p ^ (r & 15);
}

template <int ACT, int MATS, int BR, int BT, int WR, int WT>
__global__ __launch_bounds__(WR* WT* kWave) void k_mx_tile(LinArgs a) {
  using P = Tile<ACT, MATS, BR, BT, WR, WT>;
  constexpr int NW = P::NW, R = P::R, T = P::T, KB = P::KB;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
  // XCD-aware order: blocks go to the XCDs in turn, so every XCD gets a run of
  // neighbouring tiles; in a run 8 token tiles share each row tile
  const int total = a.row_tiles * a.tok_tiles;
  int id = blockIdx.x % total;
  const int part = blockIdx.x / total;
  if (total % 8 == 0) id = (id & 7) * (total / 8) + (id >> 3);
  const int grp = id / (8 * a.row_tiles), in = id - grp * 8 * a.row_tiles;
  const int gw = min(8, a.tok_tiles - grp * 8);
  const int tok0 = (grp * 8 + in % gw) * BT, row0 = (in / gw) * (BR / MATS);
  // the stages of this part of n
  const int stages_all = a.steps / KB;
  const int k_first = (int)((long long)stages_all * part / a.split);
  const int k_last = (int)((long long)stages_all * (part + 1) / a.split);

  const size_t pitch_q = (size_t)a.steps * 64, pitch_s = (size_t)a.steps * 4;
  // per-lane offsets of this wave's requests from the tile's first row
  constexpr int LW = 1024 / P::WRow, LX = 1024 / P::XRow;  // rows a request
  uint32_t ow[P::IW / NW], ox[P::IX / NW];
  const uint8_t* bw[P::IW / NW];
#pragma unroll
  for (int i = 0; i < P::IW / NW; ++i) {
    const int r = (wv + NW * i) * LW + lane / (64 / LW);  // row of the tile
    const int mat = r / (BR / MATS);
    const int rr = min(row0 + r % (BR / MATS), a.rows - 1) - row0;
    ow[i] = (uint32_t)(rr * (int)pitch_q) + 16 * swizzle<P::WRow>(r, lane % (64 / LW));
    bw[i] = a.q[MATS == 2 ? uniform(mat) : 0] + (size_t)row0 * pitch_q;
  }
#pragma unroll
  for (int i = 0; i < P::IX / NW; ++i) {
    const int r = (wv + NW * i) * LX + lane / (64 / LX);
    const int rr = min(tok0 + r, a.m - 1) - tok0;
    ox[i] = (uint32_t)rr * (uint32_t)a.ldx + 16 * swizzle<P::XRow>(r, lane % (64 / LX));
  }
  const uint8_t* bx = static_cast<const uint8_t*>(a.x) + (size_t)tok0 * a.ldx;
  constexpr int NS = P::IWs + P::IXs;          // scale requests of a stage
  constexpr int MS = (NS + NW - 1) / NW;
  uint32_t os[MS];
  const uint8_t* bs[MS];
#pragma unroll
  for (int i = 0; i < MS; ++i) {
    const int q = wv + NW * i;
    const bool of_x = q >= P::IWs;
    const int r = (of_x ? q - P::IWs : q) * (64 / KB) + lane / KB;  // one 4-byte word a lane
    const int base = of_x ? tok0 : row0, last = (of_x ? a.m : a.rows) - 1;
    const int per = of_x ? BT : BR / MATS;
    const int rr = min(base + r % per, last) - base;
    os[i] = (uint32_t)(rr * (int)pitch_s) + 4 * (lane % KB);
    const uint8_t* sc = a.s[0];  // a request of the small tile spans both matrices
    if (MATS == 2 && r >= BR / MATS) sc = a.s[1];
    bs[i] = (of_x ? a.xs : sc) + (size_t)base * pitch_s;
  }

  auto request = [&](uint8_t* __restrict__ to, int k) {
#pragma unroll
    for (int i = 0; i < P::IW / NW; ++i)
      __builtin_amdgcn_global_load_lds((glb_u8*)(bw[i] + (size_t)k * P::WRow + ow[i]),
                                       (lds_u8*)(to + (wv + NW * i) * 1024), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < P::IX / NW; ++i)
      __builtin_amdgcn_global_load_lds((glb_u8*)(bx + (size_t)k * P::XRow + ox[i]),
                                       (lds_u8*)(to + P::WBytes + (wv + NW * i) * 1024), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < MS; ++i)
      if (wv + NW * i < NS)
        __builtin_amdgcn_global_load_lds((glb_u8*)(bs[i] + (size_t)k * P::SRow + os[i]),
                                         (lds_u8*)(to + P::WBytes + P::XBytes + (wv + NW * i) * 256), 4, 0, 0);
  };

  const int wr = wv / WT, wt = wv % WT;
  const int r = lane & 15, g = lane >> 4;
  f32x4 acc[R][T];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int t = 0; t < T; ++t) acc[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  // first row of the wave's 16-row piece i in the tile: with two matrices half of
  // the pieces are W's rows and half the same rows of W_up
  auto piece_row = [&](int i) {
    if constexpr (MATS == 2)
      return (i / (R / 2)) * (BR / 2) + wr * (BR / 2 / WR) + (i % (R / 2)) * 16;
    else
      return wr * (BR / WR) + i * 16;
  };

  auto compute = [&](const uint8_t* __restrict__ from) {
    const uint8_t* wl = from;
    const uint8_t* xl = from + P::WBytes;
    const uint8_t* sl = xl + P::XBytes;
    if constexpr (ACT == kActMx) {
      uint32_t sw[R], sx[T];
#pragma unroll
      for (int i = 0; i < R; ++i)
        sw[i] = *reinterpret_cast<const uint16_t*>(sl + (piece_row(i) + r) * P::SRow + 2 * g);
#pragma unroll
      for (int t = 0; t < T; ++t)
        sx[t] = *reinterpret_cast<const uint16_t*>(sl + P::WsBytes + (wt * (BT / WT) + t * 16 + r) * P::SRow + 2 * g);
      // step s: lane group g takes block 2 g + s of the stage's 8
      u32x4 w[R], x[T];
      auto read = [&](int s) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
          const int row = wt * (BT / WT) + t * 16 + r;
          x[t] = *reinterpret_cast<const u32x4*>(xl + row * P::XRow + 16 * swizzle<P::XRow>(row, 2 * g + s));
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const int row = piece_row(i) + r;
          w[i] = *reinterpret_cast<const u32x4*>(wl + row * P::WRow + 16 * swizzle<P::WRow>(row, 2 * g + s));
        }
      };
      read(0);
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[i][t] = mfma_mx<0, 0>(w[i], x[t], acc[i][t], sw[i], sx[t]);
      read(1);
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[i][t] = mfma_mx<1, 1>(w[i], x[t], acc[i][t], sw[i], sx[t]);
    } else {
      u32x4 w[R];
      float sw[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int row = piece_row(i) + r;
        w[i] = *reinterpret_cast<const u32x4*>(wl + row * P::WRow + 16 * swizzle<P::WRow>(row, g));
        sw[i] = mx_scale(sl[row * P::SRow + g]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 x[T];
#pragma unroll
        for (int t = 0; t < T; ++t) {
          const int row = wt * (BT / WT) + t * 16 + r;
          x[t] = *reinterpret_cast<const u32x4*>(xl + row * P::XRow + 16 * swizzle<P::XRow>(row, 4 * g + j));
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const u32x4 wh = mx_half8<ACT == kActBF16>(w[i][j], sw[i]);
#pragma unroll
          for (int t = 0; t < T; ++t) acc[i][t] = mfma_half(ACT == kActBF16, wh, x[t], acc[i][t]);
        }
      }
    }
  };
  // one stage computed while the next one's requests are in flight; the two
  // halves of LDS are told apart by the pointers' restrict, without which every
  // read of LDS would wait for all requests
  auto step = [&](uint8_t* __restrict__ to, const uint8_t* __restrict__ from, int k, bool more) {
    if (more) request(to, k);
    compute(from);
  };

  if (k_first < k_last) {
    request(lds, k_first);
    for (int k = k_first; k < k_last; ++k) {
      const int cur = (k - k_first) & 1;
      wait_all_requests();
      __syncthreads();  // the stage is in LDS, and every wave has left the other half
      step(lds + (cur ^ 1) * P::Bytes, lds + cur * P::Bytes, k + 1, k + 1 < k_last);
    }
  }
  if (ACT == kActMx && a.steps % KB != 0 && part == a.split - 1) {
    // the odd 128 values at the end, straight from memory
    const int k = a.steps - 1;
    u32x4 x[T];
    uint32_t sx[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const size_t tok = min(tok0 + wt * (BT / WT) + t * 16 + r, a.m - 1);
      x[t] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.x) + tok * a.ldx + (size_t)k * 64 + g * 16);
      sx[t] = a.xs[tok * pitch_s + (size_t)k * 4 + g];
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int tr = piece_row(i) + r, mat = MATS == 2 ? piece_row(i) / (BR / 2) : 0;
      const size_t row = min(row0 + tr % (BR / MATS), a.rows - 1);
      const u32x4 w = *reinterpret_cast<const u32x4*>(a.q[mat] + row * pitch_q + (size_t)k * 64 + g * 16);
      const uint32_t sw = a.s[mat][row * pitch_s + (size_t)k * 4 + g];
#pragma unroll
      for (int t = 0; t < T; ++t) acc[i][t] = mfma_mx<0, 0>(w, x[t], acc[i][t], sw, sx[t]);
    }
  }

  // a lane holds rows 4 g .. 4 g + 3 of each piece for token r of each
  const bool vec = (a.rows & 3) == 0;
  auto put = [&](void* y, int dt, int i, int t, f32x4 v) {
    const int row = row0 + piece_row(i) % (BR / MATS) + 4 * g;
    const int tok = tok0 + wt * (BT / WT) + t * 16 + r;
    if (tok >= a.m || row >= a.rows) return;
    const size_t at = (size_t)tok * a.rows + row;
    if (vec) {
      if (dt == kF32)
        *reinterpret_cast<f32x4*>(static_cast<float*>(y) + at) = v;
      else if (dt == kBF16)
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(y) + at) = u32x2{pack_bf2(v.x, v.y), pack_bf2(v.z, v.w)};
      else
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(y) + at) = u32x2{pack_f2(v.x, v.y), pack_f2(v.z, v.w)};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (row + e < a.rows) store_one(y, at + e, dt, v[e]);
    }
  };
  if (a.part) {
    const size_t mat_size = (size_t)a.m * a.rows;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int mat = MATS == 2 ? i / (R / 2) : 0;
#pragma unroll
      for (int t = 0; t < T; ++t) put(a.part + (size_t)(part * MATS + mat) * mat_size, kF32, i, t, acc[i][t]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < R / MATS; ++i)
#pragma unroll
      for (int t = 0; t < T; ++t) {
        f32x4 v = acc[i][t];
        if constexpr (MATS == 2) {
          const f32x4 u = acc[i + R / 2][t];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = relu(v[e]) * u[e];
        } else if (a.relu) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = relu(v[e]);
        }
        put(a.y, a.y_dtype, i, t, v);
      }
  }
}

// The parts of a split product, added in their order, 4 values a thread.
template <int MATS>
__global__ __launch_bounds__(256) void k_mx_join(const float* __restrict__ part, int split, size_t size,
                                                 void* __restrict__ y, int dt, int relu1) {
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= size) return;
  const int n = (int)min(size - i, (size_t)4);
  float v[MATS][4];
#pragma unroll
  for (int w = 0; w < MATS; ++w)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[w][e] = 0.f;
  for (int p = 0; p < split; ++p)
#pragma unroll
    for (int w = 0; w < MATS; ++w) {
      const float* src = part + (size_t)(p * MATS + w) * size + i;
      if (n == 4 && (size & 3) == 0) {
        const f32x4 f = *reinterpret_cast<const f32x4*>(src);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[w][e] += f[e];
      } else {
        for (int e = 0; e < n; ++e) v[w][e] += src[e];
      }
    }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) store_one(y, i + e, dt, MATS == 2 ? relu(v[0][e]) * v[MATS - 1][e] : relu1 ? relu(v[0][e]) : v[0][e]);
}

// A copy of x with rows of whole 128 values, zeros behind the row's n: 8 values a
// thread.
__global__ __launch_bounds__(256) void k_mx_pad(const uint16_t* __restrict__ x, size_t ldx, int m, int n, int np,
                                                u32x4* __restrict__ out) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (size_t)m * (np / 8)) return;
  const size_t r = i / (np / 8);
  const int c = (int)(i - r * (np / 8)) * 8;
  const uint16_t* row = x + r * ldx;
  u32x4 v = {0, 0, 0, 0};
  if (c + 8 <= n) {
    v = *reinterpret_cast<const u32x4_e2*>(row + c);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < n) v[e >> 1] |= (uint32_t)row[c + e] << (16 * (e & 1));
  }
  out[i] = v;
}

// ---- host ----------------------------------------------------------------------

namespace {

struct Plan {
  bool pad;      // x is copied into the workspace first
  bool skinny;
  bool big;      // the large tile
  int split;
  size_t pad_bytes, part_bytes;
};

int act_of(const MxLinear& c) { return c.xq ? kActMx : c.x_dtype == kBF16 ? kActBF16 : kActF16; }

constexpr int kSkinnyTokens = 16;
constexpr int kSmallRows = 64, kSmallToks = 64;

Plan plan_of(const MxLinear& c) {
  Plan p;
  const int np = mx_padded(c.n), mats = c.q_up ? 2 : 1, act = act_of(c);
  p.pad = act != kActMx && (c.n % kMxPad != 0 || c.ldx % 8 != 0 || (reinterpret_cast<uintptr_t>(c.x) & 15u) != 0);
  p.pad_bytes = p.pad ? align256((size_t)c.m * np * 2) : 0;
  p.skinny = c.m <= kSkinnyTokens;
  p.split = 1;
  p.big = false;
  if (!p.skinny) {
    const int big_r = 256 / mats, big_t = act == kActMx ? 256 : 128;
    const long big = (long)((c.rows + big_r - 1) / big_r) * ((c.m + big_t - 1) / big_t);
    p.big = big >= 192;
    if (!p.big) {
      const long tiles = (long)((c.rows + kSmallRows / mats - 1) / (kSmallRows / mats)) * ((c.m + kSmallToks - 1) / kSmallToks);
      const int stages = np / kMxPad / (act == kActMx ? 2 : 1);
      long split = (512 + tiles - 1) / tiles;
      if (split > stages / 4) split = stages / 4;
      if (split > 16) split = 16;
      p.split = split < 1 ? 1 : (int)split;
    }
  }
  p.part_bytes = p.split > 1 ? (size_t)p.split * mats * c.m * c.rows * sizeof(float) : 0;
  return p;
}

template <int ACT, int MATS, int BR, int BT, int WR, int WT>
hipError_t tile_launch(LinArgs a, hipStream_t s) {
  using P = Tile<ACT, MATS, BR, BT, WR, WT>;
  static std::atomic<int> attr_set[kMaxDevices];
  const int ok = per_device_once(attr_set, [](int) -> int {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_mx_tile<ACT, MATS, BR, BT, WR, WT>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, 2 * P::Bytes) == hipSuccess ? 1 : -1;
  });
  if (ok != 1) return hipErrorInvalidConfiguration;
  a.row_tiles = (a.rows + BR / MATS - 1) / (BR / MATS);
  a.tok_tiles = (a.m + BT - 1) / BT;
  k_mx_tile<ACT, MATS, BR, BT, WR, WT>
      <<<(unsigned)(a.row_tiles * a.tok_tiles * a.split), WR * WT * kWave, 2 * P::Bytes, s>>>(a);
  return hipGetLastError();
}

template <int ACT, int MATS>
hipError_t linear_launch(const LinArgs& a, const Plan& p, hipStream_t s) {
  if (p.skinny) {
    k_mx_skinny<ACT, MATS><<<(unsigned)((a.rows + 15) / 16), kSW * kWave, 0, s>>>(a);
    return hipGetLastError();
  }
  hipError_t e;
  if (p.big) {
    if constexpr (ACT == kActMx)
      e = tile_launch<ACT, MATS, 256, 256, 2, 4>(a, s);
    else
      e = tile_launch<ACT, MATS, 256, 128, 4, 2>(a, s);
  } else {
    e = tile_launch<ACT, MATS, kSmallRows, kSmallToks, 2, 2>(a, s);
  }
  if (e != hipSuccess || !a.part) return e;
  const size_t size = (size_t)a.m * a.rows;
  k_mx_join<MATS><<<(unsigned)((size + 1023) / 1024), 256, 0, s>>>(a.part, a.split, size, a.y, a.y_dtype, a.relu);
  return hipGetLastError();
}

template <int ACT>
hipError_t linear_mats(const LinArgs& a, const Plan& p, hipStream_t s) {
  return a.q[1] ? linear_launch<ACT, 2>(a, p, s) : linear_launch<ACT, 1>(a, p, s);
}

}  // namespace

bool mx_linear_fits(const MxLinear& c) {
  // the finest tiles and the longest copy: fewer than 2^32 threads a launch
  const double tiles = ((double)c.rows / 32 + 1) * ((double)c.m / 64 + 1);
  return tiles * 512 < 4294967296.0 && (double)c.m * (mx_padded(c.n) / 8) < 4294967296.0;
}

size_t mx_linear_workspace(const MxLinear& c) {
  const Plan p = plan_of(c);
  return p.pad_bytes + p.part_bytes;
}

hipError_t launch_mx_linear(const MxLinear& c, hipStream_t s) {
  const Plan p = plan_of(c);
  const int np = mx_padded(c.n), act = act_of(c);
  LinArgs a = {};
  a.q[0] = c.q;
  a.q[1] = c.q_up;
  a.s[0] = c.s;
  a.s[1] = c.s_up;
  a.m = c.m;
  a.rows = c.rows;
  a.steps = np / kMxPad;
  a.y = c.y;
  a.y_dtype = c.y_dtype;
  a.split = p.split;
  a.relu = c.relu;
  a.part = p.part_bytes ? reinterpret_cast<float*>(static_cast<char*>(c.ws) + p.pad_bytes) : nullptr;
  if (act == kActMx) {
    a.x = c.xq;
    a.xs = c.xs;
    a.ldx = (size_t)a.steps * 64;
  } else if (p.pad) {
    const size_t all = (size_t)c.m * (np / 8);
    k_mx_pad<<<(unsigned)((all + 255) / 256), 256, 0, s>>>(static_cast<const uint16_t*>(c.x), c.ldx, c.m, c.n, np,
                                                           static_cast<u32x4*>(c.ws));
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    a.x = c.ws;
    a.ldx = (size_t)np * 2;
  } else {
    a.x = c.x;
    a.ldx = c.ldx * 2;
  }
  return act == kActMx ? linear_mats<kActMx>(a, p, s) : act == kActBF16 ? linear_mats<kActBF16>(a, p, s)
                                                                         : linear_mats<kActF16>(a, p, s);
}

}  // namespace si
