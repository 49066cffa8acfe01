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
//  * k_mx_tile: tiles of W and x pass through LDS in stages of 128 to 1024 values,
//    written there by the loads themselves, the next one or two in flight while
//    one is used.  Where a stage has little work for its waves they form groups
//    that each take a part of its values.  With few tiles and a long n, n is split
//    over blocks as well and k_mx_join adds the parts in order.
//    (2048 tokens, 4096 x 11008 fp16: 158 us = 1.17 PFLOP/s; 4096 tokens, 13824 x
//    5120 with MXFP4 activations: 194-213 us = 2.7-3.0 PFLOP/s; 16 tokens, 11008 x
//    4096: 8.4 us = 2.9 TB/s of weights; gated, 37 tokens, 13824 x 5120: 27.6 us.)
//  * k_mx_skinny, a few tokens and few rows: a block owns 16 rows, its waves split
//    n and stream the codes straight into registers, 48 steps of 128 values at a
//    time; the tokens pass through LDS.  (One token, 4096 x 11008: 7.8 us = 3 TB/s;
//    the bytes alone would take 4.7, but its 86 steps are two rounds, the second
//    asked for once the first is multiplied.)
#include <algorithm>
#include <type_traits>

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

// ---- a few tokens and few rows ---------------------------------------------------

constexpr int kSW = 16;        // waves of a block: each takes every 16th step
constexpr int kSAhead = 3;     // steps of a wave whose codes are in flight
constexpr int kSToks = 4;      // tokens
constexpr int kSChunk = kSW * kSAhead;  // steps of a round: their codes in flight, their x in LDS
// bytes of a token's x in LDS: 16 more than its values, so that the tokens' pieces
// lie in different banks
inline __host__ __device__ int skinny_pitch(int steps) { return (steps < kSChunk ? steps : kSChunk) * 256 + 16; }
static_assert(kSToks * (kSChunk * 256 + 16) + kSW * 2 * kWave * 16 <= kMaxLds, "x and the waves' sums");

template <int ACT, int MATS>
__global__ __launch_bounds__(kSW * kWave) void k_mx_skinny(LinArgs a) {
  __shared__ f32x4 red[kSW][MATS][kWave];
  extern __shared__ __attribute__((aligned(16))) uint8_t xl[];  // [m][pitch_x]
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int row0 = blockIdx.x * 16;
  const size_t pitch_q = (size_t)a.steps * 64, pitch_s = (size_t)a.steps * 4;
  const int row = min(row0 + r, a.rows - 1), tok = min(r, a.m - 1);
  const int pitch_x = skinny_pitch(a.steps);
  const uint8_t* xq = static_cast<const uint8_t*>(a.x) + (size_t)tok * a.ldx + g * 16;  // MXFP4 activations
  const uint8_t* xs = ACT == kActMx ? a.xs + (size_t)tok * pitch_s + g : nullptr;
  const uint8_t* xt = xl + tok * pitch_x + g * 64;
  const uint8_t* qp[MATS];
  const uint8_t* sp[MATS];
  f32x4 acc[MATS];
#pragma unroll
  for (int w = 0; w < MATS; ++w) {
    qp[w] = a.q[w] + (size_t)row * pitch_q + g * 16;
    sp[w] = a.s[w] + (size_t)row * pitch_s + g;
    acc[w] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  for (int k0 = 0; k0 < a.steps; k0 += kSChunk) {
    const int k1 = min(k0 + kSChunk, a.steps);
    u32x4 c[kSAhead][MATS], x[kSAhead];
    uint32_t sc[kSAhead][MATS], sx[kSAhead];
#pragma unroll
    for (int i = 0; i < kSAhead; ++i) {
      const int k = k0 + wv + kSW * i;
      if (k < k1) {
#pragma unroll
        for (int w = 0; w < MATS; ++w) {
          c[i][w] = *reinterpret_cast<const u32x4*>(qp[w] + (size_t)k * 64);
          sc[i][w] = sp[w][k * 4];
        }
        if constexpr (ACT == kActMx) {
          x[i] = *reinterpret_cast<const u32x4*>(xq + (size_t)k * 64);
          sx[i] = xs[k * 4];
        }
      }
    }
    if constexpr (ACT != kActMx) {
      // the tokens' values of these steps, read once for the block's 16 rows
      const int per = (k1 - k0) * 16;  // 16-byte pieces a token
      const uint8_t* src = static_cast<const uint8_t*>(a.x) + (size_t)k0 * 256;
      if (k0 > 0) __syncthreads();
      for (int t = 0; t < a.m; ++t)
        for (int i = tid; i < per; i += kSW * kWave)
          *reinterpret_cast<u32x4*>(xl + t * pitch_x + i * 16) =
              *reinterpret_cast<const u32x4*>(src + (size_t)t * a.ldx + (size_t)i * 16);
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kSAhead; ++i) {
      const int k = k0 + wv + kSW * i;
      if (k < k1) {
        u32x4 v[4];
        if constexpr (ACT != kActMx) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const u32x4*>(xt + (k - k0) * 256 + j * 16);
        }
#pragma unroll
        for (int w = 0; w < MATS; ++w) {
          if constexpr (ACT == kActMx) {
            acc[w] = mfma_mx<0, 0>(c[i][w], x[i], acc[w], sc[i][w], sx[i]);
          } else {
            const float s = mx_scale(sc[i][w]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              acc[w] = mfma_half(ACT == kActBF16, mx_half8<ACT == kActBF16>(c[i][w][j], s), v[j], acc[w]);
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

// A tile: BR rows of W (BR / MATS of each matrix) by BT tokens, WR x WT waves of
// its own part of each, WK groups of such waves that share out a stage's steps
// (KB each, of 128 values), ST stages in LDS.
template <int ACT, int MATS, int BR, int BT, int WR, int WT, int WK, int ST>
struct Tile {
  static constexpr int NW = WR * WT * WK;
  static constexpr int KB = ACT == kActMx ? 2 : 1;
  static constexpr int SK = KB * WK;  // steps of a stage
  static constexpr int R = BR / WR / 16, T = BT / WT / 16;  // 16-row and 16-token pieces of a wave
  static constexpr int WRow = 64 * SK;                      // bytes of a row's codes in a stage
  static constexpr int XRow = ACT == kActMx ? 64 * SK : 256 * SK;
  static constexpr int SRow = 4 * SK;                       // bytes of a row's scales
  // pieces from one lane group's to the next one's
  static constexpr int WDelta = ACT == kActMx ? 2 : 1, XDelta = ACT == kActMx ? 2 : 4;
  static constexpr int WBytes = BR * WRow, XBytes = BT * XRow;
  static constexpr int WsBytes = BR * SRow, XsBytes = ACT == kActMx ? BT * SRow : 0;
  static constexpr int Bytes = WBytes + XBytes + WsBytes + XsBytes;
  // wave requests of a stage: 1 KB of codes or activations, 256 bytes of scales
  static constexpr int IW = WBytes / 1024, IX = XBytes / 1024, IWs = WsBytes / 256, IXs = XsBytes / 256;
  static constexpr int NS = IWs + IXs, MS = (NS + NW - 1) / NW;
  // requests of a wave and stage, the same for every wave: the waits count them
  static constexpr int Requests = IW / NW + IX / NW + MS;
  static_assert(WRow <= 1024 && XRow <= 1024 && SK <= 64, "a request covers whole rows");
  static_assert(WBytes % 1024 == 0 && XBytes % 1024 == 0 && WsBytes % 256 == 0 && XsBytes % 256 == 0, "whole requests");
  static_assert(BR / MATS % (1024 / WRow) == 0, "a request's codes are of one matrix");
  static_assert(R % MATS == 0 && IW % NW == 0 && IX % NW == 0, "whole requests a wave");
  static_assert(Requests * (ST - 2) < 64, "what a wait can leave outstanding");
  static_assert(ST * Bytes <= kMaxLds, "LDS of a compute unit");
  static_assert((WK - 1) * BR * BT * 4 <= ST * Bytes, "the groups' sums");
};

// Wait until at most N of the wave's vector memory requests and none of its LDS
// reads are outstanding, then for the other waves.
template <int N>
__device__ inline void wait_stage() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | 0x0070 | ((N >> 4) << 14));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef const __attribute__((address_space(1))) uint8_t glb_u8;

// Where 16-byte piece p of row r of a stage lies in its row.  A read of 16 bytes a
// lane is served 16 lanes at a time, and those are not neighbours: lanes 0-3,
// 12-15, 20-23 and 24-27 go together (4-11, 16-19 and 28-31 next, and so on), that
// is rows 0-3 and 12-15 for one lane group and rows 4-11 for the next, whose piece
// lies DELTA (a power of two) further.  With DELTA taken back for rows 4-11 the 16
// rows' pieces cover all 64 banks.  (Rows in plain order instead, as 16 neighbours
// would want them: two lanes to a bank in each of these reads.)
template <int ROW, int DELTA>
__device__ inline int swizzle(int r, int p) {
  const int base = ROW == 64 ? (r >> 2) & 3 : ROW == 128 ? (r >> 1) & 7 : r & 15;
  return p ^ base ^ ((((r >> 2) ^ (r >> 3)) & 1) * DELTA);
}

template <int ACT, int MATS, int BR, int BT, int WR, int WT, int WK, int ST>
__global__ __launch_bounds__(WR* WT* WK* kWave) void k_mx_tile(LinArgs a) {
  using P = Tile<ACT, MATS, BR, BT, WR, WT, WK, ST>;
  constexpr int NW = P::NW, R = P::R, T = P::T, SK = P::SK;
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
  const int stages_all = a.steps / SK;
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
    ow[i] = (uint32_t)(rr * (int)pitch_q) + 16 * swizzle<P::WRow, P::WDelta>(r, lane % (64 / LW));
    bw[i] = a.q[MATS == 2 ? uniform(mat) : 0] + (size_t)row0 * pitch_q;
  }
#pragma unroll
  for (int i = 0; i < P::IX / NW; ++i) {
    const int r = (wv + NW * i) * LX + lane / (64 / LX);
    const int rr = min(tok0 + r, a.m - 1) - tok0;
    ox[i] = (uint32_t)rr * (uint32_t)a.ldx + 16 * swizzle<P::XRow, P::XDelta>(r, lane % (64 / LX));
  }
  const uint8_t* bx = static_cast<const uint8_t*>(a.x) + (size_t)tok0 * a.ldx;
  constexpr int NS = P::NS, MS = P::MS;  // scale requests of a stage; waves without one repeat another's
  uint32_t os[MS];
  const uint8_t* bs[MS];
#pragma unroll
  for (int i = 0; i < MS; ++i) {
    const int q = (wv + NW * i) % NS;
    const bool of_x = q >= P::IWs;
    const int r = (of_x ? q - P::IWs : q) * (64 / SK) + lane / SK;  // one 4-byte word a lane
    const int base = of_x ? tok0 : row0, last = (of_x ? a.m : a.rows) - 1;
    const int per = of_x ? BT : BR / MATS;
    const int rr = min(base + r % per, last) - base;
    os[i] = (uint32_t)(rr * (int)pitch_s) + 4 * (lane % SK);
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
      __builtin_amdgcn_global_load_lds((glb_u8*)(bs[i] + (size_t)k * P::SRow + os[i]),
                                       (lds_u8*)(to + P::WBytes + P::XBytes + (wv + NW * i) % NS * 256), 4, 0, 0);
  };

  const int wk = wv / (WR * WT), wr = wv / WT % WR, wt = wv % WT;
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
        sw[i] = *reinterpret_cast<const uint16_t*>(sl + (piece_row(i) + r) * P::SRow + 8 * wk + 2 * g);
#pragma unroll
      for (int t = 0; t < T; ++t)
        sx[t] = *reinterpret_cast<const uint16_t*>(sl + P::WsBytes + (wt * (BT / WT) + t * 16 + r) * P::SRow +
                                                 8 * wk + 2 * g);
      // step s: lane group g takes block 2 g + s of the wave's 8
      u32x4 w[R], x[T];
      auto read = [&](int s) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
          const int row = wt * (BT / WT) + t * 16 + r;
          x[t] = *reinterpret_cast<const u32x4*>(xl + row * P::XRow + 16 * swizzle<P::XRow, P::XDelta>(row, 8 * wk + 2 * g + s));
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const int row = piece_row(i) + r;
          w[i] = *reinterpret_cast<const u32x4*>(wl + row * P::WRow + 16 * swizzle<P::WRow, P::WDelta>(row, 8 * wk + 2 * g + s));
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
        w[i] = *reinterpret_cast<const u32x4*>(wl + row * P::WRow + 16 * swizzle<P::WRow, P::WDelta>(row, 4 * wk + g));
        sw[i] = mx_scale(sl[row * P::SRow + 4 * wk + g]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 x[T];
#pragma unroll
        for (int t = 0; t < T; ++t) {
          const int row = wt * (BT / WT) + t * 16 + r;
          x[t] = *reinterpret_cast<const u32x4*>(xl + row * P::XRow + 16 * swizzle<P::XRow, P::XDelta>(row, 16 * wk + 4 * g + j));
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
  // one stage computed while the requests of the next ST - 1 are in flight; the
  // parts of LDS are told apart by the pointers' restrict, without which every
  // read of LDS would wait for all requests
  auto step = [&](uint8_t* __restrict__ to, const uint8_t* __restrict__ from, int k, bool more) {
    if (more) request(to, k);
    compute(from);
  };

#pragma unroll
  for (int i = 0; i < ST - 1; ++i)
    if (k_first + i < k_last) request(lds + i * P::Bytes, k_first + i);
  int cur = 0;
  for (int k = k_first; k < k_last; ++k) {
    // stage k is in LDS, and every wave has left the part that k + ST - 1 goes to
    if (k + ST - 2 < k_last)
      wait_stage<P::Requests * (ST - 2)>();
    else
      wait_stage<0>();
    const int nxt = cur == 0 ? ST - 1 : cur - 1;
    step(lds + nxt * P::Bytes, lds + cur * P::Bytes, k + ST - 1, k + ST - 1 < k_last);
    cur = cur == ST - 1 ? 0 : cur + 1;
  }
  if constexpr (WK > 1) {
    // the groups' sums, added by the first one
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(lds) + (wv % (WR * WT)) * kWave + lane;
#pragma unroll
    for (int q = 1; q < WK; ++q)
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < T; ++t)
          if (wk == q) sums[(((q - 1) * R + i) * T + t) * (WR * WT * kWave)] = acc[i][t];
    __syncthreads();
    if (wk != 0) return;
#pragma unroll
    for (int q = 1; q < WK; ++q)
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[i][t] += sums[(((q - 1) * R + i) * T + t) * (WR * WT * kWave)];
  }
  if (SK > 1 && part == a.split - 1) {
    // the last steps that do not fill a stage, straight from memory
    for (int k = stages_all * SK; k < a.steps; ++k) {
      constexpr int XV = ACT == kActMx ? 1 : 4;
      u32x4 x[T][XV];
      uint32_t sx[T];
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const size_t tok = min(tok0 + wt * (BT / WT) + t * 16 + r, a.m - 1);
        const uint8_t* xp = static_cast<const uint8_t*>(a.x) + tok * a.ldx + (size_t)k * (64 * XV) + g * (16 * XV);
#pragma unroll
        for (int j = 0; j < XV; ++j) x[t][j] = *reinterpret_cast<const u32x4*>(xp + 16 * j);
        sx[t] = ACT == kActMx ? a.xs[tok * pitch_s + (size_t)k * 4 + g] : 0u;
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        asm volatile("" ::: "memory");  // one piece's codes at a time: the registers are the sums'
        const int tr = piece_row(i) + r;
        const size_t row = min(row0 + tr % (BR / MATS), a.rows - 1);
        const int mat = MATS == 2 ? i / (R / 2) : 0;
        const u32x4 w = *reinterpret_cast<const u32x4*>(a.q[mat] + row * pitch_q + (size_t)k * 64 + g * 16);
        const uint32_t sw = a.s[mat][row * pitch_s + (size_t)k * 4 + g];
#pragma unroll
        for (int t = 0; t < T; ++t) {
          if constexpr (ACT == kActMx) {
            acc[i][t] = mfma_mx<0, 0>(w, x[t][0], acc[i][t], sw, sx[t]);
          } else {
#pragma unroll
            for (int j = 0; j < XV; ++j)
              acc[i][t] = mfma_half(ACT == kActBF16, mx_half8<ACT == kActBF16>(w[j], mx_scale(sw)), x[t][j], acc[i][t]);
          }
        }
      }
    }
  }

  // a lane holds rows 4 g .. 4 g + 3 of each piece for token r of each
  auto put = [&](auto dtype, void* y, int i, int t, f32x4 v) {
    constexpr int DT = decltype(dtype)::value;
    const int row = row0 + piece_row(i) % (BR / MATS) + 4 * g;
    const int tok = tok0 + wt * (BT / WT) + t * 16 + r;
    if (tok >= a.m || row >= a.rows) return;
    const size_t at = (size_t)tok * a.rows + row;
    if ((a.rows & 3) == 0) {
      if constexpr (DT == kF32)
        *reinterpret_cast<f32x4*>(static_cast<float*>(y) + at) = v;
      else if constexpr (DT == kBF16)
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(y) + at) = u32x2{pack_bf2(v.x, v.y), pack_bf2(v.z, v.w)};
      else
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(y) + at) = u32x2{pack_f2(v.x, v.y), pack_f2(v.z, v.w)};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (row + e < a.rows) store_one(y, at + e, DT, v[e]);
    }
  };
  auto finish = [&](auto dtype) {
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
        put(dtype, a.y, i, t, v);
      }
  };
  if (a.part) {
    const size_t mat_size = (size_t)a.m * a.rows;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int mat = MATS == 2 ? i / (R / 2) : 0;
#pragma unroll
      for (int t = 0; t < T; ++t)
        put(std::integral_constant<int, kF32>{}, a.part + (size_t)(part * MATS + mat) * mat_size, i, t, acc[i][t]);
    }
  } else if (a.y_dtype == kF32) {
    finish(std::integral_constant<int, kF32>{});
  } else if (a.y_dtype == kBF16) {
    finish(std::integral_constant<int, kBF16>{});
  } else {
    finish(std::integral_constant<int, kF16>{});
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

// The tiles, by size: rows of W, tokens, steps of a stage.
struct Shape {
  int br, bt, sk;
};
constexpr Shape kHalfTiles[] = {{32, 16, 4},  {64, 16, 4},  {128, 16, 2}, {64, 32, 4},  {128, 32, 2},
                                {128, 48, 2}, {128, 64, 2}, {256, 64, 2}, {256, 64, 1}};
constexpr Shape kMxTiles[] = {{32, 16, 8},  {64, 16, 8},   {64, 32, 4},   {64, 64, 4},
                              {128, 64, 4}, {128, 128, 4}, {128, 128, 2}, {256, 256, 2}};
constexpr int kHalfSmall = 8, kMxSmall = 6;  // those for at most a block a compute unit
constexpr long kBlocks = 256;  // compute units

struct Plan {
  bool pad;   // x is copied into the workspace first
  int tile;   // -1: k_mx_skinny
  int split;
  size_t pad_bytes, part_bytes;
};

// Whether x is copied first: rows that end inside 128 values or start off 16 bytes.
bool copies_x(const MxLinear& c) {
  return !c.xq && (c.n % kMxPad != 0 || c.ldx % 8 != 0 || (reinterpret_cast<uintptr_t>(c.x) & 15u) != 0);
}

int act_of(const MxLinear& c) { return c.xq ? kActMx : c.x_dtype == kBF16 ? kActBF16 : kActF16; }

// Which kernel.  With one block a compute unit a tile's time is set by what it
// streams, so the smallest tile whose blocks are at most the compute units is
// the fastest (4096 x 4096, 64 tokens, us: 64 x 16 in 256 blocks 7.9, 64 x 32 in
// 128 10.8, 64 x 64 in 64 16.8; 11008 x 4096, 128 tokens: 128 x 64 in 172 blocks
// 23.5, 64 x 32 in 688 28.8).  Products too large for that take tiles two of which
// share a compute unit, so that one's products cover the other's waits (256 x 64
// against one 256 x 128: 4096 x 4096, 4096 tokens, 117 against 121, 11008 x 4096,
// 700 tokens, 65 against 116), and with 4-bit activations 256 x 256 where those
// fill three quarters of their rounds (13824 x 5120, 4096 tokens: 200 against 208
// with 128 x 128; 4096 x 4096, 2048 tokens, half a round: 41 against 28).  With up
// to 64 tokens they take the tile that pads them least, with the most rows.
// Fewer than half as many blocks with a long n share it out (4096 x 11008, 16 tokens: 12.8
// in one part, 12.1 in two; 512 x 11008, 10 tokens: 14.7 / 10.2 in four), at the
// price of a second launch, so only where a part keeps five stages.
// k_mx_skinny takes 16 rows a block: up to 4 tokens over at most 256 blocks, both
// matrices counted (4096 x 11008: one token 7.9 against 11.5, 4 tokens 9.7
// against 11.6, 8 tokens 14.7 against 12.2; 11008 x 4096, one token: 9.5 against
// 8.1).
Plan plan_of(const MxLinear& c) {
  Plan p;
  const int np = mx_padded(c.n), mats = c.q_up ? 2 : 1, act = act_of(c);
  p.pad = copies_x(c);
  p.pad_bytes = p.pad ? align256((size_t)c.m * np * 2) : 0;
  p.split = 1;
  p.tile = -1;
  if (c.m > kSToks || (long)c.rows * mats > 16 * kBlocks) {
    const Shape* tiles = act == kActMx ? kMxTiles : kHalfTiles;
    const int small = act == kActMx ? kMxSmall : kHalfSmall;
    auto blocks = [&](const Shape& t) {
      return (long)((c.rows + t.br / mats - 1) / (t.br / mats)) * ((c.m + t.bt - 1) / t.bt);
    };
    for (int i = 0; i < small && p.tile < 0; ++i)
      if (blocks(tiles[i]) <= kBlocks) p.tile = i;
    if (p.tile < 0) {
      p.tile = small;
      if (c.m <= 64) {
        for (int i = 0; i < small; ++i)
          if (tiles[i].bt >= c.m && tiles[i].bt <= tiles[p.tile].bt) p.tile = i;
      } else if (act == kActMx) {
        const long b = blocks(tiles[small + 1]), rounds = (b + kBlocks - 1) / kBlocks;
        if (4 * b >= 3 * rounds * kBlocks) p.tile = small + 1;
      }
    }
    const Shape& t = tiles[p.tile];
    const long n_blocks = blocks(t), stages = np / kMxPad / t.sk;
    if (n_blocks * 2 <= kBlocks) p.split = (int)std::max(1l, std::min(kBlocks / n_blocks, std::min(stages / 5, 8l)));
  }
  p.part_bytes = p.split > 1 ? (size_t)p.split * mats * c.m * c.rows * sizeof(float) : 0;
  return p;
}

template <int ACT, int MATS, int BR, int BT, int WR, int WT, int WK, int ST>
hipError_t tile_launch(LinArgs a, hipStream_t s) {
  using P = Tile<ACT, MATS, BR, BT, WR, WT, WK, ST>;
  static std::atomic<int> attr_set[kMaxDevices];
  const int ok = per_device_once(attr_set, [](int) -> int {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_mx_tile<ACT, MATS, BR, BT, WR, WT, WK, ST>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, ST * P::Bytes) == hipSuccess ? 1 : -1;
  });
  if (ok != 1) return hipErrorInvalidConfiguration;
  a.row_tiles = (a.rows + BR / MATS - 1) / (BR / MATS);
  a.tok_tiles = (a.m + BT - 1) / BT;
  k_mx_tile<ACT, MATS, BR, BT, WR, WT, WK, ST>
      <<<(unsigned)(a.row_tiles * a.tok_tiles * a.split), WR * WT * WK * kWave, ST * P::Bytes, s>>>(a);
  return hipGetLastError();
}

template <int ACT, int MATS>
hipError_t linear_launch(const LinArgs& a, const Plan& p, hipStream_t s) {
  if (p.tile < 0) {
    // the kernel's dynamic LDS limit, set once per device
    static std::atomic<int> attr_set[kMaxDevices];
    const int ok = per_device_once(attr_set, [](int) -> int {
      return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_mx_skinny<ACT, MATS>),
                                 hipFuncAttributeMaxDynamicSharedMemorySize,
                                 kSToks * skinny_pitch(kSChunk)) == hipSuccess ? 1 : -1;
    });
    if (ok != 1) return hipErrorInvalidConfiguration;
    const int lds = ACT == kActMx ? 0 : a.m * skinny_pitch(a.steps);
    k_mx_skinny<ACT, MATS><<<(unsigned)((a.rows + 15) / 16), kSW * kWave, lds, s>>>(a);
    return hipGetLastError();
  }
  hipError_t e = hipErrorInvalidValue;
#define SI_TILE(I, TILES, WR, WT, WK, ST)                                                    \
  case I: {                                                                                  \
    static_assert(TILES[I].sk == WK * (ACT == kActMx ? 2 : 1), "steps of a stage");          \
    e = tile_launch<ACT, MATS, TILES[I].br, TILES[I].bt, WR, WT, WK, ST>(a, s);              \
    break;                                                                                   \
  }
  if constexpr (ACT == kActMx) {
    switch (p.tile) {
      SI_TILE(0, kMxTiles, 1, 1, 4, 3)
      SI_TILE(1, kMxTiles, 2, 1, 4, 3)
      SI_TILE(2, kMxTiles, 2, 1, 2, 4)
      SI_TILE(3, kMxTiles, 2, 2, 2, 3)
      SI_TILE(4, kMxTiles, 2, 2, 2, 3)
      SI_TILE(5, kMxTiles, 2, 2, 2, 2)
      SI_TILE(6, kMxTiles, 2, 2, 1, 2)
      SI_TILE(7, kMxTiles, 2, 4, 1, 2)
    }
  } else {
    switch (p.tile) {
      SI_TILE(0, kHalfTiles, 1, 1, 4, 3)
      SI_TILE(1, kHalfTiles, 2, 1, 4, 3)
      SI_TILE(2, kHalfTiles, 4, 1, 2, 4)
      SI_TILE(3, kHalfTiles, 2, 1, 4, 2)
      SI_TILE(4, kHalfTiles, 4, 1, 2, 3)
      SI_TILE(5, kHalfTiles, 4, 1, 2, 3)
      SI_TILE(6, kHalfTiles, 4, 1, 2, 3)
      SI_TILE(7, kHalfTiles, 4, 1, 2, 2)
      SI_TILE(8, kHalfTiles, 4, 1, 1, 2)
    }
  }
#undef SI_TILE
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
  // past 256 blocks, and with half the rows where there are two matrices: from 65
  // tokens tiles of at least 64 x 64 and 256 threads, else of 32 x 16 and 512; and
  // the copy where x needs one: fewer than 2^32 threads a launch
  const double r = c.rows, m = c.m;
  const double threads = c.m > 64 ? (r / 64 + 1) * (m / 64 + 1) * 256 : (r / 32 + 1) * (m / 16 + 1) * 512;
  return threads < 4294967296.0 && (!copies_x(c) || m * (mx_padded(c.n) / 8) < 4294967296.0);
}

size_t mx_linear_workspace(const MxLinear& c) {
  const Plan p = plan_of(c);
  return p.pad_bytes + p.part_bytes;
}

int mx_linear_tile(const MxLinear& c) { return plan_of(c).tile; }

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
