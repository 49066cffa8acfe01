// The predicted sparse MLP of 1 to 8 tokens with MXFP4 weights: Eq. (1) over the
// rows that Eq. (2) (or a caller's mask) keeps, in two launches.
//
// k_mx_rows: a block owns 32 rows.  It counts the sign products of its rows from
// the packed signs (lane = row and half of the units), applies Eq. (2) as N_neg <
// T, writes the mask, and runs gate/up of the kept rows, a wave to a row: 16 bytes
// a lane hold one block of 32 codes, turned into fp16 exactly (a code has two
// significant bits), multiplied with the tokens in LDS by two-way dot products in
// fp32, and scaled once a block, so every scale byte is exact.  W_up is requested
// with W_gate where the row is surely kept, otherwise only when some token's gate
// value is positive.  h3 goes to the workspace, and a bit for each row whose h3 is
// not 0 for every token, in 64-bit words that no single-launch call takes for its
// own (si_device.h; as plain floats, half as many bytes to gather, the 7B-shaped
// layer's two launches took 13.1 us with one token and 30.9 with eight instead of
// 13.4 and 31.4).
//
// k_mx_down: a block owns 32 columns of y (16 with 5 to 8 tokens) over all rows: it
// lists the rows whose bit is set and its threads take one each, 16 bytes of codes
// (neighbouring columns lie on the same XCD, so a row's line is fetched into one L2
// and used by 8 blocks there).  The threads' sums meet in registers and LDS in a
// fixed order: no partial sums in memory, no atomics, and y is the same bits in
// every run.  (With tiles of 512 columns by chunks of rows and partial sums 13.2 us,
// the last block of a tile reading them alone.)
//
// Bound by the two launches' chains of round trips (signs, then rows; list, then
// pieces): 7B-shaped layer, one token, s = 0.9, 6.3 + 7.4 us for 12.8 MB (2.5 us of
// a copy's rate); with four tokens at 13B, 15.7 + 12.0, also by the dot products.
#include <type_traits>

#include "layer_common.h"
#include "mx.h"
#include "mx_launch.h"

namespace si {

constexpr int kMG = 32;      // rows of a block of k_mx_rows
constexpr int kMW = 8;       // waves of a block
constexpr int kMT = kMW * kWave;
// columns of y of a block of k_mx_down: one scale's where the sums of that many
// fit the registers (5120 wide, 1700 rows: one token 11.7 us with 16, 8.6 with 32,
// four tokens 14.0 and 12.0: every block asks its L2 for every row, so fewer, wider
// blocks ask less)
constexpr int down_cols(int b) { return b <= 4 ? 32 : 16; }
constexpr int kSignUnits = kMaxD / 128 / (2 * kMW);  // sign units of a lane (4)

inline __host__ __device__ int mx_groups(int k) { return (k + kMG - 1) / kMG; }

// The groups' row sets lie in the list region of the workspace (4 k bytes at an
// offset that is the same for every b; these calls keep no list there): two words a
// group of 32 rows, at most 16 (k / 32 + 1) bytes, which 4 k rounded up to 256 holds
// for every k.  A set is the low half of its word.

// Tokens in LDS: 8-value piece j of unit u (32 values) of token t at
// xs[(t * 4 + j) * U + u], so that lanes with neighbouring units read
// neighbouring 16 bytes.

// The codes and scales of a row, unit lane + 64 j.
template <int NU>
struct MxRow {
  u32x4 c[NU];
  uint32_t s[NU];
};
template <int NU>
__device__ inline void mx_load_row(const u32x4* __restrict__ q, const uint8_t* __restrict__ s, int row, int U,
                                   int lane, MxRow<NU>& r) {
  const u32x4* qr = q + (size_t)row * U;
  const uint8_t* sr = s + (size_t)row * U;
#pragma unroll
  for (int j = 0; j < NU; ++j) {
    const int u = min(lane + kWave * j, U - 1);
    r.c[j] = qr[u];
    r.s[j] = sr[u];
  }
}
// Dot products of MATS rows with the tokens, each token's values read once for
// all of them.
template <int B, int NU, int MATS>
__device__ inline void mx_dots(const MxRow<NU> (&r)[MATS], const u32x4* xs, int U, int lane, float (&out)[MATS][B]) {
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < B; ++t) out[m][t] = 0.f;
#pragma unroll
  for (int j = 0; j < NU; ++j) {
    const int u = lane + kWave * j;
    if (u < U) {
      float a[MATS][B];
#pragma unroll
      for (int m = 0; m < MATS; ++m)
#pragma unroll
        for (int t = 0; t < B; ++t) a[m][t] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x4 w[MATS];
#pragma unroll
        for (int m = 0; m < MATS; ++m) w[m] = mx_half8<false>(r[m].c[j][i], 1.0f);
#pragma unroll
        for (int t = 0; t < B; ++t) {
          const u32x4 x = xs[(t * 4 + i) * U + u];
#pragma unroll
          for (int m = 0; m < MATS; ++m) a[m][t] = dot8(w[m], x, a[m][t]);
        }
      }
#pragma unroll
      for (int m = 0; m < MATS; ++m) {
        const float sc = mx_factor(r[m].s[j]);
#pragma unroll
        for (int t = 0; t < B; ++t) out[m][t] = fmaf(a[m][t], sc, out[m][t]);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < B; ++t) out[m][t] = wave_total(out[m][t]);
}

struct MxArgs {
  const u32x4* signs;
  const u32x4* qg;
  const uint8_t* sg;
  const u32x4* qu;  // NULL: the non-gated ReLU MLP
  const uint8_t* su;
  const uint32_t* qd;
  const uint8_t* sd;
  const u32x4* x;
  const uint8_t* mask_in;
  uint8_t* mask;
  int k, d, T, margin;
  uint32_t flags;
  uint32_t* hdr;
  uint64_t* kmask;  // [groups] kept rows; high half: how many W_up rows were read
  uint64_t* dmask;  // [groups] rows whose W_down^T row is read; high half 0
  uint64_t* h3;     // [k][b] fp32 bits; high half 0
  float* y;
  int32_t* idx;
  int32_t* n_out;
  int32_t* counters;
  int groups, tiles;
};

template <int B, int NU>
__global__ __launch_bounds__(kMT) void k_mx_rows(MxArgs a) {
  extern __shared__ u32x4 xs[];  // [B][4][U]
  __shared__ __attribute__((aligned(16))) uint32_t xw[B * (NU * kWave)];
  __shared__ int cnt[kMW][B][kWave];
  __shared__ uint32_t kept[kMG];  // sure << 31 | row
  __shared__ uint32_t s_kept, s_down, s_up;
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6);
  const int U = a.d >> 5, units = U >> 2;
  const int v = blockIdx.x;
  // the signs are requested first: everything up to the counts hides behind them
  const int kpad = row_groups(a.k) * kRowGroup;
  u32x4 sg[kSignUnits];
  if (a.signs) {
    const u32x4* p = a.signs + (size_t)v * kMG + (lane & (kMG - 1));
#pragma unroll
    for (int i = 0; i < kSignUnits; ++i) {
      const int q = 2 * wv + (lane >> 5) + 2 * kMW * i;
      if (q < units) sg[i] = p[(size_t)q * kpad];
    }
  }
  // tokens to LDS with their sign bits (a byte for 8 values), all of a thread's
  // pieces in flight together
  uint8_t* xb = reinterpret_cast<uint8_t*>(xw);
  constexpr int XP = (NU * kWave * 4 + kMT - 1) / kMT;  // 16-byte pieces of a token a thread
  u32x4 xv[B][XP];
#pragma unroll
  for (int t = 0; t < B; ++t)
#pragma unroll
    for (int i = 0; i < XP; ++i) {
      const int p = tid + kMT * i;
      if (p < U * 4) xv[t][i] = a.x[(size_t)t * (U * 4) + p];
    }
#pragma unroll
  for (int t = 0; t < B; ++t)
#pragma unroll
    for (int i = 0; i < XP; ++i) {
      const int p = tid + kMT * i;
      if (p < U * 4) {
        xs[(t * 4 + (p & 3)) * U + (p >> 2)] = xv[t][i];
        xb[t * (U * 4) + p] = (uint8_t)sign_byte(xv[t][i]);
      }
    }
  if (tid == 0) {
    s_down = 0;
    s_up = 0;
    if (v == 0) a.hdr[H_H3_FORM] = kH3Untagged;
  }
  __syncthreads();
  if (a.signs) {
    int c[B];
#pragma unroll
    for (int t = 0; t < B; ++t) c[t] = 0;
#pragma unroll
    for (int i = 0; i < kSignUnits; ++i) {
      const int q = 2 * wv + (lane >> 5) + 2 * kMW * i;
      if (q < units) {
        const u32x4 s = sg[i];
#pragma unroll
        for (int t = 0; t < B; ++t) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(&xw[t * U + 4 * q]);
          c[t] += __popc(s.x ^ w.x) + __popc(s.y ^ w.y) + __popc(s.z ^ w.z) + __popc(s.w ^ w.w);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < B; ++t) cnt[wv][t][lane] = c[t];
    __syncthreads();
  }
  if (wv == 0) {
    const int row = v * kMG + lane;
    bool keep = false, sure = false;
    if (lane < kMG && row < a.k) {
      if (a.signs) {
#pragma unroll
        for (int t = 0; t < B; ++t) {
          int n_neg = 0;
#pragma unroll
          for (int w = 0; w < kMW; ++w) n_neg += cnt[w][t][lane] + cnt[w][t][lane + kMG];
          keep |= n_neg < a.T;
          sure |= n_neg < a.T - a.margin;
        }
        if (a.mask) a.mask[row] = keep ? 1 : 0;
      } else {
        keep = sure = a.mask_in[row] != 0;
      }
    }
    const uint64_t ballot = __ballot(keep);
    if (keep) kept[__popcll(ballot & lanes_below(lane))] = (uint32_t)row | (sure ? 0x80000000u : 0u);
    if (lane == 0) s_kept = (uint32_t)ballot;
  }
  __syncthreads();
  const int n = __popc(s_kept);
  const bool no_as = (a.flags & kNoAS) != 0, no_spec = (a.flags & kNoSpec) != 0;
  for (int i = wv; i < n; i += kMW) {
    const uint32_t e = (uint32_t)uniform((int)kept[i]);
    const int row = (int)(e & 0x7fffffffu);
    const bool early = a.qu && (no_as || ((e >> 31) && !no_spec));
    float g[B], u[B], h[B];
    bool up = early;
    if (early) {
      MxRow<NU> r[2];
      mx_load_row<NU>(a.qg, a.sg, row, U, lane, r[0]);
      mx_load_row<NU>(a.qu, a.su, row, U, lane, r[1]);
      float o[2][B];
      mx_dots<B, NU, 2>(r, xs, U, lane, o);
#pragma unroll
      for (int t = 0; t < B; ++t) {
        g[t] = o[0][t];
        u[t] = o[1][t];
      }
    } else {
      MxRow<NU> r[1];
      mx_load_row<NU>(a.qg, a.sg, row, U, lane, r[0]);
      float o[1][B];
      mx_dots<B, NU, 1>(r, xs, U, lane, o);
#pragma unroll
      for (int t = 0; t < B; ++t) g[t] = o[0][t];
    }
    bool any = false;
#pragma unroll
    for (int t = 0; t < B; ++t) {
      g[t] = g[t] > 0.f || g[t] != g[t] ? g[t] : 0.f;  // ReLU that keeps a NaN
      any |= g[t] != 0.f;
    }
    if (a.qu && !early && any) {
      up = true;
      MxRow<NU> r[1];
      mx_load_row<NU>(a.qu, a.su, row, U, lane, r[0]);
      float o[1][B];
      mx_dots<B, NU, 1>(r, xs, U, lane, o);
#pragma unroll
      for (int t = 0; t < B; ++t) u[t] = o[0][t];
    }
    bool nz = no_as;
#pragma unroll
    for (int t = 0; t < B; ++t) {  // as where the row is skipped: nothing of W_up where h1 is 0
      h[t] = !a.qu ? g[t] : g[t] != 0.f ? g[t] * u[t] : 0.f;
      nz |= h[t] != 0.f;
    }
#pragma unroll
    for (int t = 0; t < B; ++t)
      if (lane == t) a.h3[(size_t)row * B + t] = __float_as_uint(h[t]);
    if (lane == 0) {
      if (nz) atomicOr(&s_down, 1u << (row - v * kMG));
      if (up) atomicAdd(&s_up, 1u);
    }
  }
  __syncthreads();
  if (tid == 0) {
    a.kmask[v] = (uint64_t)s_up << 32 | s_kept;
    a.dmask[v] = s_down;
  }
}

// The ascending list, its length and the work counters, from the groups' kept
// bits (one block, beside the down-projection's).
__device__ inline void mx_lists(const MxArgs& a, int* wsum) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  int base = 0, up = 0, down = 0;
  for (int g0 = 0; g0 < a.groups; g0 += kMT) {
    const int g = g0 + tid;
    const uint64_t word = g < a.groups ? a.kmask[g] : 0u;
    uint32_t bits = (uint32_t)word;
    const int n = __popc(bits);
    const int incl = wave_incl_scan(n);
    if (lane == kWave - 1) wsum[wv] = incl;
    __syncthreads();
    int at = base + incl - n, all = 0;
    for (int w = 0; w < kMW; ++w) {
      if (w < wv) at += wsum[w];
      all += wsum[w];
    }
    base += all;
    if (a.idx) {
      while (bits) {
        a.idx[at++] = g * kMG + __builtin_ctz(bits);
        bits &= bits - 1;
      }
    }
    if (a.counters && g < a.groups) {
      up += (int)(word >> 32);
      down += __popc((uint32_t)a.dmask[g]);
    }
    __syncthreads();
  }
  if (a.counters) {
    up = wave_sum_int(up);
    down = wave_sum_int(down);
    if (lane == 0) wsum[wv] = up;
    __syncthreads();
    up = 0;
    for (int w = 0; w < kMW; ++w) up += wsum[w];
    __syncthreads();
    if (lane == 0) wsum[wv] = down;
    __syncthreads();
    down = 0;
    for (int w = 0; w < kMW; ++w) down += wsum[w];
    if (tid == 0) {
      a.counters[0] = base;
      a.counters[1] = up;
      a.counters[2] = down;
    }
  }
  if (a.n_out && tid == 0) *a.n_out = base;
}

constexpr int kDownSpan = kMT * kMG;  // rows that a block lists at a time (16384)
constexpr int kDownUnroll = 4;

// Sum over the wave's lanes of N values each (N a power of two): while there is
// more than one, a lane keeps half of them and gives the other half to the lane
// a power of two away.  Lane l ends with the total of value l % N.
template <int N>
__device__ inline float lanes_total(float (&v)[N], int lane) {
#pragma unroll
  for (int w = N / 2, m = 1; w >= 1; w /= 2, m *= 2) {
#pragma unroll
    for (int i = 0; i < w; ++i) {
      const bool odd = (lane & m) != 0;
      const float keep = odd ? v[2 * i + 1] : v[2 * i], give = odd ? v[2 * i] : v[2 * i + 1];
      v[i] = keep + __shfl_xor(give, m, kWave);
    }
  }
  float s = v[0];
#pragma unroll
  for (int m = N; m < kWave; m *= 2) s += __shfl_xor(s, m, kWave);
  return s;
}

template <int B>
__global__ __launch_bounds__(kMT) void k_mx_down(MxArgs a) {
  constexpr int CB = down_cols(B), CW = CB / 8;  // columns, words of codes
  __shared__ uint16_t rows[kDownSpan];
  __shared__ float fold[kMW][B][CB];
  __shared__ int wsum[kMW];
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6);
  if ((int)blockIdx.x == a.tiles) {
    mx_lists(a, wsum);
    return;
  }
  // each XCD a run of neighbouring tiles where their number allows
  int tile = blockIdx.x;
  if (a.tiles % 8 == 0) tile = (tile & 7) * (a.tiles >> 3) + (tile >> 3);
  const int U = a.d >> 5, col = tile * CB;
  typedef std::conditional_t<CW == 4, u32x4, u32x2> codes_t;
  const codes_t* qd = reinterpret_cast<const codes_t*>(a.qd) + tile;
  const uint8_t* sd = a.sd + (col >> 5);
  float acc[B][CB];
#pragma unroll
  for (int t = 0; t < B; ++t)
#pragma unroll
    for (int e = 0; e < CB; ++e) acc[t][e] = 0.f;

  for (int g0 = 0; g0 < a.groups; g0 += kMT) {
    uint32_t bits = g0 + tid < a.groups ? (uint32_t)a.dmask[g0 + tid] : 0u;
    const int incl = wave_incl_scan(__popc(bits));
    if (g0 > 0) __syncthreads();  // the last span's list is read
    if (lane == kWave - 1) wsum[wv] = incl;
    __syncthreads();
    int at = incl - __popc(bits), n = 0;
#pragma unroll
    for (int w = 0; w < kMW; ++w) {
      if (w < wv) at += wsum[w];
      n += wsum[w];
    }
    for (; bits; bits &= bits - 1) rows[at++] = (uint16_t)(tid * kMG + __builtin_ctz(bits));
    __syncthreads();
    // a thread takes every 512th row
    for (int i0 = tid; i0 < n; i0 += kMT * kDownUnroll) {
      codes_t c[kDownUnroll];
      uint32_t s[kDownUnroll];
      float h[kDownUnroll][B];
#pragma unroll
      for (int r = 0; r < kDownUnroll; ++r) {
        const int i = i0 + kMT * r;
        c[r] = codes_t{};
        s[r] = 0;
#pragma unroll
        for (int t = 0; t < B; ++t) h[r][t] = 0.f;
        if (i < n) {
          const size_t row = (size_t)g0 * kMG + rows[i];
          c[r] = qd[row * (U * 4 / CW)];
          s[r] = sd[row * U];
          const uint64_t* p = a.h3 + row * B;
          if constexpr (B == 1) {
            h[r][0] = __uint_as_float((uint32_t)p[0]);
          } else {
#pragma unroll
            for (int t = 0; t < B; t += 2) {
              const int o = t < B - 1 ? t : B - 2;  // the last two overlap where B is odd
              const u32x4 v = *reinterpret_cast<const u32x4_e8*>(p + o);
              h[r][o] = __uint_as_float(v.x);
              h[r][o + 1] = __uint_as_float(v.z);
            }
          }
        }
      }
#pragma unroll
      for (int r = 0; r < kDownUnroll; ++r) {
        if (i0 + kMT * r < n) {
          const float sc = mx_scale(s[r]);
#pragma unroll
          for (int p = 0; p < CW; ++p) {
            const f32x2 w0 = mx_f32x2<0>(c[r][p], sc), w1 = mx_f32x2<1>(c[r][p], sc), w2 = mx_f32x2<2>(c[r][p], sc),
                        w3 = mx_f32x2<3>(c[r][p], sc);
            const float w[8] = {w0.x, w0.y, w1.x, w1.y, w2.x, w2.y, w3.x, w3.y};
#pragma unroll
            for (int t = 0; t < B; ++t)
#pragma unroll
              for (int e = 0; e < 8; ++e) acc[t][8 * p + e] = fmaf(h[r][t], w[e], acc[t][8 * p + e]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < B; ++t) {
    const float s = lanes_total<CB>(acc[t], lane);
    if (lane < CB) fold[wv][t][lane] = s;
  }
  __syncthreads();
  if (tid < B * CB) {
    const int t = tid / CB, e = tid % CB;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kMW; ++w) s += fold[w][t][e];
    a.y[(size_t)t * a.d + col + e] = s;
  }
}

template <int B, int NU>
static hipError_t rows_launch(const MxArgs& a, hipStream_t s) {
  const size_t lds = (size_t)B * a.d * sizeof(uint16_t);
  // the kernel's dynamic LDS limit, set once per device
  static std::atomic<int> attr_set[kMaxDevices];
  const int ok = per_device_once(attr_set, [](int) -> int {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&k_mx_rows<B, NU>),
                               hipFuncAttributeMaxDynamicSharedMemorySize,
                               B * NU * kWave * kMxBlock * (int)sizeof(uint16_t)) == hipSuccess ? 1 : -1;
  });
  if (ok != 1) return hipErrorInvalidConfiguration;
  k_mx_rows<B, NU><<<a.groups, kMT, lds, s>>>(a);
  return hipGetLastError();
}

template <int B>
static hipError_t mlp_b(const MxArgs& a, hipStream_t s) {
  const int nu = (a.d / kMxBlock + kWave - 1) / kWave;
  hipError_t e = nu <= 1 ? rows_launch<B, 1>(a, s) : nu <= 2 ? rows_launch<B, 2>(a, s)
                 : nu <= 3 ? rows_launch<B, 3>(a, s) : rows_launch<B, 4>(a, s);
  if (e != hipSuccess) return e;
  const bool lists = a.idx || a.n_out || a.counters;
  k_mx_down<B><<<a.tiles + (lists ? 1 : 0), kMT, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_mx_mlp(const MxMlpCall& c, hipStream_t s) {
  const WsLayout L = ws_layout(c.k, c.b);
  char* base = static_cast<char*>(c.ws);
  MxArgs a;
  a.signs = reinterpret_cast<const u32x4*>(c.signs);
  a.qg = reinterpret_cast<const u32x4*>(c.q_gate);
  a.sg = c.s_gate;
  a.qu = reinterpret_cast<const u32x4*>(c.q_up);
  a.su = c.s_up;
  a.qd = reinterpret_cast<const uint32_t*>(c.q_down_t);
  a.sd = c.s_down_t;
  a.x = reinterpret_cast<const u32x4*>(c.x);
  a.mask_in = c.mask_in;
  a.mask = c.mask;
  a.k = c.k;
  a.d = c.d;
  a.T = c.T;
  a.margin = c.margin;
  a.flags = c.flags;
  a.hdr = reinterpret_cast<uint32_t*>(base);
  a.groups = mx_groups(c.k);
  a.kmask = reinterpret_cast<uint64_t*>(base + L.idx);
  a.dmask = a.kmask + a.groups;
  a.h3 = reinterpret_cast<uint64_t*>(base + L.h3e);
  a.y = c.y;
  a.idx = c.idx;
  a.n_out = c.n_out;
  a.counters = c.counters;
  a.tiles = c.d / down_cols(c.b);
  switch (c.b) {
    case 1: return mlp_b<1>(a, s);
    case 2: return mlp_b<2>(a, s);
    case 3: return mlp_b<3>(a, s);
    case 4: return mlp_b<4>(a, s);
    case 5: return mlp_b<5>(a, s);
    case 6: return mlp_b<6>(a, s);
    case 7: return mlp_b<7>(a, s);
    case 8: return mlp_b<8>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace si
