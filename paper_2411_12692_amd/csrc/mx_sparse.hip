// The predicted sparse MLP of 1 to 8 tokens with MXFP4 weights: Eq. (1) over the
// rows that Eq. (2) (or a caller's mask) keeps, in two launches.
//
// k_mx_rows: a block owns 32 rows.  It counts the sign products of its rows from
// the packed signs (lane = row and half of the units), applies Eq. (2) as N_neg <
// T, writes the mask and the rows' kept bits, and runs gate/up of the kept rows,
// a wave to a row: 16 bytes a lane hold one block of 32 codes, turned into fp16
// exactly (a code has two significant bits), multiplied with the tokens in LDS by
// two-way dot products in fp32, and scaled once a block, so every scale byte is
// exact.  W_up is requested with W_gate where the row is surely kept, otherwise
// only when some token's gate value is positive.  h3 goes to the workspace.
//
// k_mx_down: block (tile of 512 columns, chunk of row groups) adds h3_i *
// W_down^T[i, tile] over the kept rows of its chunk in registers, folds its
// waves in LDS and leaves the chunk's tile in the workspace; the last block of a
// tile to finish adds the chunks in their order.  No sum depends on which block
// came first: y is the same bits in every run.
//
// Bound at one token by two launches' latency chains (signs, gate/up; h3, down,
// fold, sum), not by the bytes.
#include "layer_common.h"
#include "mx.h"
#include "mx_launch.h"

namespace si {

constexpr int kMG = 32;      // rows of a block of k_mx_rows
constexpr int kMW = 8;       // waves of a block
constexpr int kMT = kMW * kWave;
// header words of the workspace that no other call uses: chunks of each tile of y
// that are done (zero between calls)
constexpr int kHdrDone = 16;
static_assert(kHdrDone > H_H3_FORM && kHdrDone + kMaxD / kTile <= H_WORDS, "a counter for each tile");
constexpr int kDownTarget = 512;  // blocks that k_mx_down aims at

inline __host__ __device__ int mx_groups(int k) { return (k + kMG - 1) / kMG; }
inline __host__ __device__ int mx_tiles(int d) { return (d + kTile - 1) / kTile; }
// chunks of row groups a tile of y is summed from
inline __host__ __device__ int mx_chunks(int k, int d) {
  const int g = mx_groups(k), c = kDownTarget / mx_tiles(d) < 64 ? kDownTarget / mx_tiles(d) : 64;
  return g < c ? g : c;
}

// Behind the workspace's common part, at offsets that depend on b: nothing here is
// read before the same call wrote it.  What has to last from call to call (the
// tiles' counters) is in the header, which lies the same for every b.
struct MxWs {
  size_t kmask;   // uint32 [groups] kept bits
  size_t counts;  // int32 [groups][2] rows whose W_up / W_down^T row was read
  size_t part;    // float [chunks][b][d]
  size_t total;
};
static MxWs mx_ws(int k, int d, int b) {
  MxWs L;
  L.kmask = ws_layout(k, b).total;
  L.counts = L.kmask + align256((size_t)mx_groups(k) * 4);
  L.part = L.counts + align256((size_t)mx_groups(k) * 8);
  L.total = L.part + align256((size_t)mx_chunks(k, d) * b * d * 4);
  return L;
}
size_t mx_mlp_workspace(int k, int d, int b) { return mx_ws(k, d, b).total; }

// Tokens in LDS: 8-value piece j of unit u (32 values) of token t at
// xs[(t * 4 + j) * U + u], so that lanes with neighbouring units read
// neighbouring 16 bytes.

// The codes and scales of a row, unit lane + 64 j; lanes past the row's end
// hold zero codes.
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
    r.c[j] = load_nt(qr + u);
    r.s[j] = sr[u];
  }
}
template <int B, int NU>
__device__ inline void mx_dots(const MxRow<NU>& r, const u32x4* xs, int U, int lane, float (&out)[B]) {
#pragma unroll
  for (int t = 0; t < B; ++t) out[t] = 0.f;
#pragma unroll
  for (int j = 0; j < NU; ++j) {
    const int u = lane + kWave * j;
    if (u < U) {
      u32x4 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = mx_half8<false>(r.c[j][i], 1.0f);
      const float sc = mx_factor(r.s[j]);
#pragma unroll
      for (int t = 0; t < B; ++t) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) a = dot8(w[i], xs[(t * 4 + i) * U + u], a);
        out[t] = fmaf(a, sc, out[t]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < B; ++t) out[t] = wave_total(out[t]);
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
  uint32_t* kmask;
  int32_t* counts;
  uint32_t* done;
  float* part;
  float* h3;
  float* y;
  int32_t* idx;
  int32_t* n_out;
  int32_t* counters;
  int groups, tiles, chunks;
};

template <int B, int NU>
__global__ __launch_bounds__(kMT) void k_mx_rows(MxArgs a) {
  extern __shared__ u32x4 xs[];  // [B][4][U]
  __shared__ __attribute__((aligned(16))) uint32_t xw[B * (kMaxD / 32)];
  __shared__ int cnt[kMW][B][kWave];
  __shared__ uint32_t kept[kMG];  // sure << 31 | row
  __shared__ int s_n, s_up, s_down;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int U = a.d >> 5;
  const int v = blockIdx.x;

  for (int i = tid; i < B * U * 4; i += kMT) {
    const int t = i / (U * 4), p = i - t * (U * 4);
    xs[(t * 4 + (p & 3)) * U + (p >> 2)] = a.x[i];
  }
  if (tid == 0) {
    s_up = 0;
    s_down = 0;
    if (v == 0) a.hdr[H_H3_FORM] = kH3PlainByRow;
  }
  __syncthreads();
  if (a.signs) {
    for (int i = tid; i < B * U; i += kMT) {
      const int t = i / U, u = i - t * U;
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) w |= sign_byte(xs[(t * 4 + j) * U + u]) << (8 * j);
      xw[i] = w;
    }
    __syncthreads();
    int c[B];
#pragma unroll
    for (int t = 0; t < B; ++t) c[t] = 0;
    const int kpad = row_groups(a.k) * kRowGroup;
    const int units = U >> 2;
    const u32x4* sg = a.signs + (size_t)v * kMG + (lane & (kMG - 1));
#pragma unroll 4
    for (int q = 2 * wv + (lane >> 5); q < units; q += 2 * kMW) {
      const u32x4 s = load_nt(sg + (size_t)q * kpad);
#pragma unroll
      for (int t = 0; t < B; ++t) {
        const u32x4 xv = *reinterpret_cast<const u32x4*>(&xw[t * U + 4 * q]);
        c[t] += __popc(s.x ^ xv.x) + __popc(s.y ^ xv.y) + __popc(s.z ^ xv.z) + __popc(s.w ^ xv.w);
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
    if (lane == 0) {
      s_n = __popcll(ballot);
      a.kmask[v] = (uint32_t)ballot;
    }
  }
  __syncthreads();
  const int n = s_n;
  const bool no_as = (a.flags & kNoAS) != 0, no_spec = (a.flags & kNoSpec) != 0;
  int n_up = 0, n_down = 0;
  for (int i = wv; i < n; i += kMW) {
    const uint32_t e = (uint32_t)uniform((int)kept[i]);
    const int row = (int)(e & 0x7fffffffu);
    const bool early = a.qu && (no_as || ((e >> 31) && !no_spec));
    MxRow<NU> rg, ru;
    mx_load_row<NU>(a.qg, a.sg, row, U, lane, rg);
    if (early) mx_load_row<NU>(a.qu, a.su, row, U, lane, ru);
    float g[B], h[B];
    mx_dots<B, NU>(rg, xs, U, lane, g);
    bool any = false;
#pragma unroll
    for (int t = 0; t < B; ++t) {
      g[t] = g[t] > 0.f || g[t] != g[t] ? g[t] : 0.f;  // ReLU that keeps a NaN
      any |= g[t] != 0.f;
      h[t] = a.qu ? 0.f : g[t];
    }
    if (a.qu && (early || any)) {
      if (!early) mx_load_row<NU>(a.qu, a.su, row, U, lane, ru);
      float u[B];
      mx_dots<B, NU>(ru, xs, U, lane, u);
#pragma unroll
      for (int t = 0; t < B; ++t) h[t] = g[t] != 0.f ? g[t] * u[t] : 0.f;  // as where the row is skipped
      ++n_up;
    }
    bool nz = no_as;
#pragma unroll
    for (int t = 0; t < B; ++t) nz |= h[t] != 0.f;
    n_down += nz ? 1 : 0;
#pragma unroll
    for (int t = 0; t < B; ++t)
      if (lane == t) a.h3[(size_t)row * B + t] = h[t];
  }
  if (a.counters) {
    if (lane == 0 && (n_up | n_down)) {
      atomicAdd(&s_up, n_up);
      atomicAdd(&s_down, n_down);
    }
    __syncthreads();
    if (tid == 0) {
      a.counts[2 * v] = s_up;
      a.counts[2 * v + 1] = s_down;
    }
  }
}

// The ascending list, its length and the work counters, from the groups' kept
// bits (one block, beside the down-projection's).
__device__ inline void mx_lists(const MxArgs& a, int* wsum) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  int base = 0, up = 0, down = 0;
  for (int g0 = 0; g0 < a.groups; g0 += kMT) {
    const int g = g0 + tid;
    uint32_t bits = g < a.groups ? a.kmask[g] : 0u;
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
      up += a.counts[2 * g];
      down += a.counts[2 * g + 1];
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

constexpr int kDownRows = 256;  // kept rows a block lists at a time
constexpr int kDownUnroll = 4;

template <int B>
__global__ __launch_bounds__(kMT) void k_mx_down(MxArgs a) {
  __shared__ float fold[kMW][kTile];
  __shared__ int rows[kDownRows + kMG];
  __shared__ float hs[kDownRows + kMG][B];
  __shared__ int wsum[kMW];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  if ((int)blockIdx.x == a.tiles * a.chunks) {
    mx_lists(a, wsum);
    return;
  }
  const int tile = blockIdx.x % a.tiles, chunk = blockIdx.x / a.tiles;
  const int g0 = (int)((long long)a.groups * chunk / a.chunks), g1 = (int)((long long)a.groups * (chunk + 1) / a.chunks);
  const int d = a.d, U = d >> 5;
  const int col = tile * kTile + lane * 8;  // the lane's first column
  const bool col_ok = col < d;
  const bool no_as = (a.flags & kNoAS) != 0;
  float acc[B][8];
#pragma unroll
  for (int t = 0; t < B; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[t][e] = 0.f;

  for (int gb = g0; gb < g1; gb += kDownRows / kMG) {
    // the kept rows of up to 8 groups, a wave to a group, with their h3
    const int g = gb + wv;
    uint32_t bits = g < g1 ? (uint32_t)uniform((int)a.kmask[g]) : 0u;
    const int row = g * kMG + lane;
    bool use = lane < kMG && ((bits >> (lane & 31)) & 1u);
    float h[B];
#pragma unroll
    for (int t = 0; t < B; ++t) h[t] = use ? a.h3[(size_t)row * B + t] : 0.f;
    bool nz = no_as;
#pragma unroll
    for (int t = 0; t < B; ++t) nz |= h[t] != 0.f;
    use = use && nz;
    const uint64_t ballot = __ballot(use);
    if (lane == 0) wsum[wv] = __popcll(ballot);
    __syncthreads();
    int at = 0, n = 0;
#pragma unroll
    for (int w = 0; w < kMW; ++w) {
      if (w < wv) at += wsum[w];
      n += wsum[w];
    }
    if (use) {
      at += __popcll(ballot & lanes_below(lane));
      rows[at] = row;
#pragma unroll
      for (int t = 0; t < B; ++t) hs[at][t] = h[t];
    }
    __syncthreads();
    for (int i0 = wv * kDownUnroll; i0 < n; i0 += kMW * kDownUnroll) {
      uint32_t c[kDownUnroll], s[kDownUnroll];
#pragma unroll
      for (int r = 0; r < kDownUnroll; ++r) {
        const int i = min(i0 + r, n - 1);
        const size_t rw = (size_t)uniform(rows[i]);
        c[r] = 0;
        s[r] = 0;
        if (col_ok) {
          c[r] = __builtin_nontemporal_load(a.qd + rw * (U * 4) + (col >> 3));
          s[r] = a.sd[rw * U + (col >> 5)];
        }
      }
#pragma unroll
      for (int r = 0; r < kDownUnroll; ++r) {
        if (i0 + r < n) {
          const float sc = mx_scale(s[r]);
          const f32x2 w0 = mx_f32x2<0>(c[r], sc), w1 = mx_f32x2<1>(c[r], sc), w2 = mx_f32x2<2>(c[r], sc),
                      w3 = mx_f32x2<3>(c[r], sc);
          const float w[8] = {w0.x, w0.y, w1.x, w1.y, w2.x, w2.y, w3.x, w3.y};
#pragma unroll
          for (int t = 0; t < B; ++t) {
            const float hv = hs[i0 + r][t];
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[t][e] = fmaf(hv, w[e], acc[t][e]);
          }
        }
      }
    }
    __syncthreads();
  }

  // fold the waves: thread = column of the tile
  const int mine = tile * kTile + tid;
  float* part = a.part + (size_t)chunk * B * d;
#pragma unroll
  for (int t = 0; t < B; ++t) {
#pragma unroll
    for (int e = 0; e < 8; ++e) fold[wv][lane * 8 + e] = acc[t][e];
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kMW; ++w) s += fold[w][tid];
    __syncthreads();
    if (mine < d) {
      if (a.chunks == 1)
        a.y[(size_t)t * d + mine] = s;
      else
        st_agent(reinterpret_cast<uint32_t*>(part + (size_t)t * d + mine), __float_as_uint(s));
    }
  }
  if (a.chunks == 1) return;
  wait_own_stores();
  __syncthreads();
  if (tid == 0) {
    const uint32_t before = __hip_atomic_fetch_add(&a.done[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = before == (uint32_t)a.chunks - 1u;
    if (s_last) st_agent(&a.done[tile], 0u);
  }
  __syncthreads();
  if (!s_last || mine >= d) return;
#pragma unroll
  for (int t = 0; t < B; ++t) {
    float s = 0.f;
    const uint32_t* p = reinterpret_cast<const uint32_t*>(a.part) + (size_t)t * d + mine;
#pragma unroll 8
    for (int q = 0; q < a.chunks; ++q) s += __uint_as_float(ld_agent(p + (size_t)q * B * d));
    a.y[(size_t)t * d + mine] = s;
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
  k_mx_down<B><<<a.tiles * a.chunks + (lists ? 1 : 0), kMT, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_mx_mlp(const MxMlpCall& c, hipStream_t s) {
  const WsLayout L = ws_layout(c.k, c.b);
  const MxWs M = mx_ws(c.k, c.d, c.b);
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
  a.kmask = reinterpret_cast<uint32_t*>(base + M.kmask);
  a.counts = reinterpret_cast<int32_t*>(base + M.counts);
  a.done = a.hdr + kHdrDone;
  a.part = reinterpret_cast<float*>(base + M.part);
  a.h3 = reinterpret_cast<float*>(base + L.h3);
  a.y = c.y;
  a.idx = c.idx;
  a.n_out = c.n_out;
  a.counters = c.counters;
  a.groups = mx_groups(c.k);
  a.tiles = mx_tiles(c.d);
  a.chunks = mx_chunks(c.k, c.d);
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
