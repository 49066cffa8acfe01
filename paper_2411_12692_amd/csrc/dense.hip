// The dense products of the MLP and their gradients, as calls of the tiles of
// dense_tile.h:
//   y  = x W^T          A = W (kRow), B = x (kRow); W_down^T [k][d]: A kCol
//   g, u = x W_gate^T, x W_up^T in one launch, h = ReLU(g) * u in its epilogue
//   dg = [g > 0] dh u,  du = dh ReLU(g)   (k_gated_grad; of the whole MLP in the epilogue
//                                          of dh = dy W_down)
//   dx = dg W_gate + du W_up               one launch, its sum over both
//   dW_gate = dg^T x,  dW_up = du^T x      one launch, a batch of two
// Operands that cannot be read in 16-byte pieces (odd lengths, unaligned rows,
// another type) are copied into the workspace first, rows padded with zeros.
#include <algorithm>
#include <cmath>

#include "dense.h"

namespace si {

// Copies of matrices, rows of n values, with rows of whole 8, zeros behind the n-th, in
// fp16 or bf16: 8 values a thread, a matrix for each blockIdx.y.
struct PadJob {
  DenseMat src;
  size_t rows;
  int n, np;
  u32x4* out;
};
struct PadJobs {
  PadJob job[6];
  int count, type;
};

__global__ __launch_bounds__(256) void k_dense_pad(PadJobs jobs) {
  const PadJob& j = jobs.job[blockIdx.y];
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= j.rows * (size_t)(j.np / 8)) return;
  const size_t r = i / (j.np / 8);
  const int c = (int)(i - r * (j.np / 8)) * 8;
  u32x4 v = {0, 0, 0, 0};
  if (j.src.dtype == jobs.type && c + 8 <= j.n) {
    v = *reinterpret_cast<const u32x4_e2*>(static_cast<const uint16_t*>(j.src.p) + r * j.src.ld + c);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < j.n) {
        const float f = load_one(j.src.p, r * j.src.ld + c + e, j.src.dtype);
        const uint32_t h = (jobs.type == kF16 ? pack_f2(f, 0.f) : pack_bf2(f, 0.f)) & 0xffffu;
        v[e >> 1] |= h << (16 * (e & 1));
      }
  }
  j.out[i] = v;
}

// dg and du of `rows` values a token, in rows of rp (zeros behind), 8 values a
// thread.  UP: g and u are the two sums; else g is h = ReLU(g).  Both are operands of
// matrix products of 16-bit values and are rounded to 16 bits here, once; the sums are
// kept in float32 (in 16 bits they were another rounding of each gradient: error of
// dW_gate in bf16 0.0033 instead of 0.0024, the output's own rounding being 0.0017, and a
// forward product 10% faster).  Bound by memory: 2048 x 11008 bf16, 55 us, 5.7 TB/s.
template <bool UP>
__global__ __launch_bounds__(256) void k_gated_grad(DenseMat dh, DenseMat gate, DenseMat up, size_t m, int rows, int rp,
                                                    int type, u32x4* __restrict__ dg, u32x4* __restrict__ du) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= m * (size_t)(rp / 8)) return;
  const size_t t = i / (rp / 8);
  const int c = (int)(i - t * (rp / 8)) * 8;
  float d[8], g[8], u[8];
  auto load = [&](const DenseMat& a, float (&f)[8]) {
    if (a.dtype == kF32 && c + 8 <= rows) {
      const float* p = static_cast<const float*>(a.p) + t * a.ld + c;
      const u32x4 lo = *reinterpret_cast<const u32x4_e4*>(p), hi = *reinterpret_cast<const u32x4_e4*>(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = __uint_as_float(lo[e]);
        f[4 + e] = __uint_as_float(hi[e]);
      }
    } else if (a.dtype != kF32 && c + 8 <= rows) {
      const u32x4 v = *reinterpret_cast<const u32x4_e2*>(static_cast<const uint16_t*>(a.p) + t * a.ld + c);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t h = v[e >> 1] >> (16 * (e & 1));
        f[e] = a.dtype == kF16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)h) : __builtin_bit_cast(float, h << 16);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = c + e < rows ? load_one(a.p, t * a.ld + c + e, a.dtype) : 0.f;
    }
  };
  load(dh, d);
  load(gate, g);
  if constexpr (UP) load(up, u);
  uint32_t a[4], b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float x[2], y[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int k = 2 * e + j;
      gated_grad(d[k], g[k], UP ? u[k] : 1.f, x[j], y[j]);
      if (c + k >= rows) x[j] = y[j] = 0.f;
    }
    a[e] = type == kF16 ? pack_f2(x[0], x[1]) : pack_bf2(x[0], x[1]);
    if constexpr (UP) b[e] = type == kF16 ? pack_f2(y[0], y[1]) : pack_bf2(y[0], y[1]);
  }
  dg[i] = u32x4{a[0], a[1], a[2], a[3]};
  if constexpr (UP) du[i] = u32x4{b[0], b[1], b[2], b[3]};
}

// The parts of a split sum, added in their order, 4 values a thread; `batches`
// outputs one behind the other, or the two sums of a gated product.
template <int MATS>
__global__ __launch_bounds__(256) void k_dense_join(DenseArgs a, size_t size) {
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= size) return;
  const int batch = blockIdx.y, n = (int)min(size - i, (size_t)4);
  float v[MATS][4];
#pragma unroll
  for (int w = 0; w < MATS; ++w)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[w][e] = 0.f;
  for (int p = 0; p < a.split; ++p)
#pragma unroll
    for (int w = 0; w < MATS; ++w) {
      const float* src = a.part + (size_t)(p * a.parts_of + batch + w) * size + i;
      if (n == 4 && (size & 3) == 0) {
        const f32x4 f = *reinterpret_cast<const f32x4*>(src);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[w][e] += f[e];
      } else {
        for (int e = 0; e < n; ++e) v[w][e] += src[e];
      }
    }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (e >= n) break;
    float y = v[0][e];
    if constexpr (MATS == 2) {
      if (a.g) {
        a.g[i + e] = y;
        a.u[i + e] = v[MATS - 1][e];
      }
      y = (y > 0.f || y != y ? y : 0.f) * v[MATS - 1][e];
    } else if (a.relu) {
      y = y > 0.f || y != y ? y : 0.f;
    }
    store_one(a.c[batch], i + e, a.c_dtype, y);
  }
}

// The same for dh: dg and du, 4 values a thread of rows of ldc.
template <bool UP>
__global__ __launch_bounds__(256) void k_dense_join_grad(DenseArgs a) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int pieces = a.ldc / 4;
  if (i >= (size_t)a.N * pieces) return;
  const int n = (int)(i / pieces), m = (int)(i - (size_t)n * pieces) * 4;
  const size_t size = (size_t)a.M * a.N, in = (size_t)n * a.M + m;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < a.split; ++p)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (m + e < a.M) v[e] += a.part[(size_t)p * size + in + e];
  put_gated_grad<UP>(a, n, m, v, gated_piece<UP, false>(a, n, m));
}

namespace {

constexpr long kBlocks = 256;  // compute units
constexpr int kTypeE4M3 = 2;   // dense_few's type of values

int pad8(int n) { return (n + 7) / 8 * 8; }

bool needs_copy(const DenseMat& a, int type, int n) {
  return a.dtype != type || n % 8 != 0 || a.ld % 8 != 0 || (reinterpret_cast<uintptr_t>(a.p) & 15u) != 0;
}
size_t copy_bytes(const DenseMat& a, int type, size_t rows, int n) {
  return a.p && needs_copy(a, type, n) ? align256(rows * pad8(n) * 2) : 0;
}

// Replaces matrices that cannot be read in whole pieces by copies in the workspace,
// all of a call's in one launch.
class Copies {
 public:
  Copies(int type, char*& ws) : ws_(ws) { jobs_.type = type; }
  void add(DenseMat& a, size_t rows, int n) {
    if (!a.p || rows == 0 || !needs_copy(a, jobs_.type, n)) return;
    const int np = pad8(n);
    jobs_.job[jobs_.count++] = PadJob{a, rows, n, np, reinterpret_cast<u32x4*>(ws_)};
    a = DenseMat{ws_, jobs_.type, (size_t)np};
    const size_t all = rows * (np / 8);
    ws_ += align256(all * 16);
    most_ = std::max(most_, all);
  }
  hipError_t launch(hipStream_t s) const {
    if (jobs_.count == 0) return hipSuccess;
    k_dense_pad<<<dim3((unsigned)((most_ + 255) / 256), (unsigned)jobs_.count), 256, 0, s>>>(jobs_);
    return hipGetLastError();
  }

 private:
  char*& ws_;
  PadJobs jobs_ = {};
  size_t most_ = 0;
};

struct Plan {
  int tile, split;
  size_t part_bytes;
};

// Which tile, and in how many parts the sum is taken, by an estimate of the time:
// rounds of blocks over the compute units, each as long as its stages and what comes
// before and behind them, and the second launch that joins parts.  The times are
// kDenseTiles' and those of the join, fitted to 438 products of random sizes (5 to 6000
// tokens, 64 to 16384 rows, sums of 64 to 8192, every tile and split timed): the tile
// taken is 2 to 3% slower than the best one on average (over 419 others 3.0%, with times
// fitted to those 2.3%).  What is right of them is the order: 4096 x 4096 x 11008 is put at
// 183 us and takes 304, the three products of 333 tokens, 1371 x 509, at 5.5, 8.3 and 6.6 and
// take 13.9, 12.2 and 12.3.  Up to 4 tokens W's rows go
// through dense_few.hip (gate and up of 11008 x 4096, one token: 35.1 us in tiles, 27.7).
Plan plan_of(int M, int N, long K, int mats, int batches, int es, bool b_rows, bool few) {
  if (few && N <= kFewTokens) return {kDenseFew, 1, 0};
  Plan best = {-1, 1, 0};
  double best_t = 1e30;
  for (int i = b_rows ? 0 : 2; i < kDenseTileCount; ++i) {
    const DenseShape& t = kDenseTiles[i];
    const long blocks = (long)((M + t.bm / mats - 1) / (t.bm / mats)) * ((N + t.bn - 1) / t.bn) * batches;
    const int kp = 128 / es * t.wk;
    const long stages = (K + kp - 1) / kp;
    for (int split = 1; split <= 16; split *= 2) {
      if (split > 1 && stages < 4 * split) break;
      if ((double)blocks * split * t.threads >= 4294967296.0) break;  // threads of a launch
      const double full = (double)kBlocks * t.resident;
      const double rounds = std::ceil((double)blocks * split / full);
      double us = rounds * ((double)((stages + split - 1) / split) * t.stage_us + t.round_us);
      const double size = (double)M * N * mats * batches * 4;
      if (split > 1) us += 4.0 + size * (2 * split + 1) / 3.3e6;
      if (us < best_t) {
        best_t = us;
        best = {i, split, split > 1 ? align256((size_t)split * mats * batches * M * N * 4) : 0};
      }
    }
  }
  return best;
}

hipError_t join(const DenseArgs& a, int mats, int batches, hipStream_t s) {
  if (!a.part) return hipSuccess;
  const size_t size = (size_t)a.M * a.N;
  const dim3 grid((unsigned)((size + 1023) / 1024), (unsigned)batches);
  if (mats == 2)
    k_dense_join<2><<<grid, 256, 0, s>>>(a, size);
  else
    k_dense_join<1><<<grid, 256, 0, s>>>(a, size);
  return hipGetLastError();
}

Plan linear_plan(const DenseLinear& c) { return plan_of(c.rows, c.m, c.n, c.w_up.p ? 2 : 1, 1, 2, true, !c.transposed); }
Plan dx_plan(const DenseGrad& c) { return plan_of(c.n, c.m, (long)c.rows * (c.w_up.p ? 2 : 1), 1, 1, 2, true, c.transposed && !c.w_up.p); }
Plan dw_plan(const DenseGrad& c) {
  return c.transposed ? plan_of(c.rows, c.n, c.m, 1, 1, 2, false, false)
                      : plan_of(c.n, c.rows, c.m, 1, c.w_up.p ? 2 : 1, 2, false, false);
}
// of the whole MLP: dh = dy W_down, dW_down = dy^T h
Plan dh_plan(const DenseGrad& c) { return plan_of(c.rows, c.m, c.n, 1, 1, 2, true, false); }
Plan dw_down_plan(const DenseGrad& c) { return plan_of(c.rows, c.n, c.m, 1, 1, 2, false, false); }
Plan fp8_plan(const DenseFp8& c) { return plan_of(c.rows, c.m, c.n, c.q_up ? 2 : 1, 1, 1, true, true); }

size_t weight_copies(const DenseMat& w, const DenseMat& w_up, bool transposed, int type, int rows, int n) {
  const int r = transposed ? n : rows, c = transposed ? rows : n;
  return copy_bytes(w, type, r, c) + copy_bytes(w_up, type, r, c);
}

void set_plan(DenseArgs& a, const Plan& p, int parts_of, char* ws) {
  a.split = p.split;
  a.parts_of = parts_of;
  a.part = p.part_bytes ? reinterpret_cast<float*>(ws) : nullptr;
}

}  // namespace

#define TRY(e)                                     \
  do {                                             \
    if (hipError_t e_ = (e); e_ != hipSuccess) return e_; \
  } while (0)

size_t dense_linear_workspace(const DenseLinear& c) {
  return copy_bytes(c.x, c.type, c.m, c.n) + weight_copies(c.w, c.w_up, c.transposed, c.type, c.rows, c.n) +
         linear_plan(c).part_bytes;
}

hipError_t launch_dense_linear(const DenseLinear& c, hipStream_t s) {
  char* ws = static_cast<char*>(c.ws);
  DenseMat x = c.x, w = c.w, up = c.w_up;
  const int wr = c.transposed ? c.n : c.rows, wc = c.transposed ? c.rows : c.n;
  Copies copies(c.type, ws);
  copies.add(x, c.m, c.n);
  copies.add(w, wr, wc);
  copies.add(up, wr, wc);
  TRY(copies.launch(s));
  const Plan p = linear_plan(c);
  const int mats = up.p ? 2 : 1;
  DenseArgs a = {};
  a.a[0] = w.p;
  a.a[1] = up.p;
  a.b[0] = x.p;
  a.lda = w.ld * 2;
  a.ldb = x.ld * 2;
  a.M = c.rows;
  a.N = c.m;
  a.K = c.n;
  a.segs = 1;
  a.c[0] = c.y;
  a.c_dtype = c.y_dtype;
  a.relu = c.relu;
  a.g = c.g;
  a.u = c.u;
  set_plan(a, p, mats, ws);
  const int type = c.type == kBF16 ? 1 : 0;
  if (p.tile == kDenseFew) return dense_few(type, mats, a, s);
  TRY(mats == 2 ? dense_gated(type, a, p.tile, s) : c.transposed ? dense_cr(type, a, p.tile, s)
                                                                 : dense_rr(type, a, p.tile, s));
  return join(a, mats, 1, s);
}

size_t dense_grad_workspace(const DenseGrad& c) {
  const size_t one = align256((size_t)c.m * pad8(c.rows) * 2) * (c.up.p ? 2 : 1);
  const bool want_w = c.dw || c.dw_up, through = (c.dx || want_w) && c.m > 0;  // dg and du are asked for
  size_t b = 0, part = 0;
  if (c.down.p) {
    b += copy_bytes(c.dy, c.type, c.m, c.n);
    if (through) {
      b += copy_bytes(c.down, c.type, c.n, c.rows) + one;
      part = dh_plan(c).part_bytes;
    }
    if (c.dw_down) {
      b += copy_bytes(c.h, c.type, c.m, c.rows);
      part = std::max(part, dw_down_plan(c).part_bytes);
    }
  } else {
    b += c.gate.p ? one : copy_bytes(c.dy, c.type, c.m, c.rows);
  }
  if (want_w) b += copy_bytes(c.x, c.type, c.m, c.n);
  if (c.dx) {
    b += weight_copies(c.w, c.w_up, c.transposed, c.type, c.rows, c.n);
    part = std::max(part, dx_plan(c).part_bytes);
  }
  if (want_w) part = std::max(part, dw_plan(c).part_bytes);
  return b + part;
}

hipError_t launch_dense_grad(const DenseGrad& c, hipStream_t s) {
  char* ws = static_cast<char*>(c.ws);
  const int type = c.type == kBF16 ? 1 : 0;
  DenseMat d = c.dy, du = {};
  DenseMat x = c.x, w = c.w, up = c.w_up, down = c.down, h = c.h;
  const bool want_w = c.dw || c.dw_up, through = (c.dx || want_w) && c.m > 0;
  Copies copies(c.type, ws);
  const int rp = pad8(c.rows);
  const size_t bytes = align256((size_t)c.m * rp * 2);
  u32x4 *dg = nullptr, *dg_up = nullptr;
  auto take = [&] {  // room for dg and du
    dg = reinterpret_cast<u32x4*>(ws);
    ws += bytes;
    if (c.up.p) {
      dg_up = reinterpret_cast<u32x4*>(ws);
      ws += bytes;
    }
  };
  DenseMat dy = c.dy;
  if (c.down.p) {
    copies.add(dy, c.m, c.n);
    if (through) {
      copies.add(down, c.n, c.rows);
      take();
    }
    if (c.dw_down) copies.add(h, c.m, c.rows);
  } else if (c.gate.p) {
    take();
  } else {
    copies.add(d, c.m, c.rows);
  }
  if (want_w) copies.add(x, c.m, c.n);
  if (c.dx) {
    const int wr = c.transposed ? c.n : c.rows, wc = c.transposed ? c.rows : c.n;
    copies.add(w, wr, wc);
    copies.add(up, wr, wc);
  }
  TRY(copies.launch(s));
  if (c.down.p && through) {
    const Plan p = dh_plan(c);
    DenseArgs a = {};
    a.a[0] = down.p;
    a.b[0] = dy.p;
    a.lda = down.ld * 2;
    a.ldb = dy.ld * 2;
    a.M = c.rows;
    a.N = c.m;
    a.K = c.n;
    a.segs = 1;
    a.c[0] = dg;
    a.c_dtype = c.type;
    a.gate = c.gate.p;
    a.up = static_cast<const float*>(c.up.p);
    a.du = dg_up;
    a.ldc = rp;
    set_plan(a, p, 1, ws);
    TRY(dense_dh(type, a, p.tile, s));
    if (a.part) {
      const size_t all = (size_t)a.N * (rp / 4);
      const unsigned grid = (unsigned)((all + 255) / 256);
      if (a.up)
        k_dense_join_grad<true><<<grid, 256, 0, s>>>(a);
      else
        k_dense_join_grad<false><<<grid, 256, 0, s>>>(a);
      TRY(hipGetLastError());
    }
  } else if (!c.down.p && c.gate.p && c.m > 0) {
    const unsigned grid = (unsigned)(((size_t)c.m * (rp / 8) + 255) / 256);
    if (c.up.p)
      k_gated_grad<true><<<grid, 256, 0, s>>>(c.dy, c.gate, c.up, c.m, c.rows, rp, c.type, dg, dg_up);
    else
      k_gated_grad<false><<<grid, 256, 0, s>>>(c.dy, c.gate, c.up, c.m, c.rows, rp, c.type, dg, nullptr);
    TRY(hipGetLastError());
  }
  if (c.gate.p) {
    d = DenseMat{dg, c.type, (size_t)rp};
    du = DenseMat{dg_up, c.type, (size_t)rp};
  }
  if (c.dw_down) {
    const Plan p = dw_down_plan(c);
    DenseArgs a = {};
    a.a[0] = h.p;
    a.b[0] = dy.p;
    a.lda = h.ld * 2;
    a.ldb = dy.ld * 2;
    a.M = c.rows;
    a.N = c.n;
    a.K = c.m;
    a.segs = 1;
    a.c[0] = c.dw_down;
    a.c_dtype = c.type;
    set_plan(a, p, 1, ws);
    TRY(dense_cc(type, a, p.tile, 1, s));
    TRY(join(a, 1, 1, s));
  }
  if (c.dx) {
    const Plan p = dx_plan(c);
    DenseArgs a = {};
    a.a[0] = w.p;
    a.a[1] = up.p;
    a.b[0] = d.p;
    a.b[1] = du.p;
    a.lda = w.ld * 2;
    a.ldb = d.ld * 2;
    a.M = c.n;
    a.N = c.m;
    a.K = c.rows;
    a.segs = up.p ? 2 : 1;
    a.c[0] = c.dx;
    a.c_dtype = c.type;
    set_plan(a, p, 1, ws);
    TRY(p.tile == kDenseFew ? dense_few(type, 1, a, s) : c.transposed ? dense_rr(type, a, p.tile, s)
                                                                      : dense_cr(type, a, p.tile, s));
    TRY(join(a, 1, 1, s));
  }
  if (want_w) {
    const Plan p = dw_plan(c);
    DenseArgs a = {};
    a.K = c.m;
    a.segs = 1;
    a.c_dtype = c.type;
    int batches = 1;
    if (c.transposed) {
      a.a[0] = d.p;
      a.b[0] = x.p;
      a.lda = d.ld * 2;
      a.ldb = x.ld * 2;
      a.M = c.rows;
      a.N = c.n;
      a.c[0] = c.dw;
    } else {
      // both matrices' gradients, or the one that is asked for
      a.a[0] = a.a[1] = x.p;
      a.lda = x.ld * 2;
      a.ldb = d.ld * 2;
      a.M = c.n;
      a.N = c.rows;
      const void* of[2] = {d.p, du.p};
      void* to[2] = {c.dw, c.dw_up};
      batches = 0;
      for (int i = 0; i < 2; ++i)
        if (to[i]) {
          a.b[batches] = of[i];
          a.c[batches++] = to[i];
        }
    }
    set_plan(a, p, batches, ws);
    TRY(dense_cc(type, a, p.tile, batches, s));
    TRY(join(a, 1, batches, s));
  }
  return hipSuccess;
}

int dense_linear_tile(const DenseLinear& c) { return linear_plan(c).tile; }
int dense_dx_tile(const DenseGrad& c) { return dx_plan(c).tile; }
int dense_dw_tile(const DenseGrad& c) { return dw_plan(c).tile; }
int dense_dh_tile(const DenseGrad& c) { return dh_plan(c).tile; }
int dense_dw_down_tile(const DenseGrad& c) { return dw_down_plan(c).tile; }
int dense_fp8_tile(const DenseFp8& c) { return fp8_plan(c).tile; }

size_t dense_fp8_workspace(const DenseFp8& c) { return fp8_plan(c).part_bytes; }

hipError_t launch_dense_fp8(const DenseFp8& c, hipStream_t s) {
  const Plan p = fp8_plan(c);
  const int mats = c.q_up ? 2 : 1;
  DenseArgs a = {};
  a.a[0] = c.q;
  a.a[1] = c.q_up;
  a.b[0] = c.xq;
  a.lda = a.ldb = (size_t)fp8_padded(c.n);
  a.M = c.rows;
  a.N = c.m;
  a.K = fp8_padded(c.n);
  a.segs = 1;
  a.c[0] = c.y;
  a.c_dtype = c.y_dtype;
  a.relu = c.relu;
  a.sa[0] = c.s;
  a.sa[1] = c.s_up;
  a.sb = c.xs;
  a.blocks = fp8_blocks(c.n);
  set_plan(a, p, mats, static_cast<char*>(c.ws));
  if (p.tile == kDenseFew) return dense_few(kTypeE4M3, mats, a, s);
  TRY(dense_fp8(a, mats, p.tile, s));
  return join(a, mats, 1, s);
}

}  // namespace si
