// C ABI of the dense MLP's products and norms with their gradients, and of the
// products with FP8 weights: argument validation and launches.
#include <algorithm>

#include "api_common.h"
#include "dense.h"

namespace {

using namespace si;

constexpr int kMaxLen = 1 << 20;              // rows of W and their length
constexpr size_t kMaxLd = (size_t)1 << 21;    // strides, in elements
constexpr int kMaxNormLen = 16384;

Rows flat(const void* p, size_t bytes) { return Rows{p, 1, bytes, bytes}; }
Rows rows_of(const DenseMat& a, size_t rows, int n) {
  const size_t e = (size_t)dtype_bytes(a.dtype);
  return Rows{a.p, rows, a.ld * e, (size_t)n * e};
}

// The stride of a single row leads nowhere: it is taken as the row's length.
size_t stride(size_t ld, int rows, int n) { return rows > 1 ? ld : (size_t)n; }

si_status check_sizes(int m, int rows, int n) {
  if (si_status s = check_rows_n("m", m, n, kMaxLen)) return s;
  if (rows < 1 || rows > kMaxLen) return fail(SI_ERR_SHAPE, "rows=%d outside [1, %d]", rows, kMaxLen);
  // copies and element-wise kernels: 8 values a thread, 2^32 threads a launch
  const double most = 34359738368.0, longer = std::max(rows, n) + 8.0;
  if (m * longer >= most || std::min(rows, n) * longer >= most)
    return fail(SI_ERR_SHAPE, "m=%d rows=%d n=%d: more than one launch can hold", m, rows, n);
  return SI_OK;
}

si_status check_type(int dtype) {
  if (dtype != SI_F16 && dtype != SI_BF16) return fail(SI_ERR_ARG, "dtype=%d: fp16 or bf16 products", dtype);
  return SI_OK;
}

si_status check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (!need) return SI_OK;
  REQUIRE_PTR(workspace);
  REQUIRE_ALIGNED(workspace);
  if (bytes < need) return fail(SI_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", bytes, need);
  return SI_OK;
}

si_status fits(int tile, int m, int rows, int n) {
  if (tile < 0) return fail(SI_ERR_SHAPE, "m=%d rows=%d n=%d: more than one launch can hold", m, rows, n);
  return SI_OK;
}

DenseLinear linear_call(const void* x, int dtype, size_t ldx, int m, int n, const void* w, const void* w_up, int rows,
                        bool transposed) {
  DenseLinear c;
  const size_t ldw = (size_t)(transposed ? rows : n);
  c.x = DenseMat{x, dtype, stride(ldx, m, n)};
  c.w = DenseMat{w, dtype, ldw};
  c.w_up = DenseMat{w_up, dtype, ldw};
  c.type = dtype;
  c.transposed = transposed;
  c.m = m;
  c.rows = rows;
  c.n = n;
  return c;
}

si_status run_linear(DenseLinear c, size_t ldx, void* workspace, size_t workspace_bytes, void* stream) {
  if (si_status s = check_type(c.type)) return s;
  const int y_dtype = c.y_dtype;
  REQUIRE_DTYPE(y_dtype);
  if (si_status s = check_sizes(c.m, c.rows, c.n)) return s;
  if (si_status s = check_ld("ldx", ldx, c.n, c.m, kMaxLd)) return s;
  if (c.m == 0) return SI_OK;
  const void *x = c.x.p, *w = c.w.p, *w_up = c.w_up.p, *y = c.y, *g = c.g, *u = c.u;
  REQUIRE_PTR(x);
  REQUIRE_PTR(w);
  REQUIRE_PTR(y);
  REQUIRE_ELEMENT_ALIGNED(x, c.type);
  REQUIRE_ELEMENT_ALIGNED(w, c.type);
  REQUIRE_ELEMENT_ALIGNED(w_up, c.type);
  REQUIRE_ALIGNED(y);
  REQUIRE_ALIGNED(g);
  REQUIRE_ALIGNED(u);
  if ((g == nullptr) != (u == nullptr)) return fail(SI_ERR_NULL, "g and u must both be given or both be NULL");
  if (g && !w_up) return fail(SI_ERR_ARG, "g and u are those of a gated product");
  if (si_status s = fits(dense_linear_tile(c), c.m, c.rows, c.n)) return s;
  const size_t size = (size_t)c.m * c.rows, wb = (size_t)c.rows * c.n * 2;
  const Rows out[3] = {flat(y, size * dtype_bytes(c.y_dtype)), flat(g, size * 4), flat(u, size * 4)};
  const Rows in[3] = {rows_of(c.x, c.m, c.n), flat(w, wb), flat(w_up, wb)};
  for (int i = 0; i < 3; ++i) {
    for (const Rows& r : in)
      if (overlap(out[i], r)) return fail(SI_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return fail(SI_ERR_ARG, "two outputs overlap");
  }
  if (si_status s = check_workspace(workspace, workspace_bytes, dense_linear_workspace(c))) return s;
  c.ws = workspace;
  return hip_status(launch_dense_linear(c, (hipStream_t)stream), "dense product launch");
}

DenseGrad grad_call(const void* dy, int dy_dtype, size_t lddy, const void* x, int dtype, size_t ldx, int m, int n,
                    const void* w, const void* w_up, int rows, bool transposed) {
  DenseGrad c;
  const size_t ldw = (size_t)(transposed ? rows : n);
  c.dy = DenseMat{dy, dy_dtype, stride(lddy, m, rows)};
  c.x = DenseMat{x, dtype, stride(ldx, m, n)};
  c.w = DenseMat{w, dtype, ldw};
  c.w_up = DenseMat{w_up, dtype, ldw};
  c.type = dtype;
  c.transposed = transposed;
  c.m = m;
  c.rows = rows;
  c.n = n;
  return c;
}

si_status run_grad(DenseGrad c, size_t lddy, size_t ldx, bool gated, void* workspace, size_t workspace_bytes,
                   void* stream) {
  if (si_status s = check_type(c.type)) return s;
  const int dy_dtype = c.dy.dtype, g_dtype = c.gate.dtype;
  REQUIRE_DTYPE(dy_dtype);
  REQUIRE_DTYPE(g_dtype);
  if (si_status s = check_sizes(c.m, c.rows, c.n)) return s;
  const int dy_n = c.down.p ? c.n : c.rows;
  if (si_status s = check_ld("lddy", lddy, dy_n, c.m, kMaxLd)) return s;
  if (si_status s = check_ld("ldx", ldx, c.n, c.m, kMaxLd)) return s;
  const void *dy = c.dy.p, *x = c.x.p, *w = c.w.p, *w_up = c.w_up.p, *w_down = c.down.p, *g = c.gate.p, *u = c.up.p,
             *h = c.h.p, *dx = c.dx, *dw = c.dw, *dw_up = c.dw_up, *dw_down = c.dw_down;
  // (without tokens dx is empty and may have no address)
  if (c.m > 0 && !dx && !dw && !dw_up && !dw_down) return fail(SI_ERR_NULL, "none of the gradients is asked for");
  if (dw_up && !w_up) return fail(SI_ERR_ARG, "dw_up without w_up");
  if (u && !w_up) return fail(SI_ERR_ARG, "u without w_up");
  const bool through = dx || dw || dw_up;
  if (c.m > 0) {
    REQUIRE_PTR(dy);
    if (gated && through) REQUIRE_PTR(g);
    if (w_up && through) REQUIRE_PTR(u);
    if (dw || dw_up) REQUIRE_PTR(x);
    if (dw_down) REQUIRE_PTR(h);
  }
  if (dx || c.m > 0) REQUIRE_PTR(w);
  REQUIRE_ELEMENT_ALIGNED(dy, dy_dtype);
  REQUIRE_ELEMENT_ALIGNED(x, c.type);
  REQUIRE_ELEMENT_ALIGNED(w, c.type);
  REQUIRE_ELEMENT_ALIGNED(w_up, c.type);
  REQUIRE_ELEMENT_ALIGNED(w_down, c.type);
  REQUIRE_ALIGNED(g);
  REQUIRE_ALIGNED(u);
  REQUIRE_ALIGNED(h);
  REQUIRE_ALIGNED(dx);
  REQUIRE_ALIGNED(dw);
  REQUIRE_ALIGNED(dw_up);
  REQUIRE_ALIGNED(dw_down);
  if (w_down && through && c.m > 0)
    if (si_status s = fits(dense_dh_tile(c), c.m, c.rows, c.n)) return s;
  if (dx && c.m > 0)
    if (si_status s = fits(dense_dx_tile(c), c.m, c.rows, c.n)) return s;
  if (dw || dw_up)
    if (si_status s = fits(dense_dw_tile(c), c.m, c.rows, c.n)) return s;
  if (dw_down)
    if (si_status s = fits(dense_dw_down_tile(c), c.m, c.rows, c.n)) return s;
  const size_t wb = (size_t)c.rows * c.n * 2;
  const Rows out[4] = {flat(dx, (size_t)c.m * c.n * 2), flat(dw, wb), flat(dw_up, wb), flat(dw_down, wb)};
  const Rows in[8] = {rows_of(c.dy, c.m, dy_n),     rows_of(c.x, c.m, c.n),     flat(w, wb),     flat(w_up, wb),
                      rows_of(c.gate, c.m, c.rows), rows_of(c.up, c.m, c.rows), flat(w_down, wb), rows_of(c.h, c.m, c.rows)};
  for (int i = 0; i < 4; ++i) {
    for (const Rows& r : in)
      if (overlap(out[i], r)) return fail(SI_ERR_ARG, "a gradient overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return fail(SI_ERR_ARG, "two gradients overlap");
  }
  if (c.m == 0) c.dx = nullptr;
  if (!c.dx && !c.dw && !c.dw_up && !c.dw_down) return SI_OK;
  if (si_status s = check_workspace(workspace, workspace_bytes, dense_grad_workspace(c))) return s;
  c.ws = workspace;
  return hip_status(launch_dense_grad(c, (hipStream_t)stream), "dense gradient launch");
}

// The gate's values of a gated product are its sums, float32; else its output.
void set_gate(DenseGrad& c, const void* g, int g_dtype, const float* u) {
  c.gate = DenseMat{g, c.w_up.p ? SI_F32 : g_dtype, (size_t)c.rows};
  c.up = DenseMat{u, SI_F32, (size_t)c.rows};
}

DenseGrad mlp_call(const void* dy, int dy_dtype, size_t lddy, const void* x, int dtype, size_t ldx, int m, int d,
                   const void* w_gate, const void* w_up, const void* w_down, int k, const void* h, const float* g,
                   const float* u) {
  DenseGrad c = grad_call(dy, dy_dtype, lddy, x, dtype, ldx, m, d, w_gate, w_up, k, false);
  c.dy.ld = stride(lddy, m, d);
  c.down = DenseMat{w_down, dtype, (size_t)k};
  c.h = DenseMat{h, dtype, (size_t)k};
  if (w_up)
    set_gate(c, g, SI_F32, u);
  else
    set_gate(c, h, dtype, u);
  return c;
}

alignas(16) const uint8_t kSome[16] = {};  // stands for operands of which only the presence counts

si_status run_fp8(DenseFp8 c, bool gated, void* workspace, size_t workspace_bytes, void* stream) {
  const int y_dtype = c.y_dtype;
  REQUIRE_DTYPE(y_dtype);
  if (si_status s = check_sizes(c.m, c.rows, c.n)) return s;
  if (c.m == 0) return SI_OK;
  const uint8_t *xq = c.xq, *q = c.q, *q_up = c.q_up;
  const float *x_scale = c.xs, *scale = c.s, *s_up = c.s_up;
  const void* y = c.y;
  if ((q_up == nullptr) != (s_up == nullptr)) return fail(SI_ERR_NULL, "q_up and s_up must both be given or both be NULL");
  REQUIRE_PTR(xq);
  REQUIRE_PTR(x_scale);
  REQUIRE_PTR(q);
  REQUIRE_PTR(scale);
  REQUIRE_PTR(y);
  REQUIRE_ALIGNED(xq);
  REQUIRE_ALIGNED(q);
  REQUIRE_ALIGNED(q_up);
  REQUIRE_ALIGNED(y);
  REQUIRE_ELEMENT_ALIGNED(x_scale, SI_F32);
  REQUIRE_ELEMENT_ALIGNED(scale, SI_F32);
  REQUIRE_ELEMENT_ALIGNED(s_up, SI_F32);
  c.relu = gated && !q_up;
  if (si_status s = fits(dense_fp8_tile(c), c.m, c.rows, c.n)) return s;
  const size_t np = fp8_padded(c.n), nb = fp8_blocks(c.n), rb = (size_t)(c.rows + 127) / 128;
  const Rows out = flat(y, (size_t)c.m * c.rows * dtype_bytes(c.y_dtype));
  const Rows in[6] = {flat(xq, c.m * np),   flat(x_scale, c.m * nb * 4), flat(q, c.rows * np), flat(scale, rb * nb * 4),
                      flat(q_up, c.rows * np), flat(s_up, rb * nb * 4)};
  for (const Rows& r : in)
    if (overlap(out, r)) return fail(SI_ERR_ARG, "y overlaps an input");
  if (si_status s = check_workspace(workspace, workspace_bytes, dense_fp8_workspace(c))) return s;
  c.ws = workspace;
  return hip_status(launch_dense_fp8(c, (hipStream_t)stream), "FP8 product launch");
}

DenseFp8 fp8_call(const uint8_t* xq, const float* xs, int m, int n, const uint8_t* q, const float* s, const uint8_t* q_up,
                  const float* s_up, int rows, void* y, int y_dtype) {
  DenseFp8 c;
  c.xq = xq;
  c.xs = xs;
  c.q = q;
  c.s = s;
  c.q_up = q_up;
  c.s_up = s_up;
  c.m = m;
  c.rows = rows;
  c.n = n;
  c.y = y;
  c.y_dtype = y_dtype;
  return c;
}

si_status quantize(bool blocks, const void* w, int w_dtype, size_t ldw, int rows, int n, uint8_t* q, float* scale,
                   void* stream) {
  REQUIRE_DTYPE(w_dtype);
  if (si_status s = check_rows_n("rows", rows, n, 1 << 24)) return s;
  if (si_status s = check_ld("ldw", ldw, n, rows, (size_t)1 << 32)) return s;
  if (rows == 0) return SI_OK;
  REQUIRE_PTR(w);
  REQUIRE_PTR(q);
  REQUIRE_PTR(scale);
  REQUIRE_ELEMENT_ALIGNED(w, w_dtype);
  REQUIRE_ALIGNED(q);
  REQUIRE_ALIGNED(scale);
  if ((double)rows * (n + 127) >= 34359738368.0)  // 8 values a thread, 2^32 threads a launch
    return fail(SI_ERR_SHAPE, "rows=%d n=%d: more than one launch can hold", rows, n);
  const size_t e = (size_t)dtype_bytes(w_dtype), ld = stride(ldw, rows, n);
  const size_t qb = si_fp8_codes_bytes(rows, n), sb = blocks ? si_fp8_block_scales_bytes(rows, n) : si_fp8_scales_bytes(rows, n);
  const Rows in = {w, (size_t)rows, ld * e, (size_t)n * e}, qr = flat(q, qb), sr = flat(scale, sb);
  if (overlap(in, qr) || overlap(in, sr) || overlap(qr, sr)) return fail(SI_ERR_ARG, "w, q and scale overlap");
  return hip_status(blocks ? launch_quantize_blocks_fp8(w, w_dtype, ld, rows, n, q, scale, (hipStream_t)stream)
                           : launch_quantize_rows_fp8(w, w_dtype, ld, (size_t)rows, n, q, scale, (hipStream_t)stream),
                    "FP8 quantize launch");
}

}  // namespace

extern "C" {

// ---- products and their gradients -------------------------------------------------

size_t si_linear_workspace_bytes(const void* x, size_t ldx, int m, int n, const void* w, int rows, int w_transposed) {
  if (check_sizes(m, rows, n) != SI_OK || m == 0) return 0;
  return dense_linear_workspace(linear_call(x, SI_F16, ldx, m, n, w, nullptr, rows, w_transposed != 0));
}

si_status si_linear(const void* x, int dtype, size_t ldx, int m, int n, const void* w, int rows, int w_transposed, void* y,
                    int y_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  DenseLinear c = linear_call(x, dtype, ldx, m, n, w, nullptr, rows, w_transposed != 0);
  c.y = y;
  c.y_dtype = y_dtype;
  return run_linear(c, ldx, workspace, workspace_bytes, stream);
}

size_t si_gated_linear_workspace_bytes(const void* x, size_t ldx, int m, int n, const void* w_gate, const void* w_up,
                                       int rows) {
  if (check_sizes(m, rows, n) != SI_OK || m == 0) return 0;
  return dense_linear_workspace(linear_call(x, SI_F16, ldx, m, n, w_gate, w_up, rows, false));
}

si_status si_gated_linear(const void* x, int dtype, size_t ldx, int m, int n, const void* w_gate, const void* w_up,
                          int rows, void* h, int h_dtype, float* g, float* u, void* workspace, size_t workspace_bytes,
                          void* stream) {
  DenseLinear c = linear_call(x, dtype, ldx, m, n, w_gate, w_up, rows, false);
  c.relu = !w_up;
  c.y = h;
  c.y_dtype = h_dtype;
  c.g = g;
  c.u = u;
  return run_linear(c, ldx, workspace, workspace_bytes, stream);
}

size_t si_linear_backward_workspace_bytes(const void* dy, int dy_dtype, size_t lddy, const void* x, size_t ldx, int m, int n,
                                          const void* w, int rows, int w_transposed, int want_dx, int want_dw) {
  if (check_sizes(m, rows, n) != SI_OK || m == 0) return 0;
  // a dy of 2 bytes has the product's own type
  DenseGrad c = grad_call(dy, dy_dtype == SI_F32 ? SI_F32 : SI_F16, lddy, x, SI_F16, ldx, m, n, w, nullptr, rows,
                          w_transposed != 0);
  c.dx = want_dx ? const_cast<uint8_t*>(kSome) : nullptr;
  c.dw = want_dw ? const_cast<uint8_t*>(kSome) : nullptr;
  return dense_grad_workspace(c);
}

si_status si_linear_backward(const void* dy, int dy_dtype, size_t lddy, const void* x, int dtype, size_t ldx, int m, int n,
                             const void* w, int rows, int w_transposed, void* dx, void* dw, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (dy_dtype != dtype && dy_dtype != SI_F32) return fail(SI_ERR_ARG, "dy_dtype=%d: the products' type or float32", dy_dtype);
  DenseGrad c = grad_call(dy, dy_dtype, lddy, x, dtype, ldx, m, n, w, nullptr, rows, w_transposed != 0);
  c.dx = dx;
  c.dw = dw;
  return run_grad(c, lddy, ldx, false, workspace, workspace_bytes, stream);
}

size_t si_gated_linear_backward_workspace_bytes(const void* x, size_t ldx, int m, int n, const void* w_gate,
                                                const void* w_up, int rows, int want_dx, int want_dw) {
  if (check_sizes(m, rows, n) != SI_OK || m == 0) return 0;
  DenseGrad c = grad_call(kSome, SI_F16, (size_t)rows, x, SI_F16, ldx, m, n, w_gate, w_up, rows, false);
  set_gate(c, kSome, SI_F16, w_up ? reinterpret_cast<const float*>(kSome) : nullptr);
  c.dx = want_dx ? const_cast<uint8_t*>(kSome) : nullptr;
  c.dw = want_dw ? const_cast<uint8_t*>(kSome) : nullptr;
  return dense_grad_workspace(c);
}

si_status si_gated_linear_backward(const void* dh, int dh_dtype, size_t lddh, const void* g, int g_dtype, const float* u,
                                   const void* x, int dtype, size_t ldx, int m, int n, const void* w_gate,
                                   const void* w_up, int rows, void* dx, void* dw_gate, void* dw_up, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  DenseGrad c = grad_call(dh, dh_dtype, lddh, x, dtype, ldx, m, n, w_gate, w_up, rows, false);
  if (w_up && g_dtype != SI_F32) return fail(SI_ERR_ARG, "g_dtype=%d: the sums of a gated product are float32", g_dtype);
  set_gate(c, g, g_dtype, u);
  c.dx = dx;
  c.dw = dw_gate;
  c.dw_up = dw_up;
  return run_grad(c, lddh, ldx, true, workspace, workspace_bytes, stream);
}

size_t si_mlp_backward_workspace_bytes(const void* dy, int dy_dtype, size_t lddy, const void* x, size_t ldx, int m, int d,
                                       const void* w_gate, const void* w_up, const void* w_down, int k, int want_dx,
                                       int want_dw, int want_dw_down) {
  if (check_sizes(m, k, d) != SI_OK || m == 0) return 0;
  const float* sums = reinterpret_cast<const float*>(kSome);
  DenseGrad c = mlp_call(dy, dy_dtype == SI_F32 ? SI_F32 : SI_F16, lddy, x, SI_F16, ldx, m, d, w_gate, w_up, w_down, k, kSome,
                         sums, w_up ? sums : nullptr);
  c.dx = want_dx ? const_cast<uint8_t*>(kSome) : nullptr;
  c.dw = want_dw ? const_cast<uint8_t*>(kSome) : nullptr;
  c.dw_down = want_dw_down ? const_cast<uint8_t*>(kSome) : nullptr;
  return dense_grad_workspace(c);
}

si_status si_mlp_backward(const void* dy, int dy_dtype, size_t lddy, const void* x, int dtype, size_t ldx, int m, int d,
                          const void* w_gate, const void* w_up, const void* w_down, int k, const void* h, const float* g,
                          const float* u, void* dx, void* dw_gate, void* dw_up, void* dw_down, void* workspace,
                          size_t workspace_bytes, void* stream) {
  if (dy_dtype != dtype && dy_dtype != SI_F32) return fail(SI_ERR_ARG, "dy_dtype=%d: the products' type or float32", dy_dtype);
  if (g && !w_up) return fail(SI_ERR_ARG, "g without w_up");
  REQUIRE_PTR(w_down);
  if (m > 0 && !w_up) REQUIRE_PTR(h);
  DenseGrad c = mlp_call(dy, dy_dtype, lddy, x, dtype, ldx, m, d, w_gate, w_up, w_down, k, h, g, u);
  c.dx = dx;
  c.dw = dw_gate;
  c.dw_up = dw_up;
  c.dw_down = dw_down;
  return run_grad(c, lddy, ldx, true, workspace, workspace_bytes, stream);
}

int si_dense_tile(int kind, int m, int rows, int n, int gated) {
  if (kind < 0 || kind > 6 || check_sizes(m, rows, n) != SI_OK || m == 0) return -2;
  const bool transposed = kind < 6 && (kind & 1);
  const void* up = gated && !transposed ? kSome : nullptr;
  int tile;
  if (kind == 6) {
    DenseFp8 c;
    c.m = m;
    c.rows = rows;
    c.n = n;
    c.q_up = gated ? kSome : nullptr;
    tile = dense_fp8_tile(c);
  } else if (kind < 2) {
    tile = dense_linear_tile(linear_call(kSome, SI_F16, (size_t)n, m, n, kSome, up, rows, transposed));
  } else {
    const DenseGrad c = grad_call(kSome, SI_F16, (size_t)rows, kSome, SI_F16, (size_t)n, m, n, kSome, up, rows, transposed);
    tile = kind < 4 ? dense_dx_tile(c) : dense_dw_tile(c);
  }
  return tile < 0 ? -2 : tile;
}

// ---- FP8 ---------------------------------------------------------------------------

size_t si_fp8_codes_bytes(int rows, int n) {
  return check_rows_n("rows", rows, n, 1 << 24) == SI_OK ? (size_t)rows * fp8_padded(n) : 0;
}

size_t si_fp8_scales_bytes(int rows, int n) {
  return check_rows_n("rows", rows, n, 1 << 24) == SI_OK ? (size_t)rows * fp8_blocks(n) * 4 : 0;
}

size_t si_fp8_block_scales_bytes(int rows, int n) {
  return check_rows_n("rows", rows, n, 1 << 24) == SI_OK ? (size_t)((rows + 127) / 128) * fp8_blocks(n) * 4 : 0;
}

si_status si_quantize_rows_fp8(const void* x, int x_dtype, size_t ldx, int rows, int n, uint8_t* q, float* scale,
                               void* stream) {
  return quantize(false, x, x_dtype, ldx, rows, n, q, scale, stream);
}

si_status si_quantize_blocks_fp8(const void* w, int w_dtype, size_t ldw, int rows, int n, uint8_t* q, float* scale,
                                 void* stream) {
  return quantize(true, w, w_dtype, ldw, rows, n, q, scale, stream);
}

si_status si_dequantize_fp8(const uint8_t* q, const float* scale, int rows_per_scale, int rows, int n, void* w, int w_dtype,
                            void* stream) {
  REQUIRE_DTYPE(w_dtype);
  if (rows_per_scale != 1 && rows_per_scale != 128)
    return fail(SI_ERR_ARG, "rows_per_scale=%d is neither 1 nor 128", rows_per_scale);
  if (si_status s = check_rows_n("rows", rows, n, 1 << 24)) return s;
  if (rows == 0) return SI_OK;
  REQUIRE_PTR(q);
  REQUIRE_PTR(scale);
  REQUIRE_PTR(w);
  REQUIRE_ALIGNED(q);
  REQUIRE_ELEMENT_ALIGNED(scale, SI_F32);
  REQUIRE_ELEMENT_ALIGNED(w, w_dtype);
  if ((double)rows * (n + 127) >= 34359738368.0)
    return fail(SI_ERR_SHAPE, "rows=%d n=%d: more than one launch can hold", rows, n);
  const Rows o = flat(w, (size_t)rows * n * dtype_bytes(w_dtype));
  const size_t sb = rows_per_scale == 1 ? si_fp8_scales_bytes(rows, n) : si_fp8_block_scales_bytes(rows, n);
  if (overlap(o, flat(q, si_fp8_codes_bytes(rows, n))) || overlap(o, flat(scale, sb)))
    return fail(SI_ERR_ARG, "w overlaps q or scale");
  return hip_status(launch_dequantize_fp8(q, scale, rows_per_scale, (size_t)rows, n, w, w_dtype, (hipStream_t)stream),
                    "FP8 dequantize launch");
}

size_t si_linear_fp8_workspace_bytes(int m, int rows, int n, int gated) {
  if (check_sizes(m, rows, n) != SI_OK || m == 0) return 0;
  DenseFp8 c;
  c.m = m;
  c.rows = rows;
  c.n = n;
  c.q_up = gated ? kSome : nullptr;
  return dense_fp8_workspace(c);
}

si_status si_linear_fp8(const uint8_t* xq, const float* x_scale, int m, int n, const uint8_t* q, const float* scale,
                        int rows, void* y, int y_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  return run_fp8(fp8_call(xq, x_scale, m, n, q, scale, nullptr, nullptr, rows, y, y_dtype), false, workspace,
                 workspace_bytes, stream);
}

si_status si_gated_linear_fp8(const uint8_t* xq, const float* x_scale, int m, int n, const uint8_t* q_gate,
                              const float* s_gate, const uint8_t* q_up, const float* s_up, int rows, void* h, int h_dtype,
                              void* workspace, size_t workspace_bytes, void* stream) {
  return run_fp8(fp8_call(xq, x_scale, m, n, q_gate, s_gate, q_up, s_up, rows, h, h_dtype), true, workspace,
                 workspace_bytes, stream);
}

// ---- LayerNorm and RMSNorm -----------------------------------------------------------

static si_status check_norm(int dtype, int w_dtype, int tokens, int d) {
  REQUIRE_DTYPE(dtype);
  REQUIRE_DTYPE(w_dtype);
  if (tokens < 0 || tokens >= (1 << 23)) return fail(SI_ERR_SHAPE, "tokens=%d outside [0, 2^23)", tokens);
  if (d < 1 || d > kMaxNormLen) return fail(SI_ERR_SHAPE, "d=%d outside [1, %d]", d, kMaxNormLen);
  return SI_OK;
}

si_status si_layer_norm(const void* x, int dtype, size_t ldx, const void* w, const void* b, int w_dtype, int center,
                        float eps, void* y, float* mean, float* rstd, int tokens, int d, void* stream) {
  if (si_status s = check_norm(dtype, w_dtype, tokens, d)) return s;
  if (si_status s = check_ld("ldx", ldx, d, tokens, (size_t)1 << 32)) return s;
  if (!(eps >= 0.f) || std::isinf(eps)) return fail(SI_ERR_ARG, "eps=%g must be finite and >= 0", (double)eps);
  if (tokens == 0) return SI_OK;
  REQUIRE_PTR(x);
  REQUIRE_PTR(w);
  REQUIRE_PTR(y);
  if (center && (mean == nullptr) != (rstd == nullptr))
    return fail(SI_ERR_NULL, "mean and rstd must both be given or both be NULL");
  REQUIRE_ELEMENT_ALIGNED(x, dtype);
  REQUIRE_ELEMENT_ALIGNED(w, w_dtype);
  REQUIRE_ELEMENT_ALIGNED(b, w_dtype);
  REQUIRE_ELEMENT_ALIGNED(y, dtype);
  REQUIRE_ELEMENT_ALIGNED(mean, SI_F32);
  REQUIRE_ELEMENT_ALIGNED(rstd, SI_F32);
  if (!center) mean = nullptr;
  const size_t e = (size_t)dtype_bytes(dtype), wb = (size_t)d * dtype_bytes(w_dtype), ld = stride(ldx, tokens, d);
  const Rows in[3] = {Rows{x, (size_t)tokens, ld * e, d * e}, flat(w, wb), flat(b, wb)};
  const Rows out[3] = {flat(y, tokens * (d * e)), flat(mean, (size_t)tokens * 4), flat(rstd, (size_t)tokens * 4)};
  for (int i = 0; i < 3; ++i) {
    for (const Rows& r : in)
      if (overlap(out[i], r)) return fail(SI_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return fail(SI_ERR_ARG, "two outputs overlap");
  }
  LayerNormArgs a = {};
  a.x = x;
  a.ldx = ld;
  a.dtype = dtype;
  a.w = w;
  a.b = b;
  a.w_dtype = w_dtype;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  a.tokens = (size_t)tokens;
  a.d = d;
  a.center = center != 0;
  a.eps = eps;
  return hip_status(launch_layer_norm(a, (hipStream_t)stream), "norm launch");
}

size_t si_layer_norm_backward_workspace_bytes(int tokens, int d) {
  return check_norm(SI_F32, SI_F32, tokens, d) == SI_OK ? layer_norm_grad_workspace((size_t)tokens, d) : 0;
}

si_status si_layer_norm_backward(const void* dy, size_t lddy, const void* x, int dtype, size_t ldx, const void* w,
                                 int w_dtype, int center, const float* mean, const float* rstd, void* dx, void* dw, void* db,
                                 int tokens, int d, void* workspace, size_t workspace_bytes, void* stream) {
  if (si_status s = check_norm(dtype, w_dtype, tokens, d)) return s;
  if (si_status s = check_ld("lddy", lddy, d, tokens, (size_t)1 << 32)) return s;
  if (si_status s = check_ld("ldx", ldx, d, tokens, (size_t)1 << 32)) return s;
  if (tokens > 0) {
    if (!dx && !dw && !db) return fail(SI_ERR_NULL, "none of the gradients is asked for");
    REQUIRE_PTR(dy);
    REQUIRE_PTR(x);
    REQUIRE_PTR(w);
    REQUIRE_PTR(rstd);
    if (center) REQUIRE_PTR(mean);
  } else if (!dw && !db) {
    return SI_OK;
  }
  REQUIRE_ELEMENT_ALIGNED(dy, dtype);
  REQUIRE_ELEMENT_ALIGNED(x, dtype);
  REQUIRE_ELEMENT_ALIGNED(w, w_dtype);
  REQUIRE_ELEMENT_ALIGNED(mean, SI_F32);
  REQUIRE_ELEMENT_ALIGNED(rstd, SI_F32);
  REQUIRE_ELEMENT_ALIGNED(dx, dtype);
  REQUIRE_ELEMENT_ALIGNED(dw, w_dtype);
  REQUIRE_ELEMENT_ALIGNED(db, w_dtype);
  if (!center) mean = nullptr;
  const size_t e = (size_t)dtype_bytes(dtype), wb = (size_t)d * dtype_bytes(w_dtype);
  const size_t ldd = stride(lddy, tokens, d), ld = stride(ldx, tokens, d);
  const Rows in[5] = {Rows{dy, (size_t)tokens, ldd * e, d * e}, Rows{x, (size_t)tokens, ld * e, d * e}, flat(w, wb),
                      flat(mean, (size_t)tokens * 4), flat(rstd, (size_t)tokens * 4)};
  const Rows out[3] = {flat(dx, tokens * (d * e)), flat(dw, wb), flat(db, wb)};
  for (int i = 0; i < 3; ++i) {
    for (const Rows& r : in)
      if (overlap(out[i], r)) return fail(SI_ERR_ARG, "a gradient overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return fail(SI_ERR_ARG, "two gradients overlap");
  }
  const bool columns = dw || db;
  if (columns)
    if (si_status s = check_workspace(workspace, workspace_bytes, layer_norm_grad_workspace((size_t)tokens, d))) return s;
  LayerNormGrad a = {};
  a.dy = dy;
  a.ldy = ldd;
  a.x = x;
  a.ldx = ld;
  a.dtype = dtype;
  a.w = w;
  a.w_dtype = w_dtype;
  a.mean = mean;
  a.rstd = rstd;
  a.dx = dx;
  a.dw = dw;
  a.db = db;
  a.tokens = (size_t)tokens;
  a.d = d;
  a.center = center != 0;
  a.part = columns ? static_cast<float*>(workspace) : nullptr;
  return hip_status(launch_layer_norm_grad(a, (hipStream_t)stream), "norm gradient launch");
}

}  // extern "C"
