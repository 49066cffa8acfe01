// C ABI of the MXFP4 operators and of the norms around a block: argument
// validation and launches.
#include "api_common.h"
#include "mx.h"
#include "mx_launch.h"

namespace {

using namespace si;

constexpr int kMaxN = 1 << 20;       // length of a sum of the products
constexpr int kMaxNormD = 16384;

bool known_dtype(int t) { return t == SI_F16 || t == SI_BF16 || t == SI_F32; }
static_assert(SI_F16 == kF16 && SI_BF16 == kBF16 && SI_F32 == kF32, "si_dtype");

#define REQUIRE_DTYPE(t) \
  if (!known_dtype(t)) return fail(SI_ERR_ARG, "%s=%d is not an si_dtype", #t, t)
// elements of 2 or 4 bytes at an address of their own size
#define REQUIRE_ELEMENT_ALIGNED(p, t) \
  if ((p) && reinterpret_cast<uintptr_t>(p) % dtype_bytes(t) != 0) return fail(SI_ERR_ALIGN, "%s is not aligned to its elements", #p)

// Rows of `w` bytes, `ld` bytes apart.
struct Rows {
  const void* p;
  size_t rows, ld, w;
};
// Whether two sets of rows share a byte; column ranges of one matrix do not.
bool overlap(const Rows& a, const Rows& b) {
  if (!a.p || !b.p || !a.rows || !b.rows || !a.w || !b.w) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  const uintptr_t ea = pa + (a.rows - 1) * a.ld + a.w, eb = pb + (b.rows - 1) * b.ld + b.w;
  if (pa >= eb || pb >= ea) return false;
  if (a.ld == b.ld && a.rows > 1 && b.rows > 1) {
    const uintptr_t off = (pb >= pa ? pb - pa : a.ld - 1 - (pa - pb - 1) % a.ld) % a.ld;  // b's first byte in a's row
    return off < a.w || off + b.w > a.ld;
  }
  return true;
}
size_t mx_codes(size_t rows, int n) { return rows * (size_t)(mx_padded(n) / 2); }
size_t mx_scales(size_t rows, int n) { return rows * (size_t)(mx_padded(n) / kMxBlock); }

si_status check_rows_n(const char* what, int rows, int n, int max_n) {
  if (rows < 0 || rows > (1 << 24)) return fail(SI_ERR_SHAPE, "%s=%d outside [0, 2^24]", what, rows);
  if (n < 1 || n > max_n) return fail(SI_ERR_SHAPE, "n=%d outside [1, %d]", n, max_n);
  return SI_OK;
}

si_status check_ld(const char* what, size_t ld, int n, int rows, size_t max_ld) {
  if (rows > 1 && (ld > max_ld || ld < (size_t)n))  // a single row's stride leads nowhere
    return fail(SI_ERR_SHAPE, "%s=%zu outside [n=%d, %zu]", what, ld, n, max_ld);
  return SI_OK;
}

// The sizes of a product, for the call and for the size of its workspace.
si_status check_product(const MxLinear& c) {
  if (si_status s = check_rows_n("m", c.m, c.n, kMaxN)) return s;
  if (c.rows < 1 || c.rows > (1 << 24)) return fail(SI_ERR_SHAPE, "rows=%d outside [1, 2^24]", c.rows);
  if (c.m > 0 && !mx_linear_fits(c))
    return fail(SI_ERR_SHAPE, "m=%d rows=%d n=%d: more than one launch can hold", c.m, c.rows, c.n);
  return SI_OK;
}

si_status run_linear(MxLinear& c, bool gated, void* workspace, size_t workspace_bytes, void* stream) {
  if (si_status s = check_product(c)) return s;
  REQUIRE_DTYPE(c.y_dtype);
  if (c.m == 0) return SI_OK;
  const uint8_t *q_up = c.q_up, *s_up = c.s_up;
  if ((q_up == nullptr) != (s_up == nullptr)) return fail(SI_ERR_NULL, "q_up and s_up must both be given or both be NULL");
  const void* y = c.y;
  const uint8_t *q = c.q, *scale = c.s;
  REQUIRE_PTR(q);
  REQUIRE_PTR(scale);
  REQUIRE_PTR(y);
  REQUIRE_ALIGNED(q);
  REQUIRE_ALIGNED(scale);
  REQUIRE_ALIGNED(q_up);
  REQUIRE_ALIGNED(s_up);
  REQUIRE_ALIGNED(y);
  c.relu = gated && !q_up;
  const size_t ey = (size_t)dtype_bytes(c.y_dtype), row = (size_t)c.rows * ey, np = mx_padded(c.n);
  const Rows out = {y, (size_t)c.m, row, row};
  auto flat = [](const void* p, size_t bytes) { return Rows{p, 1, bytes, bytes}; };
  if (overlap(out, Rows{c.x, (size_t)c.m, c.ldx * 2, (size_t)c.n * 2}) || overlap(out, flat(c.xq, c.m * np / 2)) ||
      overlap(out, flat(c.xs, c.m * np / 32)) || overlap(out, flat(q, c.rows * np / 2)) ||
      overlap(out, flat(scale, c.rows * np / 32)) || overlap(out, flat(q_up, c.rows * np / 2)) ||
      overlap(out, flat(s_up, c.rows * np / 32)))
    return fail(SI_ERR_ARG, "y overlaps an input");
  const size_t need = mx_linear_workspace(c);
  if (need) {
    REQUIRE_PTR(workspace);
    REQUIRE_ALIGNED(workspace);
    if (workspace_bytes < need)
      return fail(SI_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  }
  c.ws = workspace;
  return hip_status(launch_mx_linear(c, (hipStream_t)stream), "MXFP4 product launch");
}

alignas(16) const uint8_t kSome[16] = {};  // stands for operands of which only the presence counts

// A call of which only the sizes are known (x NULL: MXFP4 activations).
MxLinear sizes_of(const void* x, size_t ldx, int m, int rows, int n, int gated) {
  MxLinear c;
  c.x = x;
  c.ldx = ldx;
  c.xq = x ? nullptr : kSome;
  c.q_up = gated ? kSome : nullptr;
  c.m = m;
  c.rows = rows;
  c.n = n;
  return c;
}

si_status linear_f(bool gated, const void* x, int x_dtype, size_t ldx, int m, int n, const uint8_t* q,
                   const uint8_t* scale, const uint8_t* q_up, const uint8_t* s_up, int rows, void* y, int y_dtype,
                   void* workspace, size_t workspace_bytes, void* stream) {
  if (x_dtype != SI_F16 && x_dtype != SI_BF16) return fail(SI_ERR_ARG, "x_dtype=%d: fp16 or bf16 activations", x_dtype);
  if (si_status s = check_rows_n("m", m, n, kMaxN)) return s;
  if (si_status s = check_ld("ldx", ldx, n, m, (size_t)2 * kMaxN)) return s;
  if (m > 0) REQUIRE_PTR(x);
  REQUIRE_ELEMENT_ALIGNED(x, x_dtype);
  MxLinear c;
  c.x = x;
  c.x_dtype = x_dtype;
  c.ldx = ldx;
  c.q = q;
  c.s = scale;
  c.q_up = q_up;
  c.s_up = s_up;
  c.m = m;
  c.rows = rows;
  c.n = n;
  c.y = y;
  c.y_dtype = y_dtype;
  return run_linear(c, gated, workspace, workspace_bytes, stream);
}

si_status linear_q(bool gated, const uint8_t* xq, const uint8_t* x_scale, int m, int n, const uint8_t* q,
                   const uint8_t* scale, const uint8_t* q_up, const uint8_t* s_up, int rows, void* y, int y_dtype,
                   void* workspace, size_t workspace_bytes, void* stream) {
  if (m > 0) {
    REQUIRE_PTR(xq);
    REQUIRE_PTR(x_scale);
  }
  REQUIRE_ALIGNED(xq);
  REQUIRE_ALIGNED(x_scale);
  MxLinear c;
  c.xq = xq;
  c.xs = x_scale;
  c.q = q;
  c.s = scale;
  c.q_up = q_up;
  c.s_up = s_up;
  c.m = m;
  c.rows = rows;
  c.n = n;
  c.y = y;
  c.y_dtype = y_dtype;
  return run_linear(c, gated, workspace, workspace_bytes, stream);
}

}  // namespace

extern "C" {

size_t si_mxfp4_codes_bytes(int rows, int n) {
  return check_rows_n("rows", rows, n, 1 << 24) == SI_OK ? mx_codes(rows, n) : 0;
}

size_t si_mxfp4_scales_bytes(int rows, int n) {
  return check_rows_n("rows", rows, n, 1 << 24) == SI_OK ? mx_scales(rows, n) : 0;
}

si_status si_quantize_rows_mxfp4(const void* w, int w_dtype, size_t ldw, int rows, int n, uint8_t* q, uint8_t* scale,
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
  if ((double)rows * mx_padded(n) >= 137438953472.0)  // 32 values a thread, 2^32 threads a launch
    return fail(SI_ERR_SHAPE, "rows=%d n=%d: more than one launch can hold", rows, n);
  const size_t e = (size_t)dtype_bytes(w_dtype);
  const Rows in = {w, (size_t)rows, ldw * e, (size_t)n * e};
  const Rows qr = {q, 1, mx_codes(rows, n), mx_codes(rows, n)}, sr = {scale, 1, mx_scales(rows, n), mx_scales(rows, n)};
  if (overlap(in, qr) || overlap(in, sr) || overlap(qr, sr)) return fail(SI_ERR_ARG, "w, q and scale overlap");
  return hip_status(launch_quantize_mx(w, w_dtype, (size_t)rows, n, ldw, q, scale, (hipStream_t)stream),
                    "MXFP4 quantize launch");
}

si_status si_dequantize_rows_mxfp4(const uint8_t* q, const uint8_t* scale, int rows, int n, void* w, int w_dtype,
                                   void* stream) {
  REQUIRE_DTYPE(w_dtype);
  if (si_status s = check_rows_n("rows", rows, n, 1 << 24)) return s;
  if (rows == 0) return SI_OK;
  REQUIRE_PTR(q);
  REQUIRE_PTR(scale);
  REQUIRE_PTR(w);
  REQUIRE_ALIGNED(q);
  REQUIRE_ALIGNED(scale);
  REQUIRE_ELEMENT_ALIGNED(w, w_dtype);
  if ((double)rows * mx_padded(n) >= 137438953472.0)
    return fail(SI_ERR_SHAPE, "rows=%d n=%d: more than one launch can hold", rows, n);
  const size_t out = (size_t)rows * n * dtype_bytes(w_dtype);
  const Rows o = {w, 1, out, out};
  if (overlap(o, Rows{q, 1, mx_codes(rows, n), mx_codes(rows, n)}) ||
      overlap(o, Rows{scale, 1, mx_scales(rows, n), mx_scales(rows, n)}))
    return fail(SI_ERR_ARG, "w overlaps q or scale");
  return hip_status(launch_dequantize_mx(q, scale, (size_t)rows, n, w, w_dtype, (hipStream_t)stream),
                    "MXFP4 dequantize launch");
}

si_status si_pack_signs_mxfp4(const uint8_t* q_gate, int k, int d, uint32_t* signs, void* stream) {
  REQUIRE_PTR(q_gate);
  REQUIRE_PTR(signs);
  REQUIRE_ALIGNED(q_gate);
  REQUIRE_ALIGNED(signs);
  if (si_status s = check_kd(k, d)) return s;
  return hip_status(launch_pack_signs_mx(q_gate, k, d, signs, (hipStream_t)stream), "pack_signs_mxfp4 launch");
}

size_t si_linear_mxfp4_workspace_bytes(const void* x, size_t ldx, int m, int rows, int n, int gated) {
  const MxLinear c = sizes_of(x, ldx, m, rows, n, gated);
  return check_product(c) != SI_OK || m == 0 ? 0 : mx_linear_workspace(c);
}

int si_linear_mxfp4_tile(int a4, int m, int rows, int n, int gated) {
  const MxLinear c = sizes_of(a4 ? nullptr : kSome, (size_t)(n > 0 ? n : 0), m, rows, n, gated);
  return check_product(c) != SI_OK || m == 0 ? -2 : mx_linear_tile(c);
}

si_status si_linear_mxfp4(const void* x, int x_dtype, size_t ldx, int m, int n, const uint8_t* q, const uint8_t* scale,
                          int rows, void* y, int y_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  return linear_f(false, x, x_dtype, ldx, m, n, q, scale, nullptr, nullptr, rows, y, y_dtype, workspace,
                  workspace_bytes, stream);
}

si_status si_gated_linear_mxfp4(const void* x, int x_dtype, size_t ldx, int m, int n, const uint8_t* q_gate,
                                const uint8_t* s_gate, const uint8_t* q_up, const uint8_t* s_up, int rows, void* h,
                                int h_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  return linear_f(true, x, x_dtype, ldx, m, n, q_gate, s_gate, q_up, s_up, rows, h, h_dtype, workspace,
                  workspace_bytes, stream);
}

si_status si_linear_mxfp4_a4(const uint8_t* xq, const uint8_t* x_scale, int m, int n, const uint8_t* q,
                             const uint8_t* scale, int rows, void* y, int y_dtype, void* workspace,
                             size_t workspace_bytes, void* stream) {
  return linear_q(false, xq, x_scale, m, n, q, scale, nullptr, nullptr, rows, y, y_dtype, workspace, workspace_bytes,
                  stream);
}

si_status si_gated_linear_mxfp4_a4(const uint8_t* xq, const uint8_t* x_scale, int m, int n, const uint8_t* q_gate,
                                   const uint8_t* s_gate, const uint8_t* q_up, const uint8_t* s_up, int rows, void* h,
                                   int h_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  return linear_q(true, xq, x_scale, m, n, q_gate, s_gate, q_up, s_up, rows, h, h_dtype, workspace, workspace_bytes,
                  stream);
}

}  // extern "C"

// ---- the sparse MLP -----------------------------------------------------------

namespace {

si_status mlp_impl(bool predict, const uint32_t* signs, const uint8_t* q_gate, const uint8_t* s_gate,
                   const uint8_t* q_up, const uint8_t* s_up, const uint8_t* q_down_t, const uint8_t* s_down_t, int k,
                   int d, const uint16_t* x, int b, float alpha, const uint8_t* mask_in, uint8_t* mask,
                   int32_t* active_idx, int32_t* n_active, float* y, void* workspace, size_t workspace_bytes,
                   uint32_t flags, int32_t* counters, void* stream) {
  if (predict) {
    REQUIRE_PTR(signs);
  } else {
    REQUIRE_PTR(mask_in);
  }
  REQUIRE_PTR(q_gate);
  REQUIRE_PTR(s_gate);
  REQUIRE_PTR(q_down_t);
  REQUIRE_PTR(s_down_t);
  REQUIRE_PTR(x);
  REQUIRE_PTR(y);
  if ((q_up == nullptr) != (s_up == nullptr)) return fail(SI_ERR_NULL, "q_up and s_up must both be given or both be NULL");
  REQUIRE_ALIGNED(signs);
  REQUIRE_ALIGNED(q_gate);
  REQUIRE_ALIGNED(s_gate);
  REQUIRE_ALIGNED(q_up);
  REQUIRE_ALIGNED(s_up);
  REQUIRE_ALIGNED(q_down_t);
  REQUIRE_ALIGNED(s_down_t);
  REQUIRE_ALIGNED(x);
  REQUIRE_ALIGNED(y);
  REQUIRE_ALIGNED(mask_in);
  REQUIRE_ALIGNED(mask);
  REQUIRE_ALIGNED(active_idx);
  REQUIRE_ALIGNED(n_active);
  REQUIRE_ALIGNED(counters);
  if (flags & ~(SI_NO_AS | SI_NO_SPECULATION)) return fail(SI_ERR_FLAGS, "unknown flags 0x%x", flags);
  if (si_status s = check_kd(k, d)) return s;
  if (si_status s = check_b(b)) return s;
  if (predict && (std::isnan(alpha) || alpha < 0.0f))
    return fail(SI_ERR_ALPHA, "alpha=%g must be >= 0 (or +inf)", (double)alpha);
  const uintptr_t xa = reinterpret_cast<uintptr_t>(x), ya = reinterpret_cast<uintptr_t>(y);
  const uintptr_t xn = (uintptr_t)b * d * 2, yn = (uintptr_t)b * d * 4;
  if (xa < ya + yn && ya < xa + xn) return fail(SI_ERR_ARG, "x and y overlap");
  REQUIRE_PTR(workspace);
  REQUIRE_ALIGNED(workspace);
  const size_t need = ws_layout(k, b).total;
  if (workspace_bytes < need)
    return fail(SI_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  MxMlpCall c;
  c.signs = predict ? signs : nullptr;
  c.mask_in = predict ? nullptr : mask_in;
  c.q_gate = q_gate;
  c.s_gate = s_gate;
  c.q_up = q_up;
  c.s_up = s_up;
  c.q_down_t = q_down_t;
  c.s_down_t = s_down_t;
  c.x = x;
  c.k = k;
  c.d = d;
  c.b = b;
  if (predict) {
    c.T = si_alpha_threshold(alpha, d);
    c.margin = confident_margin(d, b, c.T);
    c.mask = mask;
    c.idx = active_idx;
    c.n_out = n_active;
  }
  c.flags = flags;
  c.y = y;
  c.ws = workspace;
  c.counters = counters;
  return hip_status(launch_mx_mlp(c, (hipStream_t)stream), "MXFP4 layer launch");
}

}  // namespace

extern "C" {

size_t si_mxfp4_workspace_bytes(int k, int d, int b) {
  if (check_kd(k, d) != SI_OK || check_b(b) != SI_OK) return 0;
  return ws_layout(k, b).total;
}

si_status si_sparse_mlp_mxfp4(const uint8_t* q_gate, const uint8_t* s_gate, const uint8_t* q_up, const uint8_t* s_up,
                              const uint8_t* q_down_t, const uint8_t* s_down_t, int k, int d, const uint16_t* x, int b,
                              const uint8_t* mask, float* y, void* workspace, size_t workspace_bytes, uint32_t flags,
                              int32_t* counters, void* stream) {
  return mlp_impl(false, nullptr, q_gate, s_gate, q_up, s_up, q_down_t, s_down_t, k, d, x, b, 0.0f, mask, nullptr,
                  nullptr, nullptr, y, workspace, workspace_bytes, flags, counters, stream);
}

si_status si_predict_sparse_mlp_mxfp4(const uint32_t* signs, const uint8_t* q_gate, const uint8_t* s_gate,
                                      const uint8_t* q_up, const uint8_t* s_up, const uint8_t* q_down_t,
                                      const uint8_t* s_down_t, int k, int d, const uint16_t* x, int b, float alpha,
                                      uint8_t* mask, int32_t* active_idx, int32_t* n_active, float* y, void* workspace,
                                      size_t workspace_bytes, uint32_t flags, int32_t* counters, void* stream) {
  return mlp_impl(true, signs, q_gate, s_gate, q_up, s_up, q_down_t, s_down_t, k, d, x, b, alpha, nullptr, mask,
                  active_idx, n_active, y, workspace, workspace_bytes, flags, counters, stream);
}

si_status si_norm_residual(const void* h, int h_dtype, size_t ldh, const void* branch, int branch_dtype, size_t ldb,
                           const float* post_w, const float* gate, int rows_per_gate, float scale, void* h_out,
                           size_t ldo, const float* pre_w, void* x, int x_dtype, size_t ldx, int tokens, int d,
                           float eps, void* stream) {
  REQUIRE_DTYPE(h_dtype);
  REQUIRE_DTYPE(branch_dtype);
  REQUIRE_DTYPE(x_dtype);
  if (tokens < 0 || tokens >= (1 << 23)) return fail(SI_ERR_SHAPE, "tokens=%d outside [0, 2^23)", tokens);
  if (d < 1 || d > kMaxNormD) return fail(SI_ERR_SHAPE, "d=%d outside [1, %d]", d, kMaxNormD);
  constexpr size_t max_ld = (size_t)1 << 32;
  if (si_status s = check_ld("ldh", ldh, d, tokens, max_ld)) return s;
  if (branch)
    if (si_status s = check_ld("ldb", ldb, d, tokens, max_ld)) return s;
  if (h_out)
    if (si_status s = check_ld("ldo", ldo, d, tokens, max_ld)) return s;
  if (x)
    if (si_status s = check_ld("ldx", ldx, d, tokens, max_ld)) return s;
  if (gate && rows_per_gate < 1) return fail(SI_ERR_SHAPE, "rows_per_gate=%d must be at least 1", rows_per_gate);
  if (!std::isfinite(eps) || eps < 0.0f) return fail(SI_ERR_ARG, "eps=%g must be finite and >= 0", (double)eps);
  if (!std::isfinite(scale)) return fail(SI_ERR_ARG, "scale=%g must be finite", (double)scale);
  if (tokens == 0) return SI_OK;
  REQUIRE_PTR(h);
  if (!branch && (post_w || gate || h_out))
    return fail(SI_ERR_NULL, "branch is NULL but post_w, gate or h_out is given");
  if ((pre_w == nullptr) != (x == nullptr)) return fail(SI_ERR_NULL, "pre_w and x must both be given or both be NULL");
  if (!h_out && !x) return fail(SI_ERR_NULL, "neither h_out nor x is given");
  REQUIRE_ELEMENT_ALIGNED(h, h_dtype);
  REQUIRE_ELEMENT_ALIGNED(branch, branch_dtype);
  REQUIRE_ELEMENT_ALIGNED(h_out, h_dtype);
  REQUIRE_ELEMENT_ALIGNED(x, x_dtype);
  REQUIRE_ELEMENT_ALIGNED(post_w, SI_F32);
  REQUIRE_ELEMENT_ALIGNED(gate, SI_F32);
  REQUIRE_ELEMENT_ALIGNED(pre_w, SI_F32);
  const size_t t = (size_t)tokens, eh = dtype_bytes(h_dtype), eb = dtype_bytes(branch_dtype), ex = dtype_bytes(x_dtype);
  const size_t params = (size_t)d * 4, gates = gate ? (t + rows_per_gate - 1) / rows_per_gate * params : 0;
  const Rows rh = {h, t, ldh * eh, d * eh}, rb = {branch, t, ldb * eb, d * eb}, ro = {h_out, t, ldo * eh, d * eh},
             rx = {x, t, ldx * ex, d * ex}, rp = {post_w, 1, params, params}, rg = {gate, 1, gates, gates},
             rw = {pre_w, 1, params, params};
  const bool in_place = h_out == h && (ldo == ldh || tokens == 1);  // each value is read before it is written
  for (const Rows& in : {rb, rp, rg, rw})
    if (overlap(ro, in) || overlap(rx, in)) return fail(SI_ERR_ARG, "an output overlaps an input");
  if ((!in_place && overlap(ro, rh)) || overlap(rx, rh) || overlap(rx, ro))
    return fail(SI_ERR_ARG, "h, h_out and x overlap (h_out may be h itself)");
  NormArgs a;
  a.h = h;
  a.b = branch;
  a.h_out = h_out;
  a.x = x;
  a.post_w = post_w;
  a.gate = gate;
  a.pre_w = pre_w;
  a.tokens = t;
  a.rows_per_gate = gate ? (size_t)rows_per_gate : 1;
  a.ldh = ldh;
  a.ldb = ldb;
  a.ldo = ldo;
  a.ldx = ldx;
  a.d = d;
  a.h_dtype = h_dtype;
  a.b_dtype = branch_dtype;
  a.x_dtype = x_dtype;
  a.scale = scale;
  a.eps = eps;
  return hip_status(launch_norm_residual(a, (hipStream_t)stream), "norm_residual launch");
}

}  // extern "C"
