// Argument checks and error reporting shared by the C ABI's source files.
#pragma once

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/sparseinfer.h"
#include "mx.h"
#include "si_launch.h"

namespace si {

// The calling thread's last error message (si_last_error()).
inline thread_local char g_err[512] = "";

inline si_status fail(si_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return s;
}

inline si_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return SI_OK;
  return fail(SI_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

#define REQUIRE_PTR(p) \
  if (!(p)) return fail(SI_ERR_NULL, "%s is NULL", #p)
#define REQUIRE_ALIGNED(p) \
  if ((p) && !aligned16(p)) return fail(SI_ERR_ALIGN, "%s is not 16-byte aligned", #p)

inline si_status check_kd(int k, int d) {
  if (k < 1 || k > (1 << 24)) return fail(SI_ERR_SHAPE, "k=%d outside [1, 2^24]", k);
  if (d < 128 || d > kMaxD || d % 128 != 0)
    return fail(SI_ERR_SHAPE, "d=%d must be a multiple of 128 in [128, %d]", d, kMaxD);
  return SI_OK;
}

inline si_status check_b(int b) {
  if (b < 1 || b > kMaxB) return fail(SI_ERR_SHAPE, "b=%d outside [1, %d]", b, kMaxB);
  return SI_OK;
}

// ---- calls of several element types, with rows at a stride -----------------------

inline bool known_dtype(int t) { return t == SI_F16 || t == SI_BF16 || t == SI_F32; }
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
inline bool overlap(const Rows& a, const Rows& b) {
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
inline si_status check_rows_n(const char* what, int rows, int n, int max_n) {
  if (rows < 0 || rows > (1 << 24)) return fail(SI_ERR_SHAPE, "%s=%d outside [0, 2^24]", what, rows);
  if (n < 1 || n > max_n) return fail(SI_ERR_SHAPE, "n=%d outside [1, %d]", n, max_n);
  return SI_OK;
}

inline si_status check_ld(const char* what, size_t ld, int n, int rows, size_t max_ld) {
  if (rows > 1 && (ld > max_ld || ld < (size_t)n))  // a single row's stride leads nowhere
    return fail(SI_ERR_SHAPE, "%s=%zu outside [n=%d, %zu]", what, ld, n, max_ld);
  return SI_OK;
}

// Margin of a predicting call: rows with N_neg < T - margin are surely kept.
int confident_margin(int d, int b, int T);

}  // namespace si
