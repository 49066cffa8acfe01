// Argument checks and error reporting shared by the C ABI's source files.
#pragma once

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/sparseinfer.h"
#include "si_device.h"
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

// Margin of a predicting call: rows with N_neg < T - margin are surely kept.
int confident_margin(int d, int b, int T);

}  // namespace si
