// The library's backward calls for the host tests of the autograd nodes: nothing is
// computed, each call writes a line of its arguments.  Loaded before the nodes with its
// names visible to them, so that they call these in place of the library's.
#include <cstdio>

#include "sparseinfer.h"

namespace {
unsigned long long at(const void* p) { return (unsigned long long)reinterpret_cast<uintptr_t>(p); }
}  // namespace

extern "C" {

size_t si_linear_backward_workspace_bytes(const void*, int, size_t lddy, const void*, size_t ldx, int, int, const void*, int, int,
                                          int, int) {
  printf("workspace lddy=%zu ldx=%zu\n", lddy, ldx);
  return 0;
}
si_status si_linear_backward(const void* dy, int dy_dtype, size_t lddy, const void* x, int dtype, size_t ldx, int m, int n,
                             const void* w, int rows, int w_transposed, void* dx, void* dw, void*, size_t, void*) {
  printf("linear dy=%llu dy_dtype=%d lddy=%zu x=%llu dtype=%d ldx=%zu m=%d n=%d w=%llu rows=%d transposed=%d dx=%llu dw=%llu\n",
         at(dy), dy_dtype, lddy, at(x), dtype, ldx, m, n, at(w), rows, w_transposed, at(dx), at(dw));
  return SI_OK;
}

size_t si_gated_linear_backward_workspace_bytes(const void*, size_t ldx, int, int, const void*, const void*, int, int, int) {
  printf("workspace ldx=%zu\n", ldx);
  return 0;
}
si_status si_gated_linear_backward(const void* dh, int dh_dtype, size_t lddh, const void* g, int g_dtype, const float* u,
                                   const void* x, int dtype, size_t ldx, int m, int n, const void* w_gate, const void* w_up,
                                   int rows, void* dx, void* dw_gate, void* dw_up, void*, size_t, void*) {
  printf("gated dy=%llu dy_dtype=%d lddy=%zu g=%llu g_dtype=%d u=%llu x=%llu dtype=%d ldx=%zu m=%d n=%d w=%llu w_up=%llu "
         "rows=%d dx=%llu dw=%llu dw_up=%llu\n",
         at(dh), dh_dtype, lddh, at(g), g_dtype, at(u), at(x), dtype, ldx, m, n, at(w_gate), at(w_up), rows, at(dx),
         at(dw_gate), at(dw_up));
  return SI_OK;
}

size_t si_mlp_backward_workspace_bytes(const void*, int, size_t lddy, const void*, size_t ldx, int, int, const void*, const void*,
                                       const void*, int, int, int, int) {
  printf("workspace lddy=%zu ldx=%zu\n", lddy, ldx);
  return 0;
}
si_status si_mlp_backward(const void* dy, int dy_dtype, size_t lddy, const void* x, int dtype, size_t ldx, int m, int d,
                          const void* w_gate, const void* w_up, const void* w_down, int k, const void* h, const float* g,
                          const float* u, void* dx, void* dw_gate, void* dw_up, void* dw_down, void*, size_t, void*) {
  printf("mlp dy=%llu dy_dtype=%d lddy=%zu x=%llu dtype=%d ldx=%zu m=%d n=%d w=%llu w_up=%llu w_down=%llu rows=%d h=%llu "
         "g=%llu u=%llu dx=%llu dw=%llu dw_up=%llu dw_down=%llu\n",
         at(dy), dy_dtype, lddy, at(x), dtype, ldx, m, d, at(w_gate), at(w_up), at(w_down), k, at(h), at(g), at(u), at(dx),
         at(dw_gate), at(dw_up), at(dw_down));
  return SI_OK;
}

size_t si_layer_norm_backward_workspace_bytes(int, int) { return 0; }
si_status si_layer_norm_backward(const void* dy, size_t lddy, const void* x, int dtype, size_t ldx, const void* w, int w_dtype,
                                 int center, const float* mean, const float* rstd, void* dx, void* dw, void* db, int tokens,
                                 int d, void*, size_t, void*) {
  printf("norm dy=%llu lddy=%zu x=%llu dtype=%d ldx=%zu m=%d n=%d w=%llu w_dtype=%d center=%d mean=%llu r=%llu dx=%llu "
         "dw=%llu db=%llu\n",
         at(dy), lddy, at(x), dtype, ldx, tokens, d, at(w), w_dtype, center, at(mean), at(rstd), at(dx), at(dw), at(db));
  return SI_OK;
}

}  // extern "C"
