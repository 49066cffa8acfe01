// The gradients' place in PyTorch's graph of calls: nodes whose backward pass is one call
// of the library (include/sparseinfer.h), on the stream of the forward call.  Host code:
// a node written in Python took 40 us more of a training step's host time (LayerNorm of
// 16 tokens, forward and backward: 114 us), which is more than the kernels of a small one.
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <optional>

#include "../../include/sparseinfer.h"

namespace {

using at::Tensor;
using torch::autograd::Node;
using torch::autograd::SavedVariable;
using torch::autograd::variable_list;

// fp16 also as the bit patterns of int16
int type_of(const Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return SI_F32;
    case at::kBFloat16: return SI_BF16;
    case at::kHalf:
    case at::kShort: return SI_F16;
    default: TORCH_CHECK(false, "a tensor of ", t.scalar_type(), " in the backward pass");
  }
}
void* ptr(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
float* floats(const Tensor& t) { return static_cast<float*>(ptr(t)); }

void check(si_status s) { TORCH_CHECK(s == SI_OK, "status ", (int)s, ": ", si_last_error()); }

Tensor scratch(const Tensor& like, size_t bytes) {
  return bytes ? at::empty({(int64_t)bytes}, like.options().dtype(at::kByte)) : Tensor();
}

// Rows of n values, `ld` elements from row to row.
struct Rows {
  Tensor t;
  size_t ld;
};
constexpr int64_t kMaxLd = (int64_t)1 << 21, kMaxNormLd = (int64_t)1 << 32;  // the library's longest strides
// t [rows][n] as it lies in memory; expanded, transposed or overlapping rows are copied.
Rows rows_of(Tensor t, int64_t n, int64_t max_ld) {
  const bool many = t.size(0) > 1;
  if (!t.is_contiguous() && ((n > 1 && t.stride(1) != 1) || (many && (t.stride(0) < n || t.stride(0) > max_ld))))
    t = t.contiguous();
  return {t, (size_t)(many && !t.is_contiguous() ? t.stride(0) : n)};
}

// One call of a differentiable operator: its saved tensors and sizes, m rows of n to m
// rows of `rows`.
struct Call : Node {
  SavedVariable x, w, w_up, w_down, g, u, h;  // (norms: w, and the rows' mean and r as g, u)
  int64_t m = 0, n = 0, rows = 0;
  int x_type = 0, w_type = 0, y_type = 0;
  c10::Device device{at::kCPU};
  bool flag = false;  // W^T in memory, or LayerNorm
  at::ScalarType y_scalar = at::kFloat;
  void* raw_stream = nullptr;

  void release_variables() override {
    for (SavedVariable* v : {&x, &w, &w_up, &w_down, &g, &u, &h}) v->reset_data();
  }

  // A saved tensor as it is handed back.  Hooks of saved tensors choose its place and
  // strides (save_on_cpu makes a slice contiguous), so both are taken from this tensor,
  // never from the forward call; another type, size or device is refused.
  Tensor kept(const Tensor& t, const char* name, int type, at::IntArrayRef sizes) const {
    TORCH_CHECK(t.defined(), "the saved tensor ", name, " was handed back undefined");
    TORCH_CHECK(t.device() == device, "the saved tensor ", name, " was handed back on ", t.device(), ", not ", device);
    TORCH_CHECK(t.sizes() == sizes, "the saved tensor ", name, " was handed back as ", t.sizes(), ", not ", sizes);
    TORCH_CHECK(t.layout() == at::kStrided && type_of(t) == type, "the saved tensor ", name, " was handed back as ",
                t.scalar_type(), ", another type than it had");
    return t;
  }
  Rows x_rows(int64_t max_ld = kMaxLd) const { return rows_of(kept(x.unpack(), "x", x_type, {m, n}), n, max_ld); }
  Tensor whole(const Tensor& t, const char* name, int type, at::IntArrayRef sizes) const {
    return kept(t, name, type, sizes).contiguous();
  }
  Tensor whole_if(const Tensor& t, const char* name, int type, at::IntArrayRef sizes) const {
    return t.defined() ? whole(t, name, type, sizes) : t;
  }

  // the gradients that are asked for
  virtual void run(const Tensor& grad, variable_list& out) = 0;

  // The gradient of y.  Autograd hands on one of y's size, type and device on the stream of
  // the forward call; the node's own call and its hooks are held to that here.
  Tensor gradient(const Tensor& grad) {
    TORCH_CHECK(grad.device() == device && grad.layout() == at::kStrided, "a gradient on ", grad.device(), ", not ", device);
    TORCH_CHECK(grad.dim() == 2 && grad.size(0) == m && grad.size(1) == y_n(), "a gradient of size ", grad.sizes(), ", not [", m,
                ", ", y_n(), "]");
    const auto forward = stream();
    TORCH_CHECK(!forward.has_value() || *forward == c10::impl::VirtualGuardImpl(device.type()).getStream(device),
                "the backward pass was called on another stream than the forward call's");
    return grad.to(y_scalar).resolve_neg();
  }

  virtual int64_t y_n() const { return rows; }  // values of a row of y

  variable_list apply(variable_list&& in) override {
    std::lock_guard<std::mutex> lock(mutex_);
    const bool graph = at::GradMode::is_enabled();
    variable_list out(num_outputs());
    if (!in[0].defined()) return out;
    {
      at::NoGradGuard none;
      const c10::DeviceGuard guard(device);
      run(gradient(in[0]), out);
    }
    if (!graph) return out;
    // the gradients have none of their own: a graph of them is refused where it is used
    const auto refuse = std::make_shared<torch::autograd::DelayedError>(
        "the gradients of this operator are first order: they cannot be differentiated again", (int64_t)out.size());
    for (Tensor& t : out)
      if (t.defined()) t.requires_grad_();
    return (*refuse)(std::move(out));
  }

  bool wants(size_t i) const { return task_should_compute_output(i); }
  Tensor like(bool want, const Tensor& t) const { return want ? at::empty_like(t) : Tensor(); }
  Tensor dx_of(const Tensor& xt) const { return wants(0) ? at::empty({m, n}, xt.options()) : Tensor(); }
};

// of the products' type or float32
Tensor operand(const Tensor& grad, const Tensor& xt) {
  return grad.scalar_type() == xt.scalar_type() || grad.scalar_type() == at::kFloat ? grad : grad.to(at::kFloat);
}

struct LinearGrad : Call {
  std::string name() const override { return "SparseInferLinearGrad"; }
  void run(const Tensor& grad, variable_list& out) override {
    const Rows xr = x_rows();
    const Tensor &xt = xr.t, wt = flag ? whole(w.unpack(), "w", w_type, {n, rows}) : whole(w.unpack(), "w", w_type, {rows, n});
    const Rows dy = rows_of(operand(grad, xt), rows, kMaxLd);
    out = {dx_of(xt), like(wants(1), wt)};
    const size_t bytes = si_linear_backward_workspace_bytes(ptr(dy.t), type_of(dy.t), dy.ld, ptr(xt), xr.ld, m, n, ptr(wt),
                                                            rows, flag, out[0].defined(), out[1].defined());
    const Tensor ws = scratch(xt, bytes);
    check(si_linear_backward(ptr(dy.t), type_of(dy.t), dy.ld, ptr(xt), x_type, xr.ld, m, n, ptr(wt), rows, flag, ptr(out[0]),
                             ptr(out[1]), ptr(ws), bytes, raw_stream));
  }
};

struct GatedGrad : Call {
  std::string name() const override { return "SparseInferGatedLinearGrad"; }
  void run(const Tensor& grad, variable_list& out) override {
    const Rows xr = x_rows();
    const Tensor &xt = xr.t, wt = whole(w.unpack(), "w_gate", w_type, {rows, n}),
                 up = whole_if(w_up.unpack(), "w_up", w_type, {rows, n});
    const Tensor ut = up.defined() ? whole(u.unpack(), "u", SI_F32, {m, rows}) : Tensor();
    const Tensor gt = up.defined() ? whole(g.unpack(), "g", SI_F32, {m, rows})
                                   : whole(h.unpack(shared_from_this()), "h", y_type, {m, rows});
    const Rows dh = rows_of(grad, rows, kMaxLd);
    out = {dx_of(xt), like(wants(1), wt), like(wants(2), up)};
    const size_t bytes = si_gated_linear_backward_workspace_bytes(ptr(xt), xr.ld, m, n, ptr(wt), ptr(up), rows,
                                                                  out[0].defined(), out[1].defined() || out[2].defined());
    const Tensor ws = scratch(xt, bytes);
    check(si_gated_linear_backward(ptr(dh.t), type_of(dh.t), dh.ld, ptr(gt), type_of(gt), floats(ut), ptr(xt), x_type, xr.ld,
                                   m, n, ptr(wt), ptr(up), rows, ptr(out[0]), ptr(out[1]), ptr(out[2]), ptr(ws), bytes,
                                   raw_stream));
  }
};

struct MlpGrad : Call {
  int64_t y_n() const override { return n; }
  std::string name() const override { return "SparseInferMlpGrad"; }
  void run(const Tensor& grad, variable_list& out) override {
    const Rows xr = x_rows();
    const Tensor &xt = xr.t, wt = whole(w.unpack(), "w_gate", w_type, {rows, n}),
                 up = whole_if(w_up.unpack(), "w_up", w_type, {rows, n}),
                 down = whole(w_down.unpack(), "w_down", w_type, {n, rows}), ht = whole(h.unpack(), "h", x_type, {m, rows});
    const Tensor gt = up.defined() ? whole(g.unpack(), "g", SI_F32, {m, rows}) : Tensor(),
                 ut = up.defined() ? whole(u.unpack(), "u", SI_F32, {m, rows}) : Tensor();
    const Rows dy = rows_of(operand(grad, xt), n, kMaxLd);
    out = {dx_of(xt), like(wants(1), wt), like(wants(2), up), like(wants(3), down)};
    const size_t bytes = si_mlp_backward_workspace_bytes(ptr(dy.t), type_of(dy.t), dy.ld, ptr(xt), xr.ld, m, n, ptr(wt),
                                                         ptr(up), ptr(down), rows, out[0].defined(),
                                                         out[1].defined() || out[2].defined(), out[3].defined());
    const Tensor ws = scratch(xt, bytes);
    check(si_mlp_backward(ptr(dy.t), type_of(dy.t), dy.ld, ptr(xt), x_type, xr.ld, m, n, ptr(wt), ptr(up), ptr(down), rows,
                          ptr(ht), floats(gt), floats(ut), ptr(out[0]), ptr(out[1]), ptr(out[2]), ptr(out[3]), ptr(ws), bytes,
                          raw_stream));
  }
};

struct NormGrad : Call {
  std::string name() const override { return flag ? "SparseInferLayerNormGrad" : "SparseInferRmsNormGrad"; }
  void run(const Tensor& grad, variable_list& out) override {
    const Rows xr = x_rows(kMaxNormLd);
    const Tensor &xt = xr.t, wt = whole(w.unpack(), "w", w_type, {n}), r = whole(u.unpack(), "r", SI_F32, {m});
    const Tensor mean = flag ? whole(g.unpack(), "mean", SI_F32, {m}) : Tensor();
    const Rows dy = rows_of(grad, n, kMaxNormLd);
    out = {dx_of(xt), like(wants(1), wt), like(wants(2), wt)};
    const size_t bytes = out[1].defined() || out[2].defined() ? si_layer_norm_backward_workspace_bytes(m, n) : 0;
    const Tensor ws = scratch(xt, bytes);
    check(si_layer_norm_backward(ptr(dy.t), dy.ld, ptr(xt), x_type, xr.ld, ptr(wt), w_type, flag, floats(mean), floats(r),
                                 ptr(out[0]), ptr(out[1]), ptr(out[2]), m, n, ptr(ws), bytes, raw_stream));
  }
};

using Maybe = std::optional<Tensor>;
Tensor given(const Maybe& t) { return t.value_or(Tensor()); }
SavedVariable saved(const Maybe& t, bool output = false) {
  return t.has_value() ? SavedVariable(*t, output) : SavedVariable();
}

// While an eager graph of a leaf lives, the leaf's place for gradients belongs to that
// graph's stream, and a backward pass captured on another one would end the capture, and
// the process, where autograd lets the two streams wait for each other.  A view (the rows
// of a leaf of more dimensions, a slice of one) hands its gradients to its base.
void refuse_foreign_leaf(const Tensor& t) {
  if (!t.defined() || !t.requires_grad()) return;
  const at::TensorBase& leaf = !t.is_leaf() && t.is_view() ? t._base() : t;
  if (!leaf.requires_grad() || !leaf.is_leaf()) return;
  const auto place = torch::autograd::impl::try_get_grad_accumulator(leaf);
  if (!place || !place->stream().has_value()) return;
  if (*place->stream() == c10::impl::VirtualGuardImpl(t.device().type()).getStream(t.device())) return;
  TORCH_CHECK(!py::module_::import("torch.cuda").attr("is_current_stream_capturing")().cast<bool>(),
              "a call under capture with a leaf of an eager graph that still lives: release that graph first, or capture "
              "with leaves of the graph's own");
}

// The node of a call that has been made, and y as its output.
template <class T, class... Inputs>  // (Inputs: tensors)
std::shared_ptr<T> attach(Tensor y, int m, int n, int rows, bool flag, uintptr_t stream, const Tensor& x,
                          const Tensor& w, const Inputs&... more) {
  for (const Tensor* t : {&x, &w, &more...}) refuse_foreign_leaf(*t);
  auto call = std::shared_ptr<T>(new T(), torch::autograd::deleteNode);
  call->set_next_edges(torch::autograd::collect_next_edges(x, w, more...));
  call->x = SavedVariable(x, false);
  call->w = SavedVariable(w, false);
  call->m = m;
  call->n = n;
  call->rows = rows;
  call->x_type = type_of(x);
  call->w_type = type_of(w);
  call->y_type = type_of(y);
  call->device = x.device();
  call->flag = flag;
  call->y_scalar = y.scalar_type();
  call->raw_stream = reinterpret_cast<void*>(stream);
  torch::autograd::set_history(y, call);
  return call;
}

void linear(const Tensor& y, const Tensor& x, const Tensor& w, int m, int n, int rows, bool transposed,
            uintptr_t stream) {
  attach<LinearGrad>(y, m, n, rows, transposed, stream, x, w);
}

void gated_linear(const Tensor& h, const Tensor& x, const Tensor& w_gate, const Maybe& w_up, const Maybe& g, const Maybe& u,
                  int m, int n, int rows, uintptr_t stream) {
  const auto c = attach<GatedGrad>(h, m, n, rows, false, stream, x, w_gate, given(w_up));
  c->w_up = saved(w_up);
  c->g = saved(g);
  c->u = saved(u);
  if (!w_up.has_value()) c->h = SavedVariable(h, true);
}

void mlp(const Tensor& y, const Tensor& x, const Tensor& w_gate, const Maybe& w_up, const Tensor& w_down, const Tensor& h,
         const Maybe& g, const Maybe& u, int m, int n, int rows, uintptr_t stream) {
  const auto c = attach<MlpGrad>(y, m, n, rows, false, stream, x, w_gate, given(w_up), w_down);
  c->w_up = saved(w_up);
  c->w_down = SavedVariable(w_down, false);
  c->h = SavedVariable(h, false);
  c->g = saved(g);
  c->u = saved(u);
}

void norm(const Tensor& y, const Tensor& x, const Tensor& w, const Maybe& b, const Maybe& mean, const Tensor& r, int tokens,
          int d, bool center, uintptr_t stream) {
  const auto c = attach<NormGrad>(y, tokens, d, d, center, stream, x, w, given(b));
  c->g = saved(mean);
  c->u = SavedVariable(r, false);
}

}  // namespace

PYBIND11_MODULE(_autograd, module) {
  module.def("refuse_foreign_leaf", &refuse_foreign_leaf);
  module.def("linear", &linear);
  module.def("gated_linear", &gated_linear);
  module.def("mlp", &mlp);
  module.def("norm", &norm);
}
