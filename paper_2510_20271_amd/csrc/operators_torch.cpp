// The autograd functions of the normalisation and of the head's loss in C++, for plain contiguous tensors (norm.py and loss.py
// choose; their Python functions give the same results).  Small steps are as long as the host takes for them: a step on 1024
// curves of 128 thresholds (26 us of kernels) took 122 us through the Python functions.
#include "layer_torch.h"

namespace {

ecc_dtype code_of(const Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return ECC_F32;
    case at::kHalf: return ECC_F16;
    case at::kBFloat16: return ECC_BF16;
    default: TORCH_CHECK_VALUE(false, "tensors must be float32, float16 or bfloat16");
  }
}
Tensor room(size_t bytes, const Tensor& like) { return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte)); }
void* at_or_null(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// These backward passes are not differentiable themselves: gradients made for a graph are tied to what they depend on, the saved
// inputs included, by a function that refuses.
constexpr const char* kOnce = "this operator's backward pass is not differentiable a second time";
struct Refuse : public torch::autograd::Function<Refuse> {
  static Tensor forward(AutogradContext*, const Tensor& grad, const Tensor& up, const Tensor& a, const c10::optional<Tensor>&,
                        const c10::optional<Tensor>&) {
    return grad.alias();
  }
  static variable_list backward(AutogradContext*, variable_list) { TORCH_CHECK(false, kOnce); }
};
void once(variable_list& grads, const Tensor& up, const Tensor& a, const Tensor& b, const Tensor& c = Tensor()) {
  if (!at::GradMode::is_enabled()) return;
  const auto some = [](const Tensor& t) { return t.defined() ? c10::optional<Tensor>(t) : c10::nullopt; };
  for (Tensor& g : grads)
    if (g.defined()) g = Refuse::apply(g, up, a, some(b), some(c));
}

struct NormSizes {
  int64_t batch, points;
  int channels;
  explicit NormSizes(const Tensor& x) : batch(x.size(0)), points(1), channels((int)x.size(-1)) {
    for (int64_t k = 1; k + 1 < x.dim(); ++k) points *= x.size(k);
  }
};

Tensor norm_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, int groups, float eps, int act, Tensor* stats) {
  const NormSizes s(x);
  Tensor y = at::empty(x.sizes(), x.options());
  if (stats) *stats = at::empty({s.batch, groups, 2}, x.options().dtype(at::kDouble));
  const Tensor ws = room(ecc_norm_workspace_bytes(s.batch, s.points, s.channels, groups), x);
  check(ecc_norm_fwd(x.data_ptr(), s.batch, s.points, s.channels, groups, code_of(x), f32(weight), f32(bias), eps, act,
                     y.data_ptr(), stats ? stats->data_ptr<double>() : nullptr, ws.data_ptr(), (size_t)ws.numel(), stream()));
  return y;
}

struct Norm : public torch::autograd::Function<Norm> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const c10::optional<Tensor>& w, const c10::optional<Tensor>& b,
                        int64_t groups, double eps, int64_t act) {
    const Tensor weight = w.value_or(Tensor()), bias = b.value_or(Tensor());
    Tensor stats;
    Tensor y = norm_forward(x, weight, bias, (int)groups, (float)eps, (int)act, &stats);
    ctx->save_for_backward({x, weight, bias, stats});
    ctx->saved_data["groups"] = groups;
    ctx->saved_data["act"] = act;
    return y;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const variable_list saved = ctx->get_saved_variables();
    const Tensor &x = saved[0], &weight = saved[1], &bias = saved[2], &stats = saved[3];
    const int groups = (int)ctx->saved_data["groups"].toInt(), act = (int)ctx->saved_data["act"].toInt();
    const Tensor dy = grads[0].contiguous();
    check_device(x, x.scalar_type(), -1, x.device());
    TORCH_CHECK_VALUE(x.is_cuda() && x.dim() >= 2, "x must be a device tensor [batch, (points,) channels]");
    const NormSizes s(x);
    check_device(dy, x.scalar_type(), x.numel(), x.device());
    check_device(stats, at::kDouble, s.batch * groups * 2, x.device());
    if (weight.defined()) check_device(weight, at::kFloat, s.channels, x.device());
    if (bias.defined()) check_device(bias, at::kFloat, s.channels, x.device());
    const auto opts = x.options().dtype(at::kFloat);
    Tensor dx, dw, db;
    if (ctx->needs_input_grad(0)) dx = at::empty(x.sizes(), x.options());
    // (inputs that are there are numbered without those that are not)
    if (weight.defined() && ctx->needs_input_grad(1)) dw = at::empty({s.channels}, opts);
    if (bias.defined() && ctx->needs_input_grad(weight.defined() ? 2 : 1)) db = at::empty({s.channels}, opts);
    if (dx.defined() || dw.defined() || db.defined()) {
      const Tensor ws = room(ecc_norm_workspace_bytes(s.batch, s.points, s.channels, groups), x);
      check(ecc_norm_bwd(x.data_ptr(), dy.data_ptr(), s.batch, s.points, s.channels, groups, code_of(x), f32(weight), f32(bias),
                         act, stats.data_ptr<double>(), at_or_null(dx), f32(dw), f32(db), ws.data_ptr(), (size_t)ws.numel(),
                         stream()));
    }
    variable_list out{dx, dw, db, Tensor(), Tensor(), Tensor()};
    once(out, grads[0], x, weight, bias);
    return out;
  }
};

// x contiguous [batch, ..., channels]; weight, bias contiguous float32 [channels] or none; sizes as norm.py has checked them
Tensor norm_act(const Tensor& x, const c10::optional<Tensor>& weight, const c10::optional<Tensor>& bias, int64_t groups, double eps,
                int64_t act) {
  const Tensor w = weight.value_or(Tensor()), b = bias.value_or(Tensor());
  const bool graph = at::GradMode::is_enabled() && (x.requires_grad() || (w.defined() && w.requires_grad()) ||
                                                    (b.defined() && b.requires_grad()));
  if (graph) return Norm::apply(x, weight, bias, groups, eps, act);
  return norm_forward(x, w, b, (int)groups, (float)eps, (int)act, nullptr);
}

size_t xent_room(const Tensor& h, const Tensor& w, int flags) {
  if (((uintptr_t)h.data_ptr() | (uintptr_t)w.data_ptr()) % 16 == 0) flags |= ECC_XENT_ALIGNED;
  return ecc_xent_workspace_bytes(h.size(0), (int)h.size(1), w.size(0), code_of(h), flags);
}

Tensor xent_forward(const Tensor& h, const Tensor& w, const Tensor& labels, int64_t ignore, int reduction, Tensor* stats,
                    Tensor* counted) {
  const int64_t rows = h.size(0), classes = w.size(0);
  const int dim = (int)h.size(1);
  const auto opts = h.options().dtype(at::kFloat);
  Tensor loss = reduction == ECC_EACH ? at::empty({rows}, opts) : at::empty({}, opts);
  if (stats) {
    *stats = at::empty({rows, 2}, h.options().dtype(at::kDouble));
    *counted = at::empty({}, h.options().dtype(at::kLong));
  }
  const Tensor ws = room(xent_room(h, w, 0), h);
  check(ecc_xent_fwd(h.data_ptr(), w.data_ptr(), labels.data_ptr<int64_t>(), rows, dim, classes, code_of(h), ignore, reduction,
                     loss.data_ptr<float>(), stats ? stats->data_ptr<double>() : nullptr,
                     stats ? counted->data_ptr<int64_t>() : nullptr, ws.data_ptr(), (size_t)ws.numel(), stream()));
  return loss;
}

struct Xent : public torch::autograd::Function<Xent> {
  static Tensor forward(AutogradContext* ctx, const Tensor& h, const Tensor& w, const Tensor& labels, int64_t ignore,
                        int64_t reduction) {
    Tensor stats, counted;
    Tensor loss = xent_forward(h, w, labels, ignore, (int)reduction, &stats, &counted);
    ctx->save_for_backward({h, w, labels, stats, counted});
    ctx->saved_data["ignore"] = ignore;
    ctx->saved_data["reduction"] = reduction;
    return loss;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const variable_list saved = ctx->get_saved_variables();
    const Tensor &h = saved[0], &w = saved[1], &labels = saved[2], &stats = saved[3], &counted = saved[4];
    const int64_t ignore = ctx->saved_data["ignore"].toInt();
    const int reduction = (int)ctx->saved_data["reduction"].toInt();
    const Tensor up = grads[0].contiguous().to(at::kFloat);
    check_device(h, h.scalar_type(), -1, h.device());
    TORCH_CHECK_VALUE(h.is_cuda() && h.dim() == 2 && w.dim() == 2 && w.size(1) == h.size(1),
                      "hidden must be a device tensor [rows, dim] and weight [classes, dim]");
    const int64_t rows = h.size(0), classes = w.size(0);
    const int dim = (int)h.size(1);
    check_device(w, h.scalar_type(), -1, h.device());
    check_device(labels, at::kLong, rows, h.device());
    check_device(stats, at::kDouble, rows * 2, h.device());
    check_device(counted, at::kLong, 1, h.device());
    check_device(up, at::kFloat, reduction == ECC_EACH ? rows : 1, h.device());
    Tensor dh, dw;
    if (ctx->needs_input_grad(0)) dh = at::empty(h.sizes(), h.options());
    if (ctx->needs_input_grad(1)) dw = at::empty(w.sizes(), w.options());
    if (dh.defined() || dw.defined()) {
      const Tensor ws = room(xent_room(h, w, ECC_XENT_BACKWARD), h);
      check(ecc_xent_bwd(h.data_ptr(), w.data_ptr(), labels.data_ptr<int64_t>(), rows, dim, classes, code_of(h), ignore, reduction,
                         stats.data_ptr<double>(), counted.data_ptr<int64_t>(), up.data_ptr<float>(), at_or_null(dh),
                         at_or_null(dw), ws.data_ptr(), (size_t)ws.numel(), stream()));
    }
    variable_list out{dh, dw, Tensor(), Tensor(), Tensor()};
    once(out, grads[0], h, w);
    return out;
  }
};

// hidden [rows, dim], weight [classes, dim], labels [rows], contiguous, as loss.py has checked them
Tensor linear_xent(const Tensor& h, const Tensor& w, const Tensor& labels, int64_t ignore, int64_t reduction) {
  if (at::GradMode::is_enabled() && (h.requires_grad() || w.requires_grad())) return Xent::apply(h, w, labels, ignore, reduction);
  return xent_forward(h, w, labels, ignore, (int)reduction, nullptr, nullptr);
}

}  // namespace

void bind_operators(py::module_& m) {
  m.def("norm_act", &norm_act, "Group norm with an activation, differentiable", py::call_guard<py::gil_scoped_release>());
  m.def("linear_xent", &linear_xent, "Cross entropy of a linear head, differentiable", py::call_guard<py::gil_scoped_release>());
}
