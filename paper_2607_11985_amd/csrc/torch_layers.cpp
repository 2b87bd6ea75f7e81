// torch_layers.cpp -- the layers of include/vqc.h on torch tensors, with their gradients in
// torch's autograd (the Python module vqc_torch, which layers.py wraps).
//
// Native because of the host's time: torch runs the backward of a CUDA graph on a thread of its
// own, and a backward written in Python has to take the interpreter's lock there and give it
// back: 108 us of host time for the forward and backward of a 64 x 10 scores call, against
// 24 us of both kernels' launches.  Only arguments are handled here: every computation is in
// libvqc.so, memory and streams are torch's.
#include <ATen/ATen.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <pybind11/stl.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/utils/pybind.h>

#include <string>
#include <tuple>
#include <vector>

#include "vqc.h"

namespace py = pybind11;

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// A status of the library, raised in Python as the binding's VQCError.
struct StatusError : std::runtime_error {
  int code;
  StatusError(int c, const std::string& m) : std::runtime_error(m), code(c) {}
};
PyObject* g_error_type = nullptr;

void check(int rc) {
  if (rc) throw StatusError(rc, vqc_last_error());
}

template <typename... A>
[[noreturn]] void refuse(const A&... a) {
  throw py::value_error(c10::str(a...));
}

int dtype_of(const Tensor& x, const char* name) {
  int code = -1;
  switch (x.scalar_type()) {
    case at::kFloat: code = VQC_F32; break;
    case at::kHalf: code = VQC_F16; break;
    case at::kBFloat16: code = VQC_BF16; break;
    default: refuse(name, " must be float32, float16 or bfloat16, got ", x.scalar_type());
  }
  if (!x.is_cuda()) refuse(name, " must be a cuda tensor");
  return code;
}

void check_like(const Tensor& x, const Tensor& like, const char* name) {
  if (x.scalar_type() != like.scalar_type() || x.device() != like.device())
    refuse(name, " must be ", like.scalar_type(), " on ", like.device(), ", got ",
           x.scalar_type(), " on ", x.device());
}

// Without a pending sign (torch holds the imaginary part of a conjugate with one).
Tensor signed_values(const Tensor& x) { return x.is_neg() ? x.resolve_neg() : x; }

// x as [rows, width], each row's elements adjacent (a copy only where leading dimensions do not
// merge).
Tensor matrix(const Tensor& x, int64_t width, const char* name) {
  if (x.dim() < 1 || x.size(-1) != width)
    refuse(name, " must have rows of ", width, ", got ", x.sizes());
  if (width > 1 && x.stride(-1) != 1)
    refuse("the elements of a row of ", name, " must be adjacent, got strides ", x.strides());
  if (x.dim() == 2) return signed_values(x);
  int64_t rows = 1;
  for (int64_t i = 0; i + 1 < x.dim(); ++i) rows *= x.size(i);
  return signed_values(x).reshape({rows, width});
}

Tensor vector_of(const Tensor& x, int64_t width, const Tensor& like, const char* name) {
  if (!x.defined()) return x;
  if (x.scalar_type() != like.scalar_type() || x.device() != like.device() || x.dim() != 1 ||
      x.size(0) != width || !x.is_contiguous())
    refuse(name, " must be a contiguous ", like.scalar_type(), " tensor of ", width,
           " elements on ", like.device());
  return signed_values(x);
}

// A cotangent as rows of adjacent elements (autograd may hand over expanded tensors).
Tensor cotangent(const Tensor& g, int64_t rows, int64_t width, const Tensor& like) {
  Tensor m = signed_values(g);
  if (m.dim() != 2) m = m.reshape({rows, width});
  if (m.scalar_type() != like.scalar_type()) m = m.to(like.scalar_type());
  return width <= 1 || m.stride(1) == 1 ? m : m.contiguous();
}

void* stream_of(const Tensor& x) {
  return c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(x.device().index()).stream();
}

Tensor workspace(size_t bytes, const Tensor& like) {
  if (!bytes) return Tensor();
  return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
}

template <typename T = void>
T* pointer(const Tensor& x) {
  return x.defined() ? static_cast<T*>(x.data_ptr()) : nullptr;
}

std::vector<int64_t> with_last(at::IntArrayRef shape, int64_t last) {
  std::vector<int64_t> s(shape.begin(), shape.end());
  s.back() = last;
  return s;
}

bool wants_grad(std::initializer_list<const Tensor*> xs) {
  if (!at::GradMode::is_enabled()) return false;
  for (const Tensor* x : xs)
    if (x->defined() && x->requires_grad()) return true;
  return false;
}

// A tensor that carries a tangent of forward-mode differentiation need not want a gradient, and its
// tangent would be lost in the result without a word.
void check_no_tangent(std::initializer_list<const Tensor*> xs) {
  if (!c10::AutogradState::get_tls_state().get_fw_grad_mode()) return;
  for (const Tensor* x : xs)
    if (x->defined() && x->_fw_grad(0).defined())
      refuse("the layers have no forward-mode derivatives: an input carries a tangent");
}

// A bit for each of a call's inputs.
using Inputs = int64_t;

Inputs inputs_with_grad(std::initializer_list<const Tensor*> xs) {
  Inputs bits = 0;
  int i = 0;
  for (const Tensor* x : xs) bits |= (Inputs)(x->defined() && x->requires_grad()) << i++;
  return bits;
}

// The gradients are not differentiable themselves.  With create_graph, one that depends on
// something that wants a gradient (a cotangent, or an input of its `on`) leads autograd to an error
// where it goes on through it; the others are constants.
variable_list only_once(variable_list grads, const variable_list& cotangents, Inputs with_grad,
                        std::initializer_list<Inputs> on) {
  if (!at::GradMode::is_enabled()) return grads;
  bool all = false;
  for (const auto& g : cotangents) all = all || (g.defined() && g.requires_grad());
  std::vector<size_t> which;
  variable_list raising;
  for (size_t i = 0; i < on.size(); ++i) {
    if (!grads[i].defined()) continue;
    if (!all && !(with_grad & on.begin()[i])) continue;
    which.push_back(i);
    raising.push_back(grads[i].detach().set_requires_grad(true));
  }
  if (which.empty()) return grads;
  auto node = std::make_shared<torch::autograd::DelayedError>(
      "the layers' gradients cannot be differentiated again", (int64_t)which.size());
  const variable_list out = (*node)(std::move(raising));
  for (size_t k = 0; k < which.size(); ++k) grads[which[k]] = out[k];
  return grads;
}

using Maybe = std::optional<Tensor>;
Tensor given(const Maybe& x) { return x ? *x : Tensor(); }

// Whether input i of a call wants a gradient.  Autograd counts the tensors that were given:
// `present` has a bit for each input that was.
bool wanted(AutogradContext* ctx, int64_t present, int i) {
  if (!(present >> i & 1)) return false;
  return ctx->needs_input_grad((size_t)__builtin_popcountll(present & ((1ll << i) - 1)));
}

// ------------------------------------------------------------------ layer norm

Tensor norm_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, double eps,
                    Tensor* stats) {
  const int code = dtype_of(x, "x");
  if (x.dim() < 1 || x.size(-1) < 1)
    refuse("x must have rows of at least one element, got ", x.sizes());
  const int64_t cols = x.size(-1);
  const Tensor xm = matrix(x, cols, "x");
  const int64_t rows = xm.size(0);
  const Tensor w = vector_of(weight, cols, x, "weight"), b = vector_of(bias, cols, x, "bias");
  Tensor y = at::empty(x.sizes(), x.options());
  float* mean = nullptr;
  if (stats) {
    *stats = at::empty({2, rows}, x.options().dtype(at::kFloat));
    mean = stats->data_ptr<float>();
  }
  const c10::DeviceGuard guard(x.device());
  check(vqc_layer_norm(code, rows, cols, xm.data_ptr(), xm.stride(0), pointer(w),
                       pointer(b), (float)eps, y.data_ptr(), cols, mean,
                       mean ? mean + rows : nullptr, stream_of(x)));
  return y;
}

struct LayerNorm : torch::autograd::Function<LayerNorm> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const Maybe& weight,
                        const Maybe& bias, double eps, Inputs with_grad) {
    Tensor stats;
    Tensor y = norm_forward(x, given(weight), given(bias), eps, &stats);
    ctx->save_for_backward({x, given(weight), stats});
    ctx->saved_data["with_grad"] = with_grad;
    ctx->saved_data["present"] = (int64_t)(1 | (weight ? 2 : 0) | (bias ? 4 : 0));
    return y;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const variable_list saved = ctx->get_saved_variables();
    const Tensor &x = saved[0], &stats = saved[2];
    const Tensor weight = saved[1].defined() ? signed_values(saved[1]) : saved[1];
    const int64_t cols = x.size(-1);
    const Tensor xm = matrix(x, cols, "x");
    const int64_t rows = xm.size(0);
    const Tensor dy = cotangent(grads[0], rows, cols, x);
    const int64_t present = ctx->saved_data["present"].toInt();
    Tensor dx, dw, db;
    if (wanted(ctx, present, 0)) dx = at::empty(x.sizes(), x.options());
    if (wanted(ctx, present, 1)) dw = at::empty({cols}, x.options());
    if (wanted(ctx, present, 2)) db = at::empty({cols}, x.options());
    const size_t bytes = dw.defined() || db.defined()
                             ? vqc_layer_norm_workspace_bytes(rows, cols) : 0;
    const Tensor ws = workspace(bytes, x);
    const float* mean = stats.data_ptr<float>();
    const c10::DeviceGuard guard(x.device());
    check(vqc_layer_norm_backward(dtype_of(x, "x"), rows, cols, xm.data_ptr(), xm.stride(0),
                                  pointer(weight), mean, mean + rows, dy.data_ptr(),
                                  dy.stride(0), pointer(dx), cols, pointer(dw), pointer(db),
                                  pointer(ws), bytes, stream_of(x)));
    // of x and the weight, of x, of the cotangent alone
    return only_once({dx, dw, db, Tensor(), Tensor()}, grads,
                     ctx->saved_data["with_grad"].toInt(), {3, 1, 0});
  }
};

Tensor layer_norm(const Tensor& x, const Maybe& weight, const Maybe& bias, double eps) {
  const Tensor w = given(weight), b = given(bias);
  check_no_tangent({&x, &w, &b});
  if (wants_grad({&x, &w, &b}))
    return LayerNorm::apply(x, weight, bias, eps, inputs_with_grad({&x, &w, &b}));
  return norm_forward(x, w, b, eps, nullptr);
}

// ------------------------------------------------------------------ linear

Tensor linear_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, int64_t act,
                      const Tensor& residual, Tensor* pre) {
  const int code = dtype_of(x, "x");
  if (weight.dim() != 2) refuse("weight must be [n_out, n_in], got ", weight.sizes());
  const int64_t n_out = weight.size(0), n_in = weight.size(1);
  const Tensor xm = matrix(x, n_in, "x");
  check_like(weight, x, "weight");
  const Tensor wm = matrix(weight, n_in, "weight"), b = vector_of(bias, n_out, x, "bias");
  const int64_t rows = xm.size(0);
  const std::vector<int64_t> shape = with_last(x.sizes(), n_out);
  Tensor rm;
  if (residual.defined()) {
    if (residual.sizes() != at::IntArrayRef(shape))
      refuse("residual must have shape ", at::IntArrayRef(shape), ", got ", residual.sizes());
    check_like(residual, x, "residual");
    rm = matrix(residual, n_out, "residual");
  }
  Tensor y = at::empty(shape, x.options());
  if (pre && act) *pre = at::empty({rows, n_out}, x.options().dtype(at::kFloat));
  const size_t bytes = vqc_linear_workspace_bytes(code, rows, n_in, n_out, 0);
  const Tensor ws = workspace(bytes, x);
  const c10::DeviceGuard guard(x.device());
  check(vqc_linear(code, rows, n_in, n_out, xm.data_ptr(), xm.stride(0), wm.data_ptr(),
                   wm.stride(0), pointer(b), (int32_t)act, pointer(rm),
                   rm.defined() ? rm.stride(0) : 0, y.data_ptr(), n_out,
                   pre ? pointer<float>(*pre) : nullptr, pointer(ws), bytes, stream_of(x)));
  return y;
}

struct Linear : torch::autograd::Function<Linear> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& weight,
                        const Maybe& bias, int64_t act, const Maybe& residual, Inputs with_grad) {
    Tensor pre;
    Tensor y = linear_forward(x, weight, given(bias), act, given(residual), &pre);
    ctx->save_for_backward({x, weight, pre});
    ctx->saved_data["act"] = act;
    ctx->saved_data["with_grad"] = with_grad;
    ctx->saved_data["present"] = (int64_t)(3 | (bias ? 4 : 0) | (residual ? 8 : 0));
    return y;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const int64_t present = ctx->saved_data["present"].toInt();
    const bool need_x = wanted(ctx, present, 0), need_w = wanted(ctx, present, 1),
               need_b = wanted(ctx, present, 2);
    Tensor dx, dw, db;
    if (need_x || need_w || need_b) {
      const variable_list saved = ctx->get_saved_variables();
      const Tensor &x = saved[0], &weight = saved[1], &pre = saved[2];
      const int64_t n_out = weight.size(0), n_in = weight.size(1);
      const int code = dtype_of(x, "x");
      const Tensor xm = matrix(x, n_in, "x"), wm = matrix(weight, n_in, "weight");
      const int64_t rows = xm.size(0);
      const Tensor dy = cotangent(grads[0], rows, n_out, x);
      if (need_x) dx = at::empty(x.sizes(), x.options());
      if (need_w) dw = at::empty({n_out, n_in}, x.options());
      if (need_b) db = at::empty({n_out}, x.options());
      const size_t bytes = vqc_linear_workspace_bytes(code, rows, n_in, n_out, 1);
      const Tensor ws = workspace(bytes, x);
      const c10::DeviceGuard guard(x.device());
      check(vqc_linear_backward(code, rows, n_in, n_out, xm.data_ptr(), xm.stride(0),
                                wm.data_ptr(), wm.stride(0),
                                (int32_t)ctx->saved_data["act"].toInt(), pointer<float>(pre),
                                dy.data_ptr(), dy.stride(0), pointer(dx), n_in, pointer(dw),
                                n_in, pointer(db), pointer(ws), bytes, stream_of(x)));
    }
    // a slope that is no constant makes every gradient one of x, the weight and the bias
    const int64_t act = ctx->saved_data["act"].toInt();
    const Inputs slope = act == VQC_ACT_NONE || act == VQC_ACT_RELU ? 0 : 7;
    variable_list out =
        only_once({dx, dw, db, Tensor(), Tensor(), Tensor()}, grads,
                  ctx->saved_data["with_grad"].toInt(), {slope | 2, slope | 1, slope});
    if (wanted(ctx, present, 3)) out[4] = grads[0];
    return out;
  }
};

Tensor linear(const Tensor& x, const Tensor& weight, const Maybe& bias, int64_t act,
              const Maybe& residual) {
  const Tensor b = given(bias), r = given(residual);
  check_no_tangent({&x, &weight, &b, &r});
  if (wants_grad({&x, &weight, &b, &r}))
    return Linear::apply(x, weight, bias, act, residual, inputs_with_grad({&x, &weight, &b, &r}));
  return linear_forward(x, weight, b, act, r, nullptr);
}

// ------------------------------------------------------------------ scores

// logp, entropy, top_logp and top_index; and what the backward keeps.
struct Scores {
  Tensor logp, entropy, top_logp, top_index, targets, stats;
  int64_t shots = 0;
};

Scores scores_forward(const Tensor& scores, const Tensor& targets, int64_t top, int64_t kind,
                      double inv_t, bool keep) {
  const int code = dtype_of(scores, "scores");
  if (scores.dim() < 1 || scores.size(-1) < 1)
    refuse("scores must have rows of at least one outcome, got ", scores.sizes());
  const int64_t cols = scores.size(-1);
  const at::IntArrayRef lead = scores.sizes().slice(0, scores.dim() - 1);
  if (top < 0 || top > cols || top > VQC_MAX_TOP)
    refuse("top must be in [0, min(", cols, ", ", VQC_MAX_TOP, ")], got ", top);
  const Tensor sm = matrix(scores, cols, "scores");
  const int64_t rows = sm.size(0);
  const auto f32 = scores.options().dtype(at::kFloat);
  Scores out;
  if (targets.defined()) {
    if (targets.scalar_type() != at::kLong || targets.device() != scores.device())
      refuse("targets must be int64 on ", scores.device(), ", got ", targets.scalar_type(),
             " on ", targets.device());
    if (targets.sizes() == lead)
      out.shots = 1;
    else if (targets.dim() == scores.dim() &&
             targets.sizes().slice(0, targets.dim() - 1) == lead)
      out.shots = targets.size(-1);
    else
      refuse("targets must have shape ", lead, " or one dimension more, got ", targets.sizes());
    out.targets = targets.contiguous();
    out.logp = at::empty(targets.sizes(), f32);
  } else {
    out.logp = at::empty(with_last(scores.sizes(), 0), f32);
  }
  out.entropy = at::empty(lead, f32);
  const std::vector<int64_t> tops = with_last(scores.sizes(), top);
  out.top_logp = at::empty(tops, f32);
  out.top_index = at::empty(tops, f32.dtype(at::kLong));
  if (keep) out.stats = at::empty({rows, 2}, f32);
  const size_t bytes = vqc_log_probs_workspace_bytes(rows, cols, (int32_t)top);
  const Tensor ws = workspace(bytes, scores);
  const c10::DeviceGuard guard(scores.device());
  check(vqc_log_probs((int32_t)kind, code, rows, cols, sm.data_ptr(), sm.stride(0), (float)inv_t,
                      out.shots ? pointer<int64_t>(out.targets) : nullptr, out.shots,
                      out.shots ? pointer<float>(out.logp) : nullptr,
                      pointer<float>(out.entropy), (int32_t)top,
                      top ? pointer<float>(out.top_logp) : nullptr,
                      top ? pointer<int64_t>(out.top_index) : nullptr, pointer<float>(out.stats),
                      pointer(ws), bytes, stream_of(scores)));
  return out;
}

struct LogProbs : torch::autograd::Function<LogProbs> {
  static variable_list forward(AutogradContext* ctx, const Tensor& scores, const Maybe& targets,
                               int64_t top, double inv_t) {
    Scores s = scores_forward(scores, given(targets), top, VQC_SCORES_LOGITS, inv_t, true);
    ctx->save_for_backward({scores, s.targets, s.stats, s.entropy});
    ctx->saved_data["shots"] = s.shots;
    ctx->saved_data["inv_t"] = inv_t;
    ctx->mark_non_differentiable({s.top_logp, s.top_index});
    ctx->set_materialize_grads(false);
    return {s.logp, s.entropy, s.top_logp, s.top_index};
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    Tensor dz;
    if (grads[0].defined() || grads[1].defined()) {
      const variable_list saved = ctx->get_saved_variables();
      const Tensor &scores = saved[0], &targets = saved[1];
      const int64_t shots = ctx->saved_data["shots"].toInt();
      const int64_t cols = scores.size(-1);
      const Tensor sm = matrix(scores, cols, "scores");
      dz = at::empty(scores.sizes(), scores.options());
      const Tensor g =
          grads[0].defined() && shots ? signed_values(grads[0]).contiguous() : Tensor();
      const Tensor gh = grads[1].defined() ? signed_values(grads[1]).contiguous() : Tensor();
      const c10::DeviceGuard guard(scores.device());
      check(vqc_log_probs_backward(
          dtype_of(scores, "scores"), sm.size(0), cols, sm.data_ptr(), sm.stride(0),
          (float)ctx->saved_data["inv_t"].toDouble(),
          g.defined() ? pointer<int64_t>(targets) : nullptr, shots, pointer<float>(saved[2]),
          pointer<float>(saved[3]), pointer<float>(g), pointer<float>(gh), dz.data_ptr(), cols,
          stream_of(scores)));
    }
    // (scores that came this far want a gradient)
    return only_once({dz, Tensor(), Tensor(), Tensor()}, grads, 1, {1});
  }
};

std::tuple<Tensor, Tensor, Tensor, Tensor> log_probs(const Tensor& scores,
                                                     const Maybe& targets, int64_t top,
                                                     int64_t kind, double inv_t) {
  check_no_tangent({&scores});
  if (wants_grad({&scores})) {
    if (kind != VQC_SCORES_LOGITS)
      refuse("weights have no gradient here: detach them, or give logits");
    const variable_list out = LogProbs::apply(scores, targets, top, inv_t);
    return {out[0], out[1], out[2], out[3]};
  }
  Scores s = scores_forward(scores, given(targets), top, kind, inv_t, false);
  return {s.logp, s.entropy, s.top_logp, s.top_index};
}

// ------------------------------------------------------------------ 8-bit integers

// These calls have no gradient; nothing that wants one is let through.
void check_no_grad(const char* what, std::initializer_list<const Tensor*> xs) {
  check_no_tangent(xs);
  if (wants_grad(xs)) refuse(what, " has no gradient here: detach its inputs, or use no_grad");
}

// Rows of integers, [rows, width] each row's elements adjacent, with their steps.
Tensor integers(const Tensor& x, const Tensor& scales, int64_t width, const Tensor& like,
                const char* name) {
  if (x.scalar_type() != at::kChar || x.device() != like.device())
    refuse(name, " must be int8 on ", like.device(), ", got ", x.scalar_type(), " on ",
           x.device());
  if (x.dim() < 1 || scales.scalar_type() != at::kFloat || scales.device() != like.device() ||
      scales.sizes() != x.sizes().slice(0, x.dim() - 1))
    refuse("the scales of ", name, " must be float32 of its rows ",
           x.sizes().slice(0, x.dim() ? x.dim() - 1 : 0), " on ", like.device(), ", got ",
           scales.scalar_type(), " ", scales.sizes(), " on ", scales.device());
  return matrix(x, width, name);
}

// Rows start on 16 bytes, where the products read them fastest.
std::tuple<Tensor, Tensor> quantize(const Tensor& x) {
  const int code = dtype_of(x, "x");
  if (x.dim() < 1) refuse("x must have rows, got ", x.sizes());
  check_no_grad("quantize", {&x});
  const int64_t cols = x.size(-1), ld = (cols + 15) / 16 * 16;
  const Tensor xm = matrix(x, cols, "x");
  const int64_t rows = xm.size(0);
  const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
  Tensor q = at::empty({rows, ld}, x.options().dtype(at::kChar));
  Tensor scales = at::empty(lead, x.options().dtype(at::kFloat));
  {
    const c10::DeviceGuard guard(x.device());
    check(vqc_quantize(code, rows, cols, xm.data_ptr(), xm.stride(0), q.data_ptr<int8_t>(), ld,
                       scales.data_ptr<float>(), stream_of(x)));
  }
  std::vector<int64_t> strides(x.dim(), 1);
  int64_t step = ld;
  for (int64_t i = x.dim() - 2; i >= 0; --i) {
    strides[i] = step;
    step *= std::max<int64_t>(x.size(i), 1);
  }
  return {q.as_strided(x.sizes(), strides), scales};
}

Tensor linear_quantized(const Tensor& x, const Maybe& x_scales, const Tensor& weight,
                        const Tensor& weight_scales, const Maybe& bias, int64_t act,
                        const Maybe& residual, std::optional<at::ScalarType> dtype) {
  const Tensor xs = given(x_scales), b = given(bias), r = given(residual);
  check_no_grad("linear_quantized", {&x, &xs, &weight_scales, &b, &r});
  int code = VQC_F32;
  if (!xs.defined()) {
    code = dtype_of(x, "x");
    if (dtype && *dtype != x.scalar_type())
      refuse("the result of rows of ", x.scalar_type(), " is of their type, not ", *dtype);
  } else if (dtype) {
    switch (*dtype) {
      case at::kFloat: break;
      case at::kHalf: code = VQC_F16; break;
      case at::kBFloat16: code = VQC_BF16; break;
      default: refuse("dtype must be float32, float16 or bfloat16, got ", *dtype);
    }
  }
  if (!x.is_cuda()) refuse("x must be a cuda tensor");
  const at::TensorOptions like = x.options().dtype(code == VQC_F32   ? at::kFloat
                                                   : code == VQC_F16 ? at::kHalf
                                                                     : at::kBFloat16);
  const at::ScalarType type = c10::typeMetaToScalarType(like.dtype());
  if (weight.dim() != 2) refuse("weight must be [n_out, n_in], got ", weight.sizes());
  const int64_t n_out = weight.size(0), n_in = weight.size(1);
  const Tensor wm = integers(weight, weight_scales, n_in, x, "weight");
  const Tensor xm = xs.defined() ? integers(x, xs, n_in, x, "x") : matrix(x, n_in, "x");
  if (b.defined() && (b.scalar_type() != type || b.device() != x.device() || b.dim() != 1 ||
                      b.size(0) != n_out || !b.is_contiguous()))
    refuse("bias must be a contiguous ", type, " tensor of ", n_out, " elements on ", x.device());
  const int64_t rows = xm.size(0);
  const std::vector<int64_t> shape = with_last(x.sizes(), n_out);
  Tensor rm;
  if (r.defined()) {
    if (r.sizes() != at::IntArrayRef(shape) || r.scalar_type() != type ||
        r.device() != x.device())
      refuse("residual must be ", type, " of ", at::IntArrayRef(shape), " on ", x.device(),
             ", got ", r.scalar_type(), " ", r.sizes(), " on ", r.device());
    rm = matrix(r, n_out, "residual");
  }
  const Tensor bm = b.defined() ? signed_values(b) : b;
  const Tensor xf = xs.defined() ? signed_values(xs).contiguous() : xs;
  const Tensor wf = signed_values(weight_scales).contiguous();
  Tensor y = at::empty(shape, like);
  const size_t bytes = vqc_linear_quantized_workspace_bytes(rows, n_in, n_out, xs.defined());
  const Tensor ws = workspace(bytes, x);
  const c10::DeviceGuard guard(x.device());
  check(vqc_linear_quantized(code, rows, n_in, n_out, xm.data_ptr(), xm.stride(0),
                             pointer<float>(xf), wm.data_ptr<int8_t>(), wm.stride(0),
                             wf.data_ptr<float>(), pointer(bm), (int32_t)act, pointer(rm),
                             rm.defined() ? rm.stride(0) : 0, y.data_ptr(), n_out, pointer(ws),
                             bytes, stream_of(x)));
  return y;
}

// ------------------------------------------------------------------ drafts

std::tuple<Tensor, Tensor> verify_drafts(const Tensor& target, const Maybe& draft_scores,
                                         const Tensor& drafted, const Tensor& uniforms,
                                         int64_t kind, double inv_t) {
  const Tensor draft = given(draft_scores);
  const int code = dtype_of(target, "target");
  check_no_grad("verify_drafts", {&target, &draft, &uniforms});
  if (target.dim() < 2 || target.size(-1) < 1 || target.size(-2) < 1)
    refuse("target must have [drafts + 1, outcomes] for each sequence, got ", target.sizes());
  const int64_t cols = target.size(-1), drafts = target.size(-2) - 1;
  const at::IntArrayRef lead = target.sizes().slice(0, target.dim() - 2);
  std::vector<int64_t> shape(lead.begin(), lead.end());
  shape.push_back(drafts);
  if (drafted.scalar_type() != at::kLong || drafted.device() != target.device() ||
      drafted.sizes() != at::IntArrayRef(shape))
    refuse("drafted must be int64 of ", at::IntArrayRef(shape), " on ", target.device(), ", got ",
           drafted.scalar_type(), " ", drafted.sizes(), " on ", drafted.device());
  if (draft.defined()) {
    std::vector<int64_t> rows = shape;
    rows.push_back(cols);
    if (draft.sizes() != at::IntArrayRef(rows))
      refuse("draft must have shape ", at::IntArrayRef(rows), ", got ", draft.sizes());
    check_like(draft, target, "draft");
  }
  shape.back() = drafts + 1;
  if ((uniforms.scalar_type() != at::kFloat && uniforms.scalar_type() != at::kDouble) ||
      uniforms.device() != target.device() || uniforms.sizes() != at::IntArrayRef(shape))
    refuse("uniforms must be float32 or float64 of ", at::IntArrayRef(shape), " on ",
           target.device(), ", got ", uniforms.scalar_type(), " ", uniforms.sizes(), " on ",
           uniforms.device());
  const Tensor tm = matrix(target, cols, "target");
  const Tensor dm = draft.defined() ? matrix(draft, cols, "draft") : draft;
  const int64_t sequences = tm.size(0) / (drafts + 1);
  const Tensor d = drafted.contiguous();
  const Tensor u = signed_values(uniforms).to(at::kDouble).contiguous();
  Tensor outcomes = at::empty(shape, drafted.options());
  Tensor accepted = at::empty(lead, drafted.options());
  const bool has_draft = draft.defined() && drafts > 0;
  const size_t bytes =
      vqc_verify_drafts_workspace_bytes(code, sequences, drafts, cols, has_draft);
  const Tensor ws = workspace(bytes, target);
  const c10::DeviceGuard guard(target.device());
  check(vqc_verify_drafts((int32_t)kind, code, sequences, drafts, cols, tm.data_ptr(),
                          tm.stride(0), has_draft ? pointer(dm) : nullptr,
                          has_draft ? dm.stride(0) : 0, inv_t, pointer<int64_t>(d),
                          pointer<double>(u), pointer<int64_t>(outcomes),
                          pointer<int64_t>(accepted), pointer(ws), bytes, stream_of(target)));
  return {outcomes, accepted};
}

}  // namespace

PYBIND11_MODULE(vqc_torch, m) {
  py::register_exception_translator([](std::exception_ptr p) {
    try {
      if (p) std::rethrow_exception(p);
    } catch (const StatusError& e) {
      py::tuple args = py::make_tuple(e.code, e.what());
      PyErr_SetObject(g_error_type ? g_error_type : PyExc_RuntimeError, args.ptr());
    }
  });
  m.def("set_error_type", [](py::object t) { g_error_type = t.release().ptr(); });
  m.def("layer_norm", &layer_norm);
  m.def("linear", &linear);
  m.def("log_probs", &log_probs);
  m.def("quantize", &quantize);
  m.def("linear_quantized", &linear_quantized);
  m.def("verify_drafts", &verify_drafts);
}
