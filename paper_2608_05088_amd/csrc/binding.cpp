// The host side of the operators whose calls are short against Python's: argument checks,
// allocation and autograd of the AdamW step and the norm, in C++ (module _malt).
//
// AdamW over a hundred small tensors takes the card 6 us, and checking and listing them took
// Python 250; a norm's forward and backward pass take it 10 to 60, torch's Python functions 100; a layer on
// a token in 8 bits 3.5, and the call from Python 8.
//
// Every function runs on `stream` (a handle) and allocates with torch on the current stream, which
// its caller in ops.py makes the same.  Wrong arguments raise ValueError (TypeError for what is no tensor).
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <sstream>
#include <string>
#include <vector>

#include "../../include/libmalt.h"

namespace py = pybind11;
using at::Tensor;

namespace {

template <class... A>
std::string text(const A&... a) {
  std::ostringstream s;
  (s << ... << a);
  return s.str();
}
template <class... A>
[[noreturn]] void refuse(const A&... a) { throw py::value_error(text(a...)); }

// A tensor's name in messages: "x", or "params[3]".
struct Name {
  const char* list;
  int64_t at = -1;
};
std::ostream& operator<<(std::ostream& s, const Name& n) {
  s << n.list;
  if (n.at >= 0) s << '[' << n.at << ']';
  return s;
}

const char* type_name(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return "float32";
    case at::kBFloat16: return "bfloat16";
    case at::kHalf: return "float16";
    case at::kDouble: return "float64";
    case at::kByte: return "uint8";
    default: return c10::toString(t);
  }
}

int float_code(at::ScalarType t) { return t == at::kFloat ? MALT_FLOAT32 : t == at::kBFloat16 ? MALT_BFLOAT16 : -1; }

const Tensor& unpack(PyObject* o, const Name& name) {
  if (!THPVariable_Check(o)) throw py::type_error(text(name, " must be a tensor (got ", Py_TYPE(o)->tp_name, ")"));
  return THPVariable_Unpack(o);
}
void check_place(const Tensor& x, const Name& name, const c10::Device* device) {
  if (!x.is_cuda()) refuse(name, " must be on a GPU (got ", x.device(), ")");
  if (device && x.device() != *device) refuse(name, " is on ", x.device(), ", the other tensors on ", *device);
}
int check_float(const Tensor& x, const Name& name, const c10::Device* device) {
  const int code = float_code(x.scalar_type());
  if (code < 0) refuse(name, " must be float32 or bfloat16 (got ", type_name(x.scalar_type()), ")");
  check_place(x, name, device);
  return code;
}

// What the library refuses, or a failed launch: libmalt.py's MaltError in Python.
struct Refused : std::runtime_error {
  malt_status_t status;
  std::string message;
  explicit Refused(malt_status_t st) : std::runtime_error(text(malt_status_string(st), ": ", malt_last_error())), status(st), message(malt_last_error()) {}
};
void raise_status(malt_status_t st) {
  if (st != MALT_OK) throw Refused(st);
}
void translate(std::exception_ptr p) {
  try {
    if (p) std::rethrow_exception(p);
  } catch (const Refused& e) {
    const py::object cls = py::module_::import("paper_2608_05088_amd.libmalt").attr("MaltError");
    const py::object error = cls((int)e.status, e.message);
    PyErr_SetObject(cls.ptr(), error.ptr());
  }
}

// ------------------------------------------------------------------------ AdamW
// A Python sequence's items, borrowed.
struct Items {
  PyObject* fast;
  Py_ssize_t n;
  PyObject** at;
  explicit Items(py::handle o) {
    fast = PySequence_Fast(o.ptr(), "a sequence of tensors is wanted");
    if (!fast) throw py::error_already_set();
    n = PySequence_Fast_GET_SIZE(fast);
    at = PySequence_Fast_ITEMS(fast);
  }
  ~Items() { Py_DECREF(fast); }
  Items(const Items&) = delete;
};

// Moments of a parameter of `numel` elements: their bits.
uint8_t check_state(const Tensor& st, const Name& name, int64_t numel, const c10::Device& device) {
  const auto t = st.scalar_type();
  if (t != at::kFloat && t != at::kByte) refuse(name, " must be float32 or uint8 (got ", type_name(t), ")");
  check_place(st, name, &device);
  if (t == at::kFloat) {
    if (st.dim() != 2 || st.size(0) != 2 || st.size(1) != numel || !st.is_contiguous())
      refuse(name, " must be contiguous, (2, ", numel, ") (got ", st.sizes(), ", strides ", st.strides(), ")");
    return 32;
  }
  size_t bytes;
  raise_status(malt_adamw_state_size(numel, 8, &bytes));
  if (st.dim() != 1 || st.size(0) != (int64_t)bytes || !st.is_contiguous())
    refuse(name, " must be contiguous, (", bytes, ",) (got ", st.sizes(), ", strides ", st.strides(), ")");
  return 8;
}

void changed(const Tensor& x) {
  // Saved by a backward pass, it would be read with new values there.  (What was made in inference mode is never saved.)
  if (!x.is_inference()) x.unsafeGetTensorImpl()->bump_version();
}

void adamw_step(py::handle params, py::handle grads, py::handle states, double lr, double beta1, double beta2, double eps,
               double decay, int64_t step, double grad_scale, py::handle grad_scale_at, uint64_t seed, uintptr_t stream) {
  const Items p(params), g(grads), s(states);
  if (p.n != g.n || p.n != s.n) refuse("params, grads and states must be as many (got ", p.n, ", ", g.n, ", ", s.n, ")");
  const int64_t n = p.n;
  std::vector<int64_t> numel(n);
  std::vector<void*> pp(n), sp(n);
  std::vector<const void*> gp(n);
  std::vector<uint8_t> pt(n), gt(n), bits(n);
  std::vector<Tensor> copies;
  if (n == 0) return;
  const c10::Device device = unpack(p.at[0], {"params", 0}).device();
  for (int64_t i = 0; i < n; ++i) {
    const Tensor &x = unpack(p.at[i], {"params", i}), &d = unpack(g.at[i], {"grads", i}), &st = unpack(s.at[i], {"states", i});
    pt[i] = (uint8_t)check_float(x, {"params", i}, &device);
    gt[i] = (uint8_t)check_float(d, {"grads", i}, &device);
    if (!x.is_contiguous()) refuse(Name{"params", i}, " must be contiguous (got strides ", x.strides(), ")");
    if (d.sizes() != x.sizes()) refuse(Name{"grads", i}, " must be ", x.sizes(), " (got ", d.sizes(), ")");
    numel[i] = x.numel();
    bits[i] = check_state(st, {"states", i}, numel[i], device);
    pp[i] = x.data_ptr();
    sp[i] = st.data_ptr();
  }
  malt_adamw_t h = {lr, beta1, beta2, eps, decay, step, grad_scale, nullptr, seed};
  if (!grad_scale_at.is_none()) {
    const Tensor& c = unpack(grad_scale_at.ptr(), {"grad_scale"});
    if (c.scalar_type() != at::kFloat) refuse("grad_scale must be float32 (got ", type_name(c.scalar_type()), ")");
    check_place(c, {"grad_scale"}, &device);
    if (c.numel() != 1) refuse("grad_scale must be a number or a scalar tensor (got ", c.sizes(), ")");
    h.grad_scale_at = static_cast<const float*>(c.data_ptr());
  }
  for (int64_t i = 0; i < n; ++i) {   // copies are made when nothing can be refused here any more
    const Tensor& d = THPVariable_Unpack(g.at[i]);
    if (d.is_contiguous()) {
      gp[i] = d.data_ptr();
    } else {
      at::NoGradGuard no_grad;
      copies.push_back(d.contiguous());
      gp[i] = copies.back().data_ptr();
    }
  }
  const malt_adamw_tensors_t t = {(int32_t)n, numel.data(), pp.data(), pt.data(), gp.data(), gt.data(), sp.data(), bits.data()};
  raise_status(malt_adamw_step(&t, &h, reinterpret_cast<void*>(stream)));
  for (int64_t i = 0; i < n; ++i) {
    changed(THPVariable_Unpack(p.at[i]));
    changed(THPVariable_Unpack(s.at[i]));
  }
}

// float32 (2, numel) for each parameter.
std::vector<Tensor> adamw_moments(py::handle params, py::handle states, uintptr_t stream) {
  const Items p(params), s(states);
  if (p.n != s.n) refuse("params and states must be as many (got ", p.n, ", ", s.n, ")");
  std::vector<Tensor> out;
  std::vector<int64_t> numel;
  std::vector<const void*> sp;
  std::vector<float*> mp;
  if (p.n == 0) return out;
  const c10::Device device = unpack(p.at[0], {"params", 0}).device();
  std::vector<uint8_t> bits(p.n);
  for (int64_t i = 0; i < p.n; ++i) {
    const Tensor& x = unpack(p.at[i], {"params", i});
    check_float(x, {"params", i}, &device);
    bits[i] = check_state(unpack(s.at[i], {"states", i}), {"states", i}, x.numel(), device);
  }
  at::NoGradGuard no_grad;
  for (int64_t i = 0; i < p.n; ++i) {
    const Tensor& st = THPVariable_Unpack(s.at[i]);
    if (bits[i] == 32) {
      out.push_back(st.detach().clone());
      continue;
    }
    numel.push_back(THPVariable_Unpack(p.at[i]).numel());
    out.push_back(at::empty({2, numel.back()}, st.options().dtype(at::kFloat)));
    sp.push_back(st.data_ptr());
    mp.push_back(static_cast<float*>(out.back().data_ptr()));
  }
  raise_status(malt_adamw_moments((int32_t)numel.size(), numel.data(), sp.data(), mp.data(), reinterpret_cast<void*>(stream)));
  return out;
}

// ------------------------------------------------------------------------- norm
// A tensor's rows: contiguous ones as they lie, copied where they do not.
struct Rows {
  Tensor x;
  int64_t ld;
};
Rows rows_of(const Tensor& t, int64_t width) {
  Tensor x = t.dim() == 2 ? t : t.reshape({-1, width});
  const int64_t r = x.size(0), c = width;
  if ((c > 1 && x.stride(1) != 1) || (r > 1 && !(c <= x.stride(0) && x.stride(0) <= 0x7fffffff))) x = x.contiguous();
  return {x, r > 1 ? x.stride(0) : c};
}

struct NormCheck {
  int x, w;
  int64_t rows, width;
};
NormCheck check_norm(const Tensor& x, const Tensor& w, const Tensor& residual, double eps) {
  NormCheck c;
  c.x = check_float(x, {"x"}, nullptr);
  const c10::Device device = x.device();
  c.w = check_float(w, {"weight"}, &device);
  if (x.dim() < 1 || x.size(-1) < 1 || w.dim() != 1 || w.size(0) != x.size(-1))
    refuse("x must be (..., width) and weight (width,) (got ", x.sizes(), ", ", w.sizes(), ")");
  if (residual.defined()) {
    if (residual.scalar_type() != x.scalar_type())
      refuse("residual must be ", type_name(x.scalar_type()), " (got ", type_name(residual.scalar_type()), ")");
    check_place(residual, {"residual"}, &device);
    if (residual.sizes() != x.sizes()) refuse("residual must be ", x.sizes(), " (got ", residual.sizes(), ")");
  }
  if (!(eps >= 0 && eps < std::numeric_limits<double>::infinity())) refuse("eps must be a number, 0 or more (got ", eps, ")");
  c.width = x.size(-1);
  c.rows = x.numel() / c.width;
  return c;
}

struct NormOut {
  Tensor y, scales, sum, rstd;
};
// out: the type of y, or none for 8 bits.
NormOut norm(const Tensor& x, const Tensor& weight, const Tensor& residual, double eps, std::optional<at::ScalarType> out,
             bool want_rstd, void* stream) {
  const NormCheck c = check_norm(x, weight, residual, eps);
  const auto options = x.options().requires_grad(false);
  NormOut o;
  if (residual.defined()) o.sum = at::empty(x.sizes(), options);
  if (want_rstd) o.rstd = at::empty({c.rows}, options.dtype(at::kFloat));
  if (out) {
    o.y = at::empty(x.sizes(), options.dtype(*out));
  } else {
    const int64_t blocks = (c.width + 127) / 128;
    o.y = at::empty({c.rows, blocks * 128}, options.dtype(at::kFloat8_e4m3fn));
    o.scales = at::empty({blocks, (c.rows + 255) / 256 * 256}, options.dtype(at::kByte));
  }
  if (c.rows == 0) return o;
  const Rows xr = rows_of(x, c.width), rr = residual.defined() ? rows_of(residual, c.width) : Rows{Tensor(), 0};
  const Tensor w = weight.contiguous();
  malt_rms_norm_t a = {};
  a.x = xr.x.data_ptr();
  a.type = (malt_dtype_t)c.x;
  a.rows = c.rows;
  a.width = c.width;
  a.ldx = xr.ld;
  if (residual.defined()) {
    a.residual = rr.x.data_ptr();
    a.ldr = rr.ld;
    a.sum = o.sum.data_ptr();
    a.lds = c.width;
  }
  a.weight = w.data_ptr();
  a.weight_type = (malt_dtype_t)c.w;
  a.eps = eps;
  if (out) {
    a.y = o.y.data_ptr();
    a.y_type = (malt_dtype_t)float_code(*out);
    a.ldy = c.width;
  } else {
    a.values = o.y.data_ptr();
    a.scales = o.scales.data_ptr();
  }
  if (want_rstd) a.rstd = static_cast<float*>(o.rstd.data_ptr());
  raise_status(malt_rms_norm(&a, stream));
  return o;
}

void* current_stream(const Tensor& x) { return c10::hip::getCurrentHIPStream(x.device().index()).stream(); }

// In a captured backward pass: refuses to go on in a graph that was built on the default stream (leaves
// whose eager graph still lives have such nodes).  The engine would make that stream wait for the
// capture, which no capture survives, nor the process.
void check_captured_backward() {
  const auto node = torch::autograd::get_current_node();
  if (!node) return;
  const auto here = node->stream();
  if (!here) return;
  const hipStream_t stream = c10::hip::getCurrentHIPStream(here->device_index()).stream();
  if (!stream) return;   // the default stream is never captured, and must not be asked while another one is
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(stream, &status) != hipSuccess || status == hipStreamCaptureStatusNone) return;
  for (size_t i = 0; i < node->num_outputs(); ++i) {
    const auto& edge = node->next_edge(i);
    if (!edge.is_valid() || !node->task_should_compute_output(i)) continue;
    const auto there = edge.function->stream();
    if (there && there->id() == 0)
      throw std::runtime_error("a captured backward pass reaches a graph that was built on the default stream: drop what holds it "
                               "(outputs of eager calls on the same leaves), or make those calls on a stream of their own");
  }
}

struct RmsNorm : torch::autograd::Function<RmsNorm> {
  static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const Tensor& x, const Tensor& weight,
                                                const std::optional<Tensor>& residual_, double eps, int64_t out_type) {
    ctx->set_materialize_grads(false);
    const Tensor residual = residual_ ? *residual_ : Tensor();
    ctx->saved_data["residual"] = residual.defined();
    const NormOut o = norm(x, weight, residual, eps, (at::ScalarType)out_type, true, current_stream(x));
    ctx->save_for_backward({residual.defined() ? o.sum : x, weight, o.rstd});
    if (residual.defined()) return {o.y, o.sum};
    return {o.y};
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    torch::autograd::variable_list out(5);
    check_captured_backward();
    {
      at::NoGradGuard no_grad;
      const auto saved = ctx->get_saved_variables();
      const Tensor &h = saved[0], &weight = saved[1], &rstd = saved[2];
      const bool need_x = ctx->needs_input_grad(0), need_w = ctx->needs_input_grad(1);
      const bool need_r = ctx->saved_data["residual"].toBool() && ctx->needs_input_grad(2);
      Tensor dy = grads[0], dh = grads.size() > 1 ? grads[1] : Tensor();
      if (dh.defined() && dh.scalar_type() != h.scalar_type()) dh = dh.to(h.scalar_type());
      if (!dy.defined()) {   // nothing went through the norm
        if (need_x) out[0] = dh;
        if (need_r) out[2] = dh;
      } else {
        if (float_code(dy.scalar_type()) < 0) dy = dy.to(at::kFloat);
        const int64_t width = h.size(-1), rows = h.numel() / width;
        const bool need_h = need_x || need_r;
        const auto options = h.options().requires_grad(false);
        Tensor dx, dw;
        if (need_h) dx = at::empty(h.sizes(), options);
        if (need_w) dw = at::empty({width}, options.dtype(weight.scalar_type()));
        if (rows == 0) {
          if (need_w) dw.zero_();
        } else if (need_h || need_w) {
          const Rows hr = rows_of(h, width), gr = rows_of(dy, width), sr = dh.defined() && need_h ? rows_of(dh, width) : Rows{Tensor(), 0};
          const Tensor w = weight.contiguous();
          size_t bytes;
          raise_status(malt_rms_norm_grad_size(rows, width, need_w, &bytes));
          Tensor ws;
          if (bytes) ws = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
          malt_rms_norm_grad_t a = {};
          a.h = hr.x.data_ptr();
          a.type = (malt_dtype_t)float_code(h.scalar_type());
          a.rows = rows;
          a.width = width;
          a.ldh = hr.ld;
          a.weight = w.data_ptr();
          a.weight_type = (malt_dtype_t)float_code(w.scalar_type());
          a.rstd = static_cast<const float*>(rstd.data_ptr());
          a.dy = gr.x.data_ptr();
          a.dy_type = (malt_dtype_t)float_code(gr.x.scalar_type());
          a.lddy = gr.ld;
          if (sr.x.defined()) {
            a.dsum = sr.x.data_ptr();
            a.ldds = sr.ld;
          }
          if (need_h) {
            a.dx = dx.data_ptr();
            a.lddx = width;
          }
          if (need_w) a.dweight = dw.data_ptr();
          raise_status(malt_rms_norm_grad(&a, bytes ? ws.data_ptr() : nullptr, bytes, current_stream(h)));
        }
        if (need_x) out[0] = dx;
        out[1] = dw;
        if (need_r) out[2] = dx;
      }
    }
    // Once only: gradients of these gradients would be missing without a word.
    bool again = false;
    if (at::GradMode::is_enabled())
      for (const Tensor& g : grads) again |= g.defined() && g.requires_grad();
    if (again) {
      auto error = std::make_shared<torch::autograd::DelayedError>(
          "trying to differentiate twice a function that was marked with @once_differentiable", 1);
      for (Tensor& t : out)
        if (t.defined()) t = (*error)({t.detach().set_requires_grad(true)})[0];
    }
    return out;
  }
};

Tensor optional_tensor(py::handle o, const char* name) { return o.is_none() ? Tensor() : unpack(o.ptr(), {name}); }

// y, and the sum where there is a residual.  Differentiable where `grad` says so (on the current stream then).
py::object rms_norm(py::handle x_, py::handle weight_, py::handle residual_, double eps, py::handle out_type, bool grad, uintptr_t stream) {
  const Tensor &x = unpack(x_.ptr(), {"x"}), &weight = unpack(weight_.ptr(), {"weight"});
  const Tensor residual = optional_tensor(residual_, "residual");
  at::ScalarType type = x.scalar_type();
  if (!out_type.is_none()) type = py::cast<at::ScalarType>(out_type);
  if (grad) {
    check_norm(x, weight, residual, eps);
    const auto out = RmsNorm::apply(x, weight, residual.defined() ? std::optional<Tensor>(residual) : std::nullopt, eps, (int64_t)type);
    return out.size() > 1 ? py::object(py::make_tuple(out[0], out[1])) : py::cast(out[0]);
  }
  at::NoGradGuard no_grad;
  const NormOut o = norm(x, weight, residual, eps, type, false, reinterpret_cast<void*>(stream));
  return residual.defined() ? py::object(py::make_tuple(o.y, o.sum)) : py::cast(o.y);
}

// Values, scales and the sum (or None).
py::tuple rms_norm_fp8(py::handle x, py::handle weight, py::handle residual_, double eps, uintptr_t stream) {
  const Tensor residual = optional_tensor(residual_, "residual");
  at::NoGradGuard no_grad;
  const NormOut o = norm(unpack(x.ptr(), {"x"}), unpack(weight.ptr(), {"weight"}), residual, eps, std::nullopt, false,
                         reinterpret_cast<void*>(stream));
  return py::make_tuple(o.y, o.scales, residual.defined() ? py::cast(o.sum) : py::object(py::none()));
}

// ------------------------------------------------- a layer on activations in 8 bits
const Tensor* operand(py::handle o, at::ScalarType type, const c10::Device& device) {
  if (!THPVariable_Check(o.ptr())) return nullptr;
  const Tensor& t = THPVariable_Unpack(o.ptr());
  return t.scalar_type() == type && t.device() == device && t.dim() == 2 && t.is_contiguous() ? &t : nullptr;
}

// None where an argument is not what it has to be: ops.py then says which.  (In Python the checks and the
// allocation took as long as the launch.)
py::object fp8_rows(py::handle x_values, py::handle x_scales, py::handle shape, py::handle values, py::handle scales, int out_type,
                    uintptr_t stream) {
  if (!THPVariable_Check(values.ptr()) || !PyTuple_Check(shape.ptr())) return py::none();
  const c10::Device device = THPVariable_Unpack(values.ptr()).device();
  const Tensor *xv = operand(x_values, at::kFloat8_e4m3fn, device), *xs = operand(x_scales, at::kByte, device),
               *wv = operand(values, at::kFloat8_e4m3fn, device), *ws = operand(scales, at::kByte, device);
  const Py_ssize_t dims = PyTuple_GET_SIZE(shape.ptr());
  if (!device.is_cuda() || !xv || !xs || !wv || !ws || dims < 1) return py::none();
  c10::SmallVector<int64_t, 4> out;
  for (Py_ssize_t i = 0; i < dims; ++i) {
    const int64_t n = PyLong_AsLongLong(PyTuple_GET_ITEM(shape.ptr(), i));
    if (n < 0) {
      PyErr_Clear();
      return py::none();
    }
    out.push_back(n);
  }
  const int64_t k = out.back(), kb = (k + 127) / 128, m = xv->size(0), n = wv->size(0);
  out.back() = n;
  int64_t rows = 1;
  for (Py_ssize_t i = 0; i + 1 < dims; ++i)
    if (__builtin_mul_overflow(rows, out[i], &rows)) return py::none();
  if (k < 1 || n < 1 || rows != m || xv->size(1) != kb * 128 || wv->size(1) != kb * 128 || xs->size(0) != kb ||
      xs->size(1) != (m + 255) / 256 * 256 || ws->size(0) != (n + 127) / 128 || ws->size(1) != kb)
    return py::none();
  at::NoGradGuard no_grad;
  const Tensor y = at::empty(out, xv->options().dtype(out_type == MALT_FLOAT32 ? at::kFloat : at::kBFloat16).requires_grad(false));
  if (m == 0) return py::cast(y);
  size_t bytes = 0;
  if (m > 32) raise_status(malt_block_matmul_size(m, n, k, (malt_dtype_t)out_type, &bytes));
  Tensor workspace;
  if (bytes) workspace = at::empty({(int64_t)bytes}, xs->options());
  raise_status(malt_block_linear_operand(xv->data_ptr(), xs->data_ptr(), m, k, wv->data_ptr(), ws->data_ptr(), n, y.data_ptr(),
                                         (malt_dtype_t)out_type, n, bytes ? workspace.data_ptr() : nullptr, bytes,
                                         reinterpret_cast<void*>(stream)));
  return py::cast(y);
}

}  // namespace

PYBIND11_MODULE(_malt, m) {
  py::register_exception_translator(&translate);
  m.def("adamw_step", &adamw_step);
  m.def("adamw_moments", &adamw_moments);
  m.def("rms_norm", &rms_norm);
  m.def("rms_norm_fp8", &rms_norm_fp8);
  m.def("fp8_rows", &fp8_rows);
  m.def("check_captured_backward", &check_captured_backward);
}
