// PyTorch binding of the sequence-model operators (include/rc_ops.h): checks
// of arguments, outputs and scratch from PyTorch's allocator, the current
// stream, and autograd.  Native, because a single token's kernels take a few
// microseconds and the same work in Python took several times that.
// ops.py documents the functions.
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/extension.h>

#include "rc_ops.h"

namespace py = pybind11;
using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;
using Opt = std::optional<Tensor>;

namespace {

constexpr int64_t kMaxTaps = 8, kMaxStates = 64, kMaxNormWidth = 16384, kMaxHead = 256;

// A library error as rcdp.RcError.
[[noreturn]] void fail(int status, const char* where) {
  py::gil_scoped_acquire gil;
  const py::object type = py::module_::import("paper_1905_11722_amd.rcdp").attr("RcError");
  PyErr_SetObject(type.ptr(), type(status, where).ptr());
  throw py::error_already_set();
}
void check(int status, const char* where) {
  if (status) fail(status, where);
}

// Absent tensors are undefined ones here, and empty optionals where autograd looks.
Tensor given(const Opt& t) { return t.has_value() ? *t : Tensor(); }
Opt opt(const Tensor& t) { return t.defined() ? Opt(t) : Opt(); }

int32_t code(at::ScalarType t) {
  return t == at::kFloat ? RC_F32 : t == at::kBFloat16 ? RC_BF16 : RC_F16;
}

void activations(const char* name, const Tensor& t) {
  TORCH_CHECK_VALUE(t.is_cuda(), name, " must be on a GPU: there is no CPU path");
  TORCH_CHECK_VALUE(t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16 ||
                        t.scalar_type() == at::kHalf,
                    name, " must be float32, bfloat16 or float16, not ", t.scalar_type());
}
// The tensor that gives sizes, type and device.
void main_tensor(const char* name, const Tensor& t, int64_t dims) {
  activations(name, t);
  TORCH_CHECK_VALUE(t.dim() == dims, name, " must have ", dims, " dimensions, not ", t.dim());
  for (const int64_t n : t.sizes()) TORCH_CHECK_VALUE(n < (int64_t)1 << 31, name, " is too large");
}

void expect(const char* name, const Tensor& t, at::IntArrayRef shape, at::ScalarType type,
            const Tensor& main) {
  TORCH_CHECK_VALUE(t.sizes() == shape, name, " must have shape ", shape, ", not ", t.sizes());
  TORCH_CHECK_VALUE(t.scalar_type() == type, name, " must be ", type, ", not ", t.scalar_type());
  TORCH_CHECK_VALUE(t.device() == main.device(), name, " must be on ", main.device(), ", not on ",
                    t.device());
}

// t with contiguous channels and its values in memory (not those of a view that negates them):
// itself, or a copy.
Tensor plain(const Tensor& t) { return t.is_neg() ? t.resolve_neg() : t; }
Tensor rows(const Tensor& t) {
  if (!t.defined()) return t;
  return plain(t.size(-1) <= 1 || t.stride(-1) == 1 ? t : t.contiguous());
}
Tensor dense(const Tensor& t) {
  if (!t.defined()) return t;
  return plain(t.is_contiguous() ? t : t.contiguous());
}

// A (batch, time, channel) or (batch, channel) tensor.
rc_view view(const Tensor& t) {
  if (!t.defined()) return {nullptr, 0, 0};
  return {t.data_ptr(), t.stride(0), t.dim() > 2 ? t.stride(1) : 0};
}
template <class P = void>
P* ptr(const Tensor& t) {
  return t.defined() ? static_cast<P*>(t.data_ptr()) : nullptr;
}

// Parameters of one type: float32 or the activations'.
int32_t param_type(std::initializer_list<std::pair<const char*, const Tensor*>> params,
                   const Tensor& main) {
  at::ScalarType type = at::kFloat;
  for (const auto& p : params)
    if (p.second->defined()) {
      type = p.second->scalar_type();
      TORCH_CHECK_VALUE(type == at::kFloat || type == main.scalar_type(), p.first,
                        " must be float32 or ", main.scalar_type(), ", not ", type);
      break;
    }
  for (const auto& p : params)
    if (p.second->defined())
      TORCH_CHECK_VALUE(p.second->scalar_type() == type, p.first, " must be ", type, ", not ",
                        p.second->scalar_type());
  return code(type);
}

Tensor lengths_of(const Opt& t, const Tensor& main) {
  if (!t) return Tensor();
  expect("lengths", *t, {main.size(0)}, at::kInt, main);
  return dense(*t);
}
Tensor slots_of(const Opt& t, const Tensor& main, const Tensor& state) {
  const int64_t slots = state.size(0);
  TORCH_CHECK_VALUE(!state.is_neg(), "state must not be a view that negates its memory");
  TORCH_CHECK_VALUE(slots < (int64_t)1 << 31, "state has too many slots: ", slots);
  if (t) {
    expect("slots", *t, {main.size(0)}, at::kInt, main);
    return dense(*t);
  }
  TORCH_CHECK_VALUE(slots >= main.size(0), "state has ", slots, " slots for ", main.size(0), " rows");
  return Tensor();
}

// Whether some of `rows` rows of `width` elements at i * slot + k * row, i < slots, share memory.
bool overlap(int64_t slots, int64_t slot, int64_t rows, int64_t row, int64_t width) {
  if (slots == 0 || rows == 0 || width == 0) return false;
  if (slots > 1 && slot < width) return true;
  for (int64_t k = 1; k < rows; k++) {                 // rows k apart: the slots that come closest
    const int64_t last = slots - 1, i = slot ? std::min(k * row / slot, last) : 0;
    for (const int64_t j : {i, std::min(i + 1, last)})
      if (std::abs(k * row - j * slot) < width) return true;
  }
  return false;
}

template <class Args>
Tensor scratch(int (*size)(const Args*, uint64_t*), Args& args, const Tensor& main,
               const char* name) {
  uint64_t n = 0;
  check(size(&args, &n), name);
  if (n == 0) return Tensor();
  Tensor t = at::empty({(int64_t)n}, main.options().dtype(at::kByte));
  args.workspace = t.data_ptr();
  args.workspace_bytes = n;
  return t;
}

void* stream_of(const Tensor& t) {
  return c10::hip::getCurrentHIPStream(t.device().index()).stream();
}

// Forward mode does not ask requires_grad: a tangent that is not refused would be dropped.
void no_tangent(const Tensor& t) {
  if (t.defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode())
    TORCH_CHECK_NOT_IMPLEMENTED(!t._fw_grad(0).defined(),
                                "the sequence-model operators have no forward-mode derivatives");
}

// Whether autograd records this call.
bool differentiated(std::initializer_list<const Tensor*> tensors) {
  for (const Tensor* t : tensors) no_tangent(*t);
  if (!at::GradMode::is_enabled()) return false;
  for (const Tensor* t : tensors)
    if (t->defined() && t->requires_grad()) return true;
  return false;
}

// The token forms have no gradients: where one is asked for they raise, rather than
// cut what they return from its past.
void not_differentiated(const char* name, std::initializer_list<const Tensor*> tensors) {
  TORCH_CHECK_VALUE(!differentiated(tensors), name,
                    " has no gradients: call it under torch.no_grad(), or with detached tensors");
}

// A tensor that a kernel has written through its pointer: what autograd has
// saved of it is out of date, as after torch's own operators in place.
void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// Gradients that must not be differentiated again say so if they are.
variable_list once(variable_list grads) {
  if (!at::GradMode::is_enabled()) return grads;
  variable_list list;
  for (const Tensor& g : grads)
    if (g.defined()) list.push_back(g.detach().set_requires_grad(true));
  const auto error = std::make_shared<torch::autograd::DelayedError>(
      "the sequence-model operators can be differentiated once only", (int64_t)list.size());
  list = (*error)(std::move(list));
  size_t i = 0;
  for (Tensor& g : grads)
    if (g.defined()) g = list[i++];
  return grads;
}

Tensor like(const Tensor& t, bool want = true) {
  return t.defined() && want ? at::empty(t.sizes(), t.options()) : Tensor();
}

// ---------------------------------------------------------------- convolution

rc_conv_args conv_args(const Tensor& x, const Tensor& w, const Tensor& b, const Tensor& state,
                       const Tensor& lengths, int64_t act, int64_t param) {
  rc_conv_args a = {};
  a.dtype = code(x.scalar_type());
  a.param_dtype = (int32_t)param;
  a.activation = (int32_t)act;
  a.batch = (int32_t)x.size(0);
  a.length = (int32_t)x.size(1);
  a.width = (int32_t)x.size(2);
  a.taps = (int32_t)w.size(1);
  a.x = view(x);
  a.state_in = view(state);
  a.weight = ptr(w);
  a.bias = ptr(b);
  a.lengths = ptr<int32_t>(lengths);
  return a;
}

variable_list conv_forward(const Tensor& x, const Tensor& w, const Tensor& b, const Tensor& state,
                           const Tensor& lengths, int64_t act, int64_t param, bool want_state) {
  const c10::DeviceGuard guard(x.device());
  rc_conv_args a = conv_args(x, w, b, state, lengths, act, param);
  variable_list out = {like(x)};
  a.y = view(out[0]);
  if (want_state) {
    out.push_back(at::empty({x.size(0), w.size(1) - 1, x.size(2)}, x.options()));
    a.state_out = view(out[1]);
  }
  check(rc_conv_forward(&a, stream_of(x)), "rc_conv_forward");
  return out;
}

struct Conv : torch::autograd::Function<Conv> {
  static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& w,
                               const Opt& bias, const Opt& state_in, const Opt& ends, int64_t act,
                               int64_t param, bool want_state) {
    const Tensor b = given(bias), state = given(state_in), lengths = given(ends);
    ctx->save_for_backward({x, w, b, state, lengths});
    ctx->saved_data["act"] = act;
    ctx->saved_data["param"] = param;
    ctx->set_materialize_grads(false);
    return conv_forward(x, w, b, state, lengths, act, param, want_state);
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    for (const Tensor& g : grads) no_tangent(g);
    const auto saved = ctx->get_saved_variables();
    const Tensor &x = saved[0], &w = saved[1], &b = saved[2], &state = saved[3];
    const c10::DeviceGuard guard(x.device());
    rc_conv_args a = conv_args(x, w, b, state, saved[4], ctx->saved_data["act"].toInt(),
                               ctx->saved_data["param"].toInt());
    const Tensor dy = grads[0].defined() ? rows(grads[0]) : at::zeros_like(x);
    const Tensor dout = grads.size() > 1 ? rows(grads[1]) : Tensor();
    const Tensor dx = like(x), dw = like(w, w.requires_grad()),
                 db = like(b, b.defined() && b.requires_grad()),
                 ds = like(state, state.defined() && state.requires_grad());
    a.dy = view(dy);
    a.dstate_out = view(dout);
    a.dx = view(dx);
    a.dstate_in = view(ds);
    a.dweight = ptr(dw);
    a.dbias = ptr(db);
    const Tensor work = dw.defined() || db.defined()
                            ? scratch(rc_conv_backward_workspace, a, x, "rc_conv_backward_workspace")
                            : Tensor();
    check(rc_conv_backward(&a, stream_of(x)), "rc_conv_backward");
    return once({dx, dw, db, ds, Tensor(), Tensor(), Tensor(), Tensor()});
  }
};

int64_t taps_of(const Tensor& w, const Tensor& x) {
  TORCH_CHECK_VALUE(w.dim() == 2, "weight must be a (width, taps) tensor");
  const int64_t k = w.size(1);
  TORCH_CHECK_VALUE(k >= 1 && k <= kMaxTaps, "weight must have 1 to ", kMaxTaps, " taps, not ", k);
  expect("weight", w, {x.size(-1), k}, w.scalar_type(), x);
  return k;
}

variable_list causal_conv(const Tensor& x, const Tensor& weight, const Opt& bias_, const Opt& state_,
                          const Opt& lengths_, int64_t act, bool want_state) {
  main_tensor("x", x, 3);
  const Tensor bias = given(bias_), state = given(state_);
  const int64_t k = taps_of(weight, x);
  if (bias.defined()) expect("bias", bias, {x.size(2)}, bias.scalar_type(), x);
  const int32_t param = param_type({{"weight", &weight}, {"bias", &bias}}, x);
  if (state.defined())
    expect("state", state, {x.size(0), k - 1, x.size(2)}, x.scalar_type(), x);
  const Tensor lengths = lengths_of(lengths_, x);
  if (differentiated({&x, &weight, &bias, &state}))
    return Conv::apply(rows(x), dense(weight), opt(dense(bias)), opt(rows(state)), opt(lengths),
                       act, (int64_t)param, want_state);
  return conv_forward(rows(x), dense(weight), dense(bias), rows(state), lengths, act, param,
                      want_state);
}

Tensor causal_conv_step(const Tensor& state, const Tensor& x_, const Tensor& weight_,
                        const Opt& bias_, const Opt& slots_, int64_t act) {
  main_tensor("x", x_, 2);
  const int64_t k = taps_of(weight_, x_), d = x_.size(1);
  const Tensor weight = dense(weight_), bias = dense(given(bias_)), x = rows(x_);
  if (bias.defined()) expect("bias", bias, {d}, bias.scalar_type(), x);
  rc_conv_step_args a = {};
  a.param_dtype = param_type({{"weight", &weight}, {"bias", &bias}}, x);
  TORCH_CHECK_VALUE(state.dim() == 3, "state must have 3 dimensions");
  expect("state", state, {state.size(0), k - 1, d}, x.scalar_type(), x);
  TORCH_CHECK_VALUE(state.stride(2) == 1 || d <= 1, "state must have contiguous channels");
  TORCH_CHECK_VALUE(!overlap(state.size(0), state.stride(0), k - 1, state.stride(1), d),
                    "states must not share memory");
  const Tensor slots = slots_of(slots_, x, state);
  not_differentiated("causal_conv_step", {&state, &x, &weight, &bias});
  const c10::DeviceGuard guard(x.device());
  const Tensor y = at::empty({x.size(0), d}, x.options());
  a.dtype = code(x.scalar_type());
  a.activation = (int32_t)act;
  a.batch = (int32_t)x.size(0);
  a.width = (int32_t)d;
  a.taps = (int32_t)k;
  a.num_slots = (int32_t)state.size(0);
  a.x = view(x);
  a.y = view(y);
  a.state = view(state);
  a.weight = ptr(weight);
  a.bias = ptr(bias);
  a.slots = ptr<int32_t>(slots);
  check(rc_conv_step(&a, stream_of(x)), "rc_conv_step");
  written(state);
  return y;
}

// ----------------------------------------------------------------------- scan

struct ScanIn {
  Tensor u, dt, A, B, C, D, z, dt_bias, state, lengths;
};

rc_scan_args scan_args(const ScanIn& t, int64_t softplus) {
  rc_scan_args a = {};
  a.dtype = code(t.u.scalar_type());
  a.softplus = (int32_t)softplus;
  a.batch = (int32_t)t.u.size(0);
  a.length = (int32_t)t.u.size(1);
  a.width = (int32_t)t.u.size(2);
  a.states = (int32_t)t.A.size(1);
  a.groups = t.B.dim() == 4 ? (int32_t)t.B.size(2) : 1;
  a.u = view(t.u);
  a.dt = view(t.dt);
  a.z = view(t.z);
  a.B = view(t.B);
  a.C = view(t.C);
  a.B_group = t.B.dim() == 4 ? t.B.stride(2) : 0;
  a.C_group = t.C.dim() == 4 ? t.C.stride(2) : 0;
  a.A = ptr<float>(t.A);
  a.D = ptr<float>(t.D);
  a.dt_bias = ptr<float>(t.dt_bias);
  a.state_in = ptr<float>(t.state);
  a.lengths = ptr<int32_t>(t.lengths);
  return a;
}

// y, and the final state if wanted; the kept states into *kept if that is not null.
variable_list scan_forward(const ScanIn& t, int64_t softplus, bool want_state, Tensor* kept) {
  const c10::DeviceGuard guard(t.u.device());
  rc_scan_args a = scan_args(t, softplus);
  variable_list out = {like(t.u)};
  a.y = view(out[0]);
  if (want_state) {
    out.push_back(at::empty({t.u.size(0), t.A.size(0), t.A.size(1)}, t.A.options()));
    a.state_out = ptr<float>(out[1]);
  }
  if (kept) {
    uint64_t n = 0;
    check(rc_scan_kept_bytes(&a, &n), "rc_scan_kept_bytes");
    *kept = at::empty({(int64_t)n / 4}, t.A.options());
    a.kept = ptr<float>(*kept);
  }
  const Tensor work = scratch(rc_scan_forward_workspace, a, t.u, "rc_scan_forward_workspace");
  check(rc_scan_forward(&a, stream_of(t.u)), "rc_scan_forward");
  return out;
}

struct Scan : torch::autograd::Function<Scan> {
  static variable_list forward(AutogradContext* ctx, const Tensor& u, const Tensor& dt,
                               const Tensor& A, const Tensor& B, const Tensor& C, const Opt& skip,
                               const Opt& gate, const Opt& bias, const Opt& state_in,
                               const Opt& ends, int64_t softplus, bool want_state) {
    const Tensor D = given(skip), z = given(gate), dt_bias = given(bias), state = given(state_in),
                 lengths = given(ends);
    Tensor kept;
    variable_list out = scan_forward({u, dt, A, B, C, D, z, dt_bias, state, lengths}, softplus,
                                     want_state, &kept);
    ctx->save_for_backward({u, dt, A, B, C, D, z, dt_bias, state, lengths, kept});
    ctx->saved_data["softplus"] = softplus;
    ctx->set_materialize_grads(false);
    return out;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    for (const Tensor& g : grads) no_tangent(g);
    const auto s = ctx->get_saved_variables();
    const ScanIn t = {s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7], s[8], s[9]};
    const c10::DeviceGuard guard(t.u.device());
    rc_scan_args a = scan_args(t, ctx->saved_data["softplus"].toInt());
    const Tensor dy = grads[0].defined() ? rows(grads[0]) : at::zeros_like(t.u);
    const Tensor dout = grads.size() > 1 ? dense(grads[1]) : Tensor();
    const Tensor du = like(t.u), ddt = like(t.dt), dA = like(t.A), dD = like(t.D), dz = like(t.z),
                 dbias = like(t.dt_bias),
                 ds = like(t.state, t.state.defined() && t.state.requires_grad());
    const Tensor dB = at::empty(t.B.sizes(), t.B.options()), dC = at::empty(t.C.sizes(), t.C.options());
    a.kept = ptr<float>(s[10]);
    a.dy = view(dy);
    a.du = view(du);
    a.ddt = view(ddt);
    a.dz = view(dz);
    a.dB = ptr(dB);
    a.dC = ptr(dC);
    a.dstate_out = ptr<float>(dout);
    a.dA = ptr<float>(dA);
    a.dD = ptr<float>(dD);
    a.ddt_bias = ptr<float>(dbias);
    a.dstate_in = ptr<float>(ds);
    const Tensor work = scratch(rc_scan_backward_workspace, a, t.u, "rc_scan_backward_workspace");
    check(rc_scan_backward(&a, stream_of(t.u)), "rc_scan_backward");
    return once({du, ddt, dA, dB, dC, dD, dz, dbias, ds, Tensor(), Tensor(), Tensor()});
  }
};

// Checks of what scan and step share; tokens: (batch, length) or (batch).
void scan_expect(const ScanIn& t, at::IntArrayRef tokens) {
  const Tensor& u = t.u;
  const int64_t d = u.size(-1);
  TORCH_CHECK_VALUE(t.A.dim() == 2, "A must be a (width, states) tensor");
  const int64_t n = t.A.size(1);
  TORCH_CHECK_VALUE(n >= 1 && n <= kMaxStates, "A must have 1 to ", kMaxStates, " states, not ", n);
  expect("A", t.A, {d, n}, at::kFloat, u);
  const int64_t dims = (int64_t)tokens.size();
  TORCH_CHECK_VALUE(t.B.dim() == dims + 1 || t.B.dim() == dims + 2, "B must have ", dims + 1, " or ",
                    dims + 2, " dimensions, not ", t.B.dim());
  TORCH_CHECK_VALUE(t.C.dim() == t.B.dim(), "C must have ", t.B.dim(), " dimensions, not ", t.C.dim());
  std::vector<int64_t> shape(tokens.begin(), tokens.end());
  if (t.B.dim() == dims + 2) {
    const int64_t g = t.B.size(dims);
    TORCH_CHECK_VALUE(g >= 1 && d % g == 0, g, " groups of B do not divide ", d, " channels");
    shape.push_back(g);
  }
  shape.push_back(n);
  expect("B", t.B, shape, u.scalar_type(), u);
  expect("C", t.C, shape, u.scalar_type(), u);
  expect("dt", t.dt, u.sizes(), u.scalar_type(), u);
  if (t.z.defined()) expect("z", t.z, u.sizes(), u.scalar_type(), u);
  if (t.D.defined()) expect("D", t.D, {d}, at::kFloat, u);
  if (t.dt_bias.defined()) expect("dt_bias", t.dt_bias, {d}, at::kFloat, u);
}

variable_list selective_scan(const Tensor& u, const Tensor& dt, const Tensor& A, const Tensor& B,
                             const Tensor& C, const Opt& D, const Opt& z, const Opt& dt_bias,
                             bool softplus, const Opt& state, const Opt& lengths, bool want_state) {
  main_tensor("u", u, 3);
  ScanIn t = {u, dt, A, B, C, given(D), given(z), given(dt_bias), given(state), Tensor()};
  scan_expect(t, {u.size(0), u.size(1)});
  if (state) expect("state", *state, {u.size(0), u.size(2), A.size(1)}, at::kFloat, u);
  t.lengths = lengths_of(lengths, u);
  const bool grad = differentiated({&u, &dt, &A, &B, &C, &t.D, &t.z, &t.dt_bias, &t.state});
  t = {rows(u), rows(dt), dense(A), rows(B), rows(C), dense(t.D), rows(t.z), dense(t.dt_bias),
       dense(t.state), t.lengths};
  if (grad)
    return Scan::apply(t.u, t.dt, t.A, t.B, t.C, opt(t.D), opt(t.z), opt(t.dt_bias), opt(t.state),
                       opt(t.lengths), (int64_t)softplus, want_state);
  return scan_forward(t, softplus, want_state, nullptr);
}

Tensor selective_scan_step(const Tensor& state, const Tensor& u, const Tensor& dt, const Tensor& A,
                           const Tensor& B, const Tensor& C, const Opt& D, const Opt& z,
                           const Opt& dt_bias, bool softplus, const Opt& slots_) {
  main_tensor("u", u, 2);
  ScanIn t = {u, dt, A, B, C, given(D), given(z), given(dt_bias), Tensor(), Tensor()};
  scan_expect(t, {u.size(0)});
  const int64_t d = u.size(1), n = A.size(1);
  TORCH_CHECK_VALUE(state.dim() == 3, "state must have 3 dimensions");
  expect("state", state, {state.size(0), d, n}, at::kFloat, u);
  TORCH_CHECK_VALUE((state.stride(2) == 1 || n <= 1) && (state.stride(1) == n || d <= 1),
                    "each slot of state must be contiguous");
  TORCH_CHECK_VALUE(!overlap(state.size(0), state.stride(0), 1, 0, d * n),
                    "states must not share memory");
  const Tensor slots = slots_of(slots_, u, state);
  not_differentiated("selective_scan_step",
                     {&state, &u, &dt, &A, &B, &C, &t.D, &t.z, &t.dt_bias});
  t = {rows(u), rows(dt), dense(A), rows(B), rows(C), dense(t.D), rows(t.z), dense(t.dt_bias),
       Tensor(), Tensor()};
  const c10::DeviceGuard guard(u.device());
  const Tensor y = at::empty({u.size(0), d}, u.options());
  rc_scan_step_args a = {};
  a.dtype = code(u.scalar_type());
  a.softplus = softplus;
  a.batch = (int32_t)u.size(0);
  a.width = (int32_t)d;
  a.states = (int32_t)n;
  a.groups = t.B.dim() == 3 ? (int32_t)t.B.size(1) : 1;
  a.num_slots = (int32_t)state.size(0);
  a.u = view(t.u);
  a.dt = view(t.dt);
  a.z = view(t.z);
  a.B = view(t.B);
  a.C = view(t.C);
  a.y = view(y);
  a.B_group = t.B.dim() == 3 ? t.B.stride(1) : 0;
  a.C_group = t.C.dim() == 3 ? t.C.stride(1) : 0;
  a.A = ptr<float>(t.A);
  a.D = ptr<float>(t.D);
  a.dt_bias = ptr<float>(t.dt_bias);
  a.state = ptr<float>(state);
  a.state_slot = state.stride(0);
  a.slots = ptr<int32_t>(slots);
  check(rc_scan_step(&a, stream_of(u)), "rc_scan_step");
  written(state);
  return y;
}

// ---------------------------------------------------------------------- norms

// (..., width) as rows with contiguous channels: a view where strides allow it.
Tensor flat(const Tensor& t, int64_t n) {
  if (!t.defined()) return t;
  return rows(t.dim() == 2 ? t : t.reshape({n, t.size(-1)}));
}
// A contiguous tensor of any number of dimensions as rows.
rc_view row_view(const Tensor& t) {
  return t.defined() ? rc_view{t.data_ptr(), t.size(-1), 0} : rc_view{nullptr, 0, 0};
}

struct NormIn {
  Tensor block, residual, gate, post, scale, pre;
};

rc_norm_args norm_args(const NormIn& t, int64_t act, int64_t param, double eps, Tensor* keep) {
  const int64_t d = t.residual.size(-1), n = d ? t.residual.numel() / d : 0;
  keep[0] = flat(t.block, n);
  keep[1] = flat(t.residual, n);
  keep[2] = flat(t.gate, n);
  rc_norm_args a = {};
  a.dtype = code((t.block.defined() ? t.block : t.residual).scalar_type());
  a.residual_dtype = code(t.residual.scalar_type());
  a.param_dtype = (int32_t)param;
  a.gate_activation = (int32_t)act;
  a.rows = (int32_t)n;
  a.width = (int32_t)d;
  a.eps = (float)eps;
  a.block = view(keep[0]);
  a.residual = view(keep[1]);
  a.gate = view(keep[2]);
  a.post_weight = ptr(t.post);
  a.scale = ptr(t.scale);
  a.pre_weight = ptr(t.pre);
  return a;
}

// out (with a block) and normed (with pre_weight), those that there are.
variable_list norm_forward(const NormIn& t, int64_t act, int64_t param, double eps, Tensor* stats) {
  const c10::DeviceGuard guard(t.residual.device());
  Tensor keep[3];
  rc_norm_args a = norm_args(t, act, param, eps, keep);
  variable_list out;
  if (t.block.defined()) {
    out.push_back(like(t.residual));
    a.out = row_view(out.back());
  }
  if (t.pre.defined()) {
    out.push_back(like(t.block.defined() ? t.block : t.residual));
    a.normed = row_view(out.back());
  }
  if (stats) {
    *stats = at::empty({a.rows, 2}, t.residual.options().dtype(at::kFloat));
    a.stats = ptr<float>(*stats);
  }
  check(rc_norm_forward(&a, stream_of(t.residual)), "rc_norm_forward");
  return out;
}

struct Norm : torch::autograd::Function<Norm> {
  static variable_list forward(AutogradContext* ctx, const Opt& block, const Tensor& residual,
                               const Opt& gate, const Opt& post, const Opt& scale, const Opt& pre,
                               int64_t act, int64_t param, double eps) {
    const NormIn t = {given(block), residual, given(gate), given(post), given(scale), given(pre)};
    Tensor stats;
    variable_list out = norm_forward(t, act, param, eps, &stats);
    ctx->save_for_backward({t.block, t.residual, t.gate, t.post, t.scale, t.pre, stats});
    ctx->saved_data["act"] = act;
    ctx->saved_data["param"] = param;
    ctx->saved_data["eps"] = eps;
    ctx->set_materialize_grads(false);
    return out;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    for (const Tensor& g : grads) no_tangent(g);
    const auto s = ctx->get_saved_variables();
    const NormIn t = {s[0], s[1], s[2], s[3], s[4], s[5]};
    const c10::DeviceGuard guard(t.residual.device());
    Tensor keep[5];
    rc_norm_args a = norm_args(t, ctx->saved_data["act"].toInt(), ctx->saved_data["param"].toInt(),
                               ctx->saved_data["eps"].toDouble(), keep);
    size_t i = 0;
    const Tensor dout = t.block.defined() ? grads[i++] : Tensor();
    const Tensor dnormed = t.pre.defined() ? grads[i++] : Tensor();
    keep[3] = flat(dout, a.rows);
    keep[4] = flat(dnormed, a.rows);
    const Tensor dblock = like(t.block), dresidual = like(t.residual), dgate = like(t.gate),
                 dpost = like(t.post, t.post.defined() && t.post.requires_grad()),
                 dscale = like(t.scale, t.scale.defined() && t.scale.requires_grad()),
                 dpre = like(t.pre, t.pre.defined() && t.pre.requires_grad());
    a.stats = ptr<float>(s[6]);
    a.dout = view(keep[3]);
    a.dnormed = view(keep[4]);
    a.dblock = row_view(dblock);
    a.dgate = row_view(dgate);
    a.dresidual = row_view(dresidual);
    a.dpost_weight = ptr(dpost);
    a.dscale = ptr(dscale);
    a.dpre_weight = ptr(dpre);
    const Tensor work = scratch(rc_norm_backward_workspace, a, t.residual, "rc_norm_backward_workspace");
    check(rc_norm_backward(&a, stream_of(t.residual)), "rc_norm_backward");
    return once({dblock, dresidual, dgate, dpost, dscale, dpre, Tensor(), Tensor(), Tensor()});
  }
};

std::pair<Tensor, Opt> norm_residual(const Opt& block_, const Tensor& residual, const Opt& gate_,
                                     const Opt& post_, const Opt& scale_, const Opt& pre_,
                                     int64_t act, double eps) {
  NormIn t = {given(block_), residual, given(gate_), given(post_), given(scale_), given(pre_)};
  TORCH_CHECK_VALUE(residual.dim() >= 1, "residual must have a dimension of channels");
  const Tensor& main = t.block.defined() ? t.block : t.residual;
  main_tensor(t.block.defined() ? "block" : "residual", main, residual.dim());
  const int64_t d = residual.size(-1);
  TORCH_CHECK_VALUE(d <= kMaxNormWidth, "at most ", kMaxNormWidth, " channels, not ", d);
  TORCH_CHECK_VALUE(d == 0 || residual.numel() / d < (int64_t)1 << 31, "too many rows");
  expect("residual", residual, main.sizes(),
         residual.scalar_type() == at::kFloat ? at::kFloat : main.scalar_type(), main);
  if (t.block.defined()) {
    if (t.gate.defined()) expect("gate", t.gate, main.sizes(), main.scalar_type(), main);
  } else {
    TORCH_CHECK_VALUE(!t.gate.defined() && !t.post.defined() && !t.scale.defined(),
                      "gate, post_weight and scale belong to a block");
    TORCH_CHECK_VALUE(t.pre.defined(), "without a block, pre_weight is needed");
  }
  if (t.post.defined()) expect("post_weight", t.post, {d}, t.post.scalar_type(), main);
  if (t.scale.defined()) expect("scale", t.scale, {d}, t.scale.scalar_type(), main);
  if (t.pre.defined()) expect("pre_weight", t.pre, {d}, t.pre.scalar_type(), main);
  const int64_t param = param_type(
      {{"post_weight", &t.post}, {"scale", &t.scale}, {"pre_weight", &t.pre}}, main);
  const bool grad = differentiated({&t.block, &t.residual, &t.gate, &t.post, &t.scale, &t.pre});
  t.post = dense(t.post);
  t.scale = dense(t.scale);
  t.pre = dense(t.pre);
  const variable_list out =
      grad ? Norm::apply(opt(t.block), t.residual, opt(t.gate), opt(t.post), opt(t.scale), opt(t.pre),
                         act, param, eps)
           : norm_forward(t, act, param, eps, nullptr);
  if (!t.block.defined()) return {residual, out[0]};
  return {out[0], t.pre.defined() ? Opt(out[1]) : Opt()};
}

// ----------------------------------------------------------------- delta rule

// A (batch, time, head, channel) or (batch, head, channel) tensor.
rc_heads heads_view(const Tensor& t) {
  if (!t.defined()) return {nullptr, 0, 0, 0};
  if (t.dim() == 3) return {t.data_ptr(), t.stride(0), 0, t.stride(1)};
  return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}

struct DeltaIn {
  Tensor q, k, v, g, beta, state, lengths;
};

rc_delta_args delta_args(const DeltaIn& t, double scale) {
  rc_delta_args a = {};
  a.dtype = code(t.v.scalar_type());
  a.batch = (int32_t)t.v.size(0);
  a.length = (int32_t)t.v.size(1);
  a.heads = (int32_t)t.v.size(2);
  a.value = (int32_t)t.v.size(3);
  a.key_heads = (int32_t)t.q.size(2);
  a.key = (int32_t)t.q.size(3);
  a.scale = (float)scale;
  a.q = heads_view(t.q);
  a.k = heads_view(t.k);
  a.v = heads_view(t.v);
  a.g = view(t.g);
  a.beta = view(t.beta);
  a.state_in = ptr<float>(t.state);
  a.lengths = ptr<int32_t>(t.lengths);
  return a;
}

// o, and the final state if wanted; what the backward pass needs into *kept if that is not null.
variable_list delta_forward(const DeltaIn& t, double scale, bool want_state, Tensor* kept) {
  const c10::DeviceGuard guard(t.v.device());
  rc_delta_args a = delta_args(t, scale);
  variable_list out = {like(t.v)};
  a.o = heads_view(out[0]);
  const auto floats = t.v.options().dtype(at::kFloat);
  if (want_state) {
    out.push_back(at::empty({t.v.size(0), t.v.size(2), t.q.size(3), t.v.size(3)}, floats));
    a.state_out = ptr<float>(out[1]);
  }
  if (kept) {
    uint64_t n = 0;
    check(rc_delta_kept_bytes(&a, &n), "rc_delta_kept_bytes");
    *kept = at::empty({(int64_t)n / 4}, floats);
    a.kept = ptr<float>(*kept);
  }
  const Tensor work = scratch(rc_delta_forward_workspace, a, t.v, "rc_delta_forward_workspace");
  check(rc_delta_forward(&a, stream_of(t.v)), "rc_delta_forward");
  return out;
}

struct Delta : torch::autograd::Function<Delta> {
  static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& v,
                               const Opt& decay, const Tensor& beta, const Opt& state_in,
                               const Opt& ends, double scale, bool want_state) {
    const Tensor g = given(decay), state = given(state_in), lengths = given(ends);
    Tensor kept;
    variable_list out = delta_forward({q, k, v, g, beta, state, lengths}, scale, want_state, &kept);
    ctx->save_for_backward({q, k, v, g, beta, state, lengths, kept});
    ctx->saved_data["scale"] = scale;
    ctx->set_materialize_grads(false);
    return out;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    for (const Tensor& g : grads) no_tangent(g);
    const auto s = ctx->get_saved_variables();
    const DeltaIn t = {s[0], s[1], s[2], s[3], s[4], s[5], s[6]};
    const c10::DeviceGuard guard(t.v.device());
    rc_delta_args a = delta_args(t, ctx->saved_data["scale"].toDouble());
    const Tensor d_o = grads[0].defined() ? rows(grads[0]) : at::zeros_like(t.v);
    const Tensor dout = grads.size() > 1 ? dense(grads[1]) : Tensor();
    const Tensor dq = like(t.q), dk = like(t.k), dv = like(t.v), dg = like(t.g), dbeta = like(t.beta),
                 ds = like(t.state, t.state.defined() && t.state.requires_grad());
    a.kept = ptr<float>(s[7]);
    a.do_ = heads_view(d_o);
    a.dq = heads_view(dq);
    a.dk = heads_view(dk);
    a.dv = heads_view(dv);
    a.dg = ptr<float>(dg);
    a.dbeta = ptr<float>(dbeta);
    a.dstate_out = ptr<float>(dout);
    a.dstate_in = ptr<float>(ds);
    const Tensor work = scratch(rc_delta_backward_workspace, a, t.v, "rc_delta_backward_workspace");
    check(rc_delta_backward(&a, stream_of(t.v)), "rc_delta_backward");
    return once({dq, dk, dv, dg, dbeta, ds, Tensor(), Tensor(), Tensor()});
  }
};

// Checks of what the whole and the single-token form share; t.v is (tokens.., heads, value).
void delta_expect(const DeltaIn& t) {
  const int64_t dims = t.v.dim();
  TORCH_CHECK_VALUE(t.q.dim() == dims, "q must have ", dims, " dimensions, not ", t.q.dim());
  const int64_t h = t.v.size(-2), hk = t.q.size(-2), dk = t.q.size(-1), dv = t.v.size(-1);
  TORCH_CHECK_VALUE(h == 0 ? hk == 0 : hk > 0 && h % hk == 0, hk, " heads of q do not divide ", h, " heads of v");
  TORCH_CHECK_VALUE(dk >= 1 && dk <= kMaxHead, "q must have 1 to ", kMaxHead, " channels, not ", dk);
  TORCH_CHECK_VALUE(dv >= 1 && dv <= kMaxHead, "v must have 1 to ", kMaxHead, " channels, not ", dv);
  std::vector<int64_t> shape(t.v.sizes().begin(), t.v.sizes().end() - 2);
  shape.push_back(h);
  expect("beta", t.beta, shape, at::kFloat, t.v);
  if (t.g.defined()) expect("g", t.g, shape, at::kFloat, t.v);
  shape.back() = hk;
  shape.push_back(dk);
  expect("q", t.q, shape, t.v.scalar_type(), t.v);
  expect("k", t.k, shape, t.v.scalar_type(), t.v);
}

variable_list gated_delta(const Tensor& q, const Tensor& k, const Tensor& v, const Opt& g,
                          const Tensor& beta, double scale, const Opt& state, const Opt& lengths,
                          bool want_state) {
  main_tensor("v", v, 4);
  DeltaIn t = {q, k, v, given(g), beta, given(state), Tensor()};
  delta_expect(t);
  if (state) expect("state", *state, {v.size(0), v.size(2), q.size(3), v.size(3)}, at::kFloat, v);
  t.lengths = lengths_of(lengths, v);
  const bool grad = differentiated({&q, &k, &v, &t.g, &beta, &t.state});
  t = {rows(q), rows(k), rows(v), rows(t.g), rows(beta), dense(t.state), t.lengths};
  if (grad)
    return Delta::apply(t.q, t.k, t.v, opt(t.g), t.beta, opt(t.state), opt(t.lengths), scale, want_state);
  return delta_forward(t, scale, want_state, nullptr);
}

Tensor gated_delta_step(const Tensor& state, const Tensor& q, const Tensor& k, const Tensor& v,
                        const Opt& g, const Tensor& beta, double scale, const Opt& slots_) {
  main_tensor("v", v, 3);
  DeltaIn t = {q, k, v, given(g), beta, Tensor(), Tensor()};
  delta_expect(t);
  const int64_t h = v.size(1), dk = q.size(2), dv = v.size(2);
  TORCH_CHECK_VALUE(state.dim() == 4, "state must have 4 dimensions");
  expect("state", state, {state.size(0), h, dk, dv}, at::kFloat, v);
  TORCH_CHECK_VALUE((state.stride(3) == 1 || dv <= 1) && (state.stride(2) == dv || dk <= 1) &&
                        (state.stride(1) == dk * dv || h <= 1),
                    "each slot of state must be contiguous");
  TORCH_CHECK_VALUE(!overlap(state.size(0), state.stride(0), 1, 0, h * dk * dv),
                    "states must not share memory");
  const Tensor slots = slots_of(slots_, v, state);
  not_differentiated("gated_delta_step", {&state, &q, &k, &v, &t.g, &beta});
  t = {rows(q), rows(k), rows(v), rows(t.g), rows(beta), Tensor(), Tensor()};
  const c10::DeviceGuard guard(v.device());
  const Tensor o = at::empty(v.sizes(), v.options());
  rc_delta_step_args a = {};
  a.dtype = code(v.scalar_type());
  a.batch = (int32_t)v.size(0);
  a.key_heads = (int32_t)q.size(1);
  a.heads = (int32_t)h;
  a.key = (int32_t)dk;
  a.value = (int32_t)dv;
  a.num_slots = (int32_t)state.size(0);
  a.scale = (float)scale;
  a.q = heads_view(t.q);
  a.k = heads_view(t.k);
  a.v = heads_view(t.v);
  a.o = heads_view(o);
  a.g = view(t.g);
  a.beta = view(t.beta);
  a.state = ptr<float>(state);
  a.state_slot = state.stride(0);
  a.slots = ptr<int32_t>(slots);
  check(rc_delta_step(&a, stream_of(v)), "rc_delta_step");
  written(state);
  return o;
}

// ----------------------------------------------------------- queries and keys

struct QkIn {
  Tensor q, k, qw, kw, freq, positions, lengths;
};

rc_qk_args qk_args(const QkIn& t, int64_t norm, bool interleaved, int64_t param, double eps) {
  rc_qk_args a = {};
  a.dtype = code(t.q.scalar_type());
  a.param_dtype = (int32_t)param;
  a.norm = (int32_t)norm;
  a.interleaved = interleaved;
  a.batch = (int32_t)t.q.size(0);
  a.length = (int32_t)t.q.size(1);
  a.heads = (int32_t)t.q.size(2);
  a.key_heads = (int32_t)t.k.size(2);
  a.channels = (int32_t)t.q.size(3);
  a.rotated = t.freq.defined() ? 2 * (int32_t)t.freq.size(0) : 0;
  a.eps = (float)eps;
  a.q = heads_view(t.q);
  a.k = heads_view(t.k);
  a.q_weight = ptr(t.qw);
  a.k_weight = ptr(t.kw);
  a.inv_freq = ptr<float>(t.freq);
  if (t.positions.defined()) {
    a.positions = ptr<int32_t>(t.positions);
    a.positions_batch = t.positions.stride(0);
    a.positions_time = t.positions.stride(1);
  }
  a.lengths = ptr<int32_t>(t.lengths);
  return a;
}

variable_list qk_forward(const QkIn& t, int64_t norm, bool interleaved, int64_t param, double eps) {
  const c10::DeviceGuard guard(t.q.device());
  rc_qk_args a = qk_args(t, norm, interleaved, param, eps);
  variable_list out = {like(t.q), like(t.k)};
  a.q_out = heads_view(out[0]);
  a.k_out = heads_view(out[1]);
  check(rc_qk_forward(&a, stream_of(t.q)), "rc_qk_forward");
  return out;
}

struct Qk : torch::autograd::Function<Qk> {
  static variable_list forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Opt& qw,
                               const Opt& kw, const Opt& freq, const Opt& positions, const Opt& ends,
                               int64_t norm, bool interleaved, int64_t param, double eps) {
    const QkIn t = {q, k, given(qw), given(kw), given(freq), given(positions), given(ends)};
    ctx->save_for_backward({t.q, t.k, t.qw, t.kw, t.freq, t.positions, t.lengths});
    ctx->saved_data["norm"] = norm;
    ctx->saved_data["interleaved"] = interleaved;
    ctx->saved_data["param"] = param;
    ctx->saved_data["eps"] = eps;
    ctx->set_materialize_grads(false);
    return qk_forward(t, norm, interleaved, param, eps);
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    for (const Tensor& g : grads) no_tangent(g);
    const auto s = ctx->get_saved_variables();
    const QkIn t = {s[0], s[1], s[2], s[3], s[4], s[5], s[6]};
    const c10::DeviceGuard guard(t.q.device());
    rc_qk_args a = qk_args(t, ctx->saved_data["norm"].toInt(), ctx->saved_data["interleaved"].toBool(),
                           ctx->saved_data["param"].toInt(), ctx->saved_data["eps"].toDouble());
    const Tensor gq = rows(grads[0]), gk = rows(grads[1]), dq = like(t.q), dk = like(t.k),
                 dqw = like(t.qw, t.qw.defined() && t.qw.requires_grad()),
                 dkw = like(t.kw, t.kw.defined() && t.kw.requires_grad());
    a.dq_out = heads_view(gq);
    a.dk_out = heads_view(gk);
    a.dq = heads_view(dq);
    a.dk = heads_view(dk);
    a.dq_weight = ptr(dqw);
    a.dk_weight = ptr(dkw);
    const Tensor work = scratch(rc_qk_backward_workspace, a, t.q, "rc_qk_backward_workspace");
    check(rc_qk_backward(&a, stream_of(t.q)), "rc_qk_backward");
    return once({dq, dk, dqw, dkw, Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor()});
  }
};

variable_list qk_norm(const Tensor& q, const Tensor& k, const Opt& qw, const Opt& kw, const Opt& freq,
                      const Opt& positions, const Opt& lengths, int64_t norm, bool interleaved,
                      double eps) {
  main_tensor("q", q, 4);
  QkIn t = {q, k, given(qw), given(kw), given(freq), given(positions), Tensor()};
  const int64_t d = q.size(3);
  TORCH_CHECK_VALUE(d >= 1 && d <= kMaxHead, "q must have 1 to ", kMaxHead, " channels, not ", d);
  TORCH_CHECK_VALUE(k.dim() == 4, "k must have 4 dimensions, not ", k.dim());
  expect("k", k, {q.size(0), q.size(1), k.size(2), d}, q.scalar_type(), q);
  if (t.qw.defined()) expect("q_weight", t.qw, {d}, t.qw.scalar_type(), q);
  if (t.kw.defined()) expect("k_weight", t.kw, {d}, t.kw.scalar_type(), q);
  const int64_t param = param_type({{"q_weight", &t.qw}, {"k_weight", &t.kw}}, q);
  if (t.freq.defined()) {
    TORCH_CHECK_VALUE(t.freq.dim() == 1 && 2 * t.freq.size(0) <= d, "inv_freq must have at most ", d / 2,
                      " numbers in one dimension, not ", t.freq.sizes());
    expect("inv_freq", t.freq, t.freq.sizes(), at::kFloat, q);
    if (t.freq.size(0) == 0) t.freq = Tensor();
  }
  TORCH_CHECK_VALUE(!differentiated({&t.freq}), "inv_freq has no gradient: detach it");
  if (t.positions.defined()) expect("positions", t.positions, {q.size(0), q.size(1)}, at::kInt, q);
  t.lengths = lengths_of(lengths, q);
  const bool grad = differentiated({&q, &k, &t.qw, &t.kw});
  if (t.positions.defined()) t.positions = plain(t.positions);
  t = {rows(q), rows(k), dense(t.qw), dense(t.kw), dense(t.freq), t.positions, t.lengths};
  if (grad)
    return Qk::apply(t.q, t.k, opt(t.qw), opt(t.kw), opt(t.freq), opt(t.positions), opt(t.lengths), norm,
                     interleaved, param, eps);
  return qk_forward(t, norm, interleaved, param, eps);
}

// -------------------------------------------------------------------- dropout

rc_dropout_args dropout_args(const Tensor& seed, int64_t number, int64_t tag, double p) {
  rc_dropout_args a = {};
  a.p = p;
  a.seed = number;
  a.tag = tag;
  a.seed_device = ptr<const int64_t>(seed);
  return a;
}
// x and out (its gradient backward) as rows; both of the same shape.
void dropout_rows(rc_dropout_args& a, const Tensor& x, const Tensor& out) {
  a.dtype = code(x.scalar_type());
  a.out_dtype = code(out.scalar_type());
  a.rows = x.size(0);
  a.width = x.size(1);
  a.x = view(x);
  a.out = view(out);
}
// Any shape as rows of the last dimension.
Tensor as_rows(const Tensor& t) {
  if (!t.defined()) return t;
  const int64_t d = t.dim() ? t.size(-1) : 1;
  return flat(t.dim() ? t : t.reshape({1, 1}), d ? t.numel() / d : 0);
}

Tensor dropout_forward(const Tensor& x, const Tensor& residual, const Tensor& seed, int64_t number,
                       int64_t tag, double p) {
  const c10::DeviceGuard guard(x.device());
  const Tensor out = at::empty(x.sizes(), (residual.defined() ? residual : x).options());
  const Tensor xs = as_rows(x), rs = as_rows(residual), ys = as_rows(out);
  rc_dropout_args a = dropout_args(seed, number, tag, p);
  dropout_rows(a, xs, ys);
  a.residual = view(rs);
  check(rc_dropout_forward(&a, stream_of(x)), "rc_dropout_forward");
  return out;
}

struct Dropout : torch::autograd::Function<Dropout> {
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const Opt& residual, const Opt& seed,
                        int64_t number, int64_t tag, double p) {
    ctx->save_for_backward({given(seed)});
    ctx->saved_data["number"] = number;
    ctx->saved_data["tag"] = tag;
    ctx->saved_data["p"] = p;
    ctx->saved_data["dtype"] = x.scalar_type();
    ctx->saved_data["residual"] = residual.has_value();
    return dropout_forward(x, given(residual), given(seed), number, tag, p);
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    for (const Tensor& g : grads) no_tangent(g);
    const Tensor seed = ctx->get_saved_variables()[0], &g = grads[0];
    const c10::DeviceGuard guard(g.device());
    const Tensor dx = at::empty(g.sizes(), g.options().dtype(ctx->saved_data["dtype"].toScalarType()));
    const Tensor gs = as_rows(g), xs = as_rows(dx);
    rc_dropout_args a = dropout_args(seed, ctx->saved_data["number"].toInt(), ctx->saved_data["tag"].toInt(),
                                     ctx->saved_data["p"].toDouble());
    dropout_rows(a, xs, gs);
    check(rc_dropout_backward(&a, stream_of(g)), "rc_dropout_backward");
    const Tensor dr = ctx->saved_data["residual"].toBool() ? g : Tensor();
    return once({dx, dr, Tensor(), Tensor(), Tensor(), Tensor()});
  }
};

Tensor dropout(const Tensor& x, double p, const Opt& seed_, int64_t number, int64_t tag,
               const Opt& residual_) {
  activations("x", x);
  const Tensor residual = given(residual_);
  Tensor seed = given(seed_);
  TORCH_CHECK_VALUE(p >= 0 && p <= 1, "p must be from 0 to 1, not ", p);
  if (residual.defined())
    expect("residual", residual, x.sizes(),
           residual.scalar_type() == at::kFloat ? at::kFloat : x.scalar_type(), x);
  if (seed.defined()) {
    TORCH_CHECK_VALUE(seed.numel() == 1, "seed must be one number, not ", seed.sizes());
    expect("seed", seed, seed.sizes(), at::kLong, x);
    seed = plain(seed);
  }
  if (differentiated({&x, &residual})) return Dropout::apply(x, opt(residual), opt(seed), number, tag, p);
  return dropout_forward(x, residual, seed, number, tag, p);
}

}  // namespace

PYBIND11_MODULE(_ops, m) {
  m.def("causal_conv", &causal_conv);
  m.def("causal_conv_step", &causal_conv_step);
  m.def("selective_scan", &selective_scan);
  m.def("selective_scan_step", &selective_scan_step);
  m.def("norm_residual", &norm_residual);
  m.def("gated_delta", &gated_delta);
  m.def("gated_delta_step", &gated_delta_step);
  m.def("qk_norm", &qk_norm);
  m.def("dropout", &dropout);
}
