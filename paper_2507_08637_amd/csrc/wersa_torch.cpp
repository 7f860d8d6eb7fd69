// The attention core, and the causal operators, as nodes of torch's autograd graph, in C++: what a training step pays for on the host beyond the launches.  The engine runs
// a backward on a thread of its own, and interpreter state, reference counts and runtime structures that both threads touch move between their
// caches at every change.  2 x 4 slices of 1000 tokens, d 64, m 256, bf16, forward and backward: 235 to 246 us where the engine's thread runs far from
// the caller's and 128 to 136 where near with a node written in Python, 128 to 138 and 98 with this one; its kernels take 97.
//
// The library is reached through the addresses of its entry points (bind): this module has no link to it, and loads whichever the
// binding loaded.  The forward's arguments are checked by the caller, what the backward unpacks is checked here; the library checks the
// rest, and its status is raised as the binding's error.
#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/utils/pybind.h>

#include <algorithm>
#include <cstring>

#include "../../include/wersa.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

decltype(&wersa_forward) forward_fn = nullptr;
decltype(&wersa_backward) backward_fn = nullptr;
decltype(&wersa_workspace_bytes) workspace_bytes_fn = nullptr;
decltype(&wersa_saved_bytes) saved_bytes_fn = nullptr;
decltype(&wersa_selected_path) selected_path_fn = nullptr;

wersa_desc desc_of(const std::string &bytes) {
  wersa_desc d;
  TORCH_CHECK(bytes.size() == sizeof(d), "descriptor of another size");
  std::memcpy(&d, bytes.data(), sizeof(d));
  return d;
}

// Raises WersaError(status) in whichever thread this is.
void check(wersa_status status) {
  if (status == WERSA_OK) return;
  pybind11::gil_scoped_acquire gil;
  try {
    pybind11::module_::import("paper_2507_08637_amd.binding").attr("_check")((int)status);
  } catch (pybind11::error_already_set &e) {
    e.restore();
    python_error err;
    err.persist();
    throw err;
  }
}

// Raises AssertionError, as the binding's checks do, unless `holds`.
void require(bool holds, const char *text) {
  if (holds) return;
  pybind11::gil_scoped_acquire gil;
  PyErr_SetString(PyExc_AssertionError, text);
  python_error err;
  err.persist();
  throw err;
}

// (host tensors have no stream: entry points that only note their arguments are given such)
void *stream(const Tensor &t) { return t.is_cuda() ? (void *)c10::hip::getCurrentHIPStream().stream() : nullptr; }
Tensor scratch(int64_t bytes, const Tensor &like) {
  return at::empty({bytes < 256 ? 256 : bytes}, like.options().dtype(at::kByte));
}
const float *floats(const Tensor &t) { return static_cast<const float *>(t.const_data_ptr()); }
float *floats_out(const Tensor &t) { return static_cast<float *>(t.mutable_data_ptr()); }

bool same_layout(const Tensor &a, const Tensor &b) { return a.sizes() == b.sizes() && a.strides() == b.strides() && a.dtype() == b.dtype(); }
bool holds_floats(const Tensor &t, int64_t count) { return t.dtype() == at::kFloat && t.is_contiguous() && t.numel() >= count; }

struct Attention : torch::autograd::Function<Attention> {
  static Tensor forward(AutogradContext *ctx, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &omega, const Tensor &sigma,
                        const Tensor &gate_w, const Tensor &gate_b, const Tensor &scale_w, const std::string &desc, int64_t saved_bytes,
                        int64_t workspace) {
    const wersa_desc d = desc_of(desc);
    const Tensor out = at::empty_strided(q.sizes(), q.strides(), q.options());
    const Tensor saved = at::empty({saved_bytes / 4}, q.options().dtype(at::kFloat));
    const Tensor ws = scratch(workspace, q);
    check(forward_fn(&d, q.const_data_ptr(), k.const_data_ptr(), v.const_data_ptr(), omega.const_data_ptr(), floats(sigma), floats(gate_w),
                     floats(gate_b), floats(scale_w), out.mutable_data_ptr(), saved.mutable_data_ptr(), ws.mutable_data_ptr(), ws.nbytes(),
                     stream(q)));
    ctx->save_for_backward({q, k, v, omega, sigma, gate_w, gate_b, scale_w, out, saved});
    ctx->saved_data["desc"] = desc;
    return out;
  }

  // Saved-tensor hooks may give the tensors back in another layout than the forward had them in (save_on_cpu makes them dense, or contiguous):
  // the call, its workspace and its outputs are described by the tensors that are there now.
  static variable_list backward(AutogradContext *ctx, const variable_list &grads) {
    const variable_list t = ctx->get_saved_variables();
    Tensor q = t[0], k = t[1], v = t[2], out = t[8], dout = grads[0];
    const Tensor &omega = t[3], &sigma = t[4], &gate_w = t[5], &gate_b = t[6], &scale_w = t[7], &saved = t[9];
    const wersa_desc then = desc_of(ctx->saved_data["desc"].toStringRef());
    wersa_desc d = then;
    require(q.dim() == 4 && q.sizes() == at::IntArrayRef({d.B, d.H, d.n, d.d}) && q.stride(3) == 1 &&
                q.dtype() == (d.dtype == WERSA_F32 ? at::kFloat : at::kBFloat16),
            "expect q as it was saved: (B, H, n, d) with contiguous last dim");
    d.stride_b = q.stride(0), d.stride_h = q.stride(1), d.stride_n = q.stride(2);
    require(same_layout(q, k) && same_layout(q, v) && same_layout(q, out), "q, k, v, out and gradients must share shape, strides and dtype");
    const int path = selected_path_fn(&d);
    if (path >= 0 && path != selected_path_fn(&then)) {   // `saved` is laid out for the other path (strides of 8 elements or not): back to its strides
      d = then;
      for (Tensor *x : {&q, &k, &v, &out}) *x = at::empty_strided(x->sizes(), {d.stride_b, d.stride_h, d.stride_n, 1}, x->options()).copy_(*x);
    }
    auto like_q = [&]() { return at::empty_strided(q.sizes(), q.strides(), q.options()); };
    if (dout.strides() != q.strides()) dout = like_q().copy_(dout);
    require(same_layout(q, dout), "q, k, v, out and gradients must share shape, strides and dtype");
    const int64_t matrices = d.flags & WERSA_FLAG_SEPARATE_OMEGA ? 2 : 1;
    require(omega.is_contiguous() && omega.dtype() == q.dtype() && omega.numel() == matrices * d.d * d.m &&
                holds_floats(sigma, 1) && holds_floats(gate_w, (int64_t)d.H * (d.L + 1) * d.d) && holds_floats(gate_b, (int64_t)d.H * (d.L + 1)) &&
                holds_floats(scale_w, d.L + 1),
            "expect omega and the parameters as they were saved");
    require(holds_floats(saved, (int64_t)saved_bytes_fn(&d) / 4), "the saved buffer holds less than wersa_saved_bytes asks for");
    for (const Tensor &x : t) require(x.device() == dout.device(), "saved tensors on another device");
    const Tensor dq = like_q(), dk = like_q(), dv = like_q(), dgw = at::empty_like(gate_w), dgb = at::empty_like(gate_b),
                 dsw = at::empty_like(scale_w), dsg = at::empty({1}, sigma.options());
    const Tensor ws = scratch((int64_t)workspace_bytes_fn(&d, 1), q);
    check(backward_fn(&d, q.const_data_ptr(), k.const_data_ptr(), v.const_data_ptr(), omega.const_data_ptr(), floats(sigma), floats(gate_w),
                      floats(gate_b), floats(scale_w), out.const_data_ptr(), dout.const_data_ptr(), saved.const_data_ptr(), dq.mutable_data_ptr(),
                      dk.mutable_data_ptr(), dv.mutable_data_ptr(), floats_out(dgw), floats_out(dgb), floats_out(dsw), floats_out(dsg),
                      ws.mutable_data_ptr(), ws.nbytes(), stream(q)));
    return {dq, dk, dv, Tensor(), dsg, dgw, dgb, dsw, Tensor(), Tensor(), Tensor()};
  }
};

Tensor attention(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &omega, const Tensor &sigma, const Tensor &gate_w,
                 const Tensor &gate_b, const Tensor &scale_w, const pybind11::bytes &desc, int64_t saved_bytes, int64_t workspace) {
  const std::string d = desc;
  pybind11::gil_scoped_release nogil;
  return Attention::apply(q, k, v, omega, sigma, gate_w, gate_b, scale_w, d, saved_bytes, workspace);
}

// ---- the causal operators ------------------------------------------------------------------------------
// Decay attention and the RMS norm, whose kernels for some thousand tokens take less than the host's part of a step.  128000 rows of 128, float32, forward and backward of the norm: 95 us
// with a node in Python where the engine's thread runs near the caller's, 175 where it runs far; its kernels take 89.
decltype(&wersa_decay_forward) decay_forward_fn = nullptr;
decltype(&wersa_decay_backward) decay_backward_fn = nullptr;
decltype(&wersa_decay_workspace_bytes) decay_workspace_bytes_fn = nullptr;
decltype(&wersa_decay_saved_bytes) decay_saved_bytes_fn = nullptr;
decltype(&wersa_rms_norm_forward) norm_forward_fn = nullptr;
decltype(&wersa_rms_norm_backward) norm_backward_fn = nullptr;
decltype(&wersa_rms_norm_workspace_bytes) norm_workspace_bytes_fn = nullptr;

Tensor or_none(const std::optional<Tensor> &t) { return t ? *t : Tensor(); }
const void *in(const Tensor &t) { return t.defined() ? t.const_data_ptr() : nullptr; }
void *out_of(const Tensor &t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
int32_t dtype_of(const Tensor &t) { return t.scalar_type() == at::kFloat ? WERSA_F32 : t.scalar_type() == at::kBFloat16 ? WERSA_BF16 : -1; }
// A backward runs with gradients enabled where a graph of it is wanted: there is none of what the kernels do.
void once() { TORCH_CHECK(!at::GradMode::is_enabled(), "the causal operators are differentiable once"); }

// Rows with contiguous columns that do not share memory, heads and sequences that are not one: as the library reads them.
bool rows_apart(const Tensor &t) {
  return t.stride(3) == 1 && (t.stride(0) > 0 || t.size(0) == 1) && (t.stride(1) > 0 || t.size(1) == 1) && (t.stride(2) >= t.size(3) || t.size(2) <= 1);
}
void put_strides(int64_t *to, const Tensor &t) {
  for (int i = 0; i < 3; ++i) to[i] = t.stride(i);
}
// A new tensor of t's shape, with its dimensions in t's order in memory but none apart from or on another: t may be a slice, or windows that overlap.
Tensor dense_like(const Tensor &t) {
  int order[3] = {0, 1, 2};
  std::stable_sort(order, order + 3, [&](int a, int b) { return t.stride(a) < t.stride(b); });
  int64_t strides[4] = {1, 1, 1, 1}, step = t.size(3);
  for (const int i : order) {
    strides[i] = step;
    step *= std::max<int64_t>(1, t.size(i));
  }
  return at::empty_strided(t.sizes(), strides, t.options());
}

struct DecayAttention : torch::autograd::Function<DecayAttention> {
  static variable_list forward(AutogradContext *ctx, const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &log_decay, const std::optional<Tensor> &initial_state,
                               const std::optional<Tensor> &sequences, const std::string &desc, int64_t saved_bytes) {
    const Tensor initial = or_none(initial_state), offsets = or_none(sequences);
    wersa_decay_desc d;
    TORCH_CHECK(desc.size() == sizeof(d), "descriptor of another size");
    std::memcpy(&d, desc.data(), sizeof(d));
    const Tensor out = dense_like(v);
    put_strides(d.stride_o, out);
    d.clear = d.packed;
    const auto f32 = q.options().dtype(at::kFloat);
    const Tensor final_state = at::empty({d.B, d.H, d.dk, d.dv}, f32), saved = at::empty({saved_bytes / 4}, f32);
    check(decay_forward_fn(&d, in(q), in(k), in(v), floats(log_decay), (const int32_t *)in(offsets), (const float *)in(initial), floats_out(final_state), nullptr,
                           d.B, out.mutable_data_ptr(), saved.mutable_data_ptr(), nullptr, 0, stream(q)));
    ctx->save_for_backward({q, k, v, log_decay, initial, offsets, saved});
    ctx->saved_data["desc"] = desc;
    ctx->set_materialize_grads(false);
    return {out, final_state};
  }

  // As above, the call is described by the tensors that are there now.  `saved` does not depend on their strides.
  static variable_list backward(AutogradContext *ctx, const variable_list &grads) {
    once();
    const variable_list t = ctx->get_saved_variables();
    const Tensor &q = t[0], &k = t[1], &v = t[2], &log_decay = t[3], &initial = t[4], &offsets = t[5], &saved = t[6];
    wersa_decay_desc d;
    std::memcpy(&d, ctx->saved_data["desc"].toStringRef().data(), sizeof(d));
    const int64_t N = d.packed ? 1 : d.B;
    for (const Tensor *x : {&q, &k, &v})
      require(x->dim() == 4 && x->sizes() == at::IntArrayRef({N, d.H, d.n, x == &v ? d.dv : d.dk}) && dtype_of(*x) == d.dtype && rows_apart(*x),
              "expect q, k and v as they were saved: (B, H, n, d) with contiguous last dim");
    auto states = [&](const Tensor &x) { return !x.defined() || (holds_floats(x, (int64_t)d.B * d.H * d.dk * d.dv)); };
    require(holds_floats(log_decay, d.H) && states(initial) && holds_floats(saved, (int64_t)decay_saved_bytes_fn(&d) / 4) &&
                (offsets.defined() ? d.packed && offsets.scalar_type() == at::kInt && offsets.is_contiguous() && offsets.numel() == d.B + 1 : !d.packed),
            "expect log_decay, the states and the offsets as they were saved");
    Tensor dout = grads[0], dfinal = grads[1];
    if (!dout.defined()) dout = at::zeros(v.sizes(), v.options());
    if (!rows_apart(dout)) dout = dout.contiguous();
    if (dfinal.defined()) dfinal = dfinal.contiguous();
    require(dout.sizes() == v.sizes() && dout.dtype() == v.dtype() && states(dfinal), "gradients of other shapes or types than the outputs");
    for (const Tensor &x : t) require(!x.defined() || x.device() == dout.device(), "saved tensors on another device");
    put_strides(d.stride_q, q);
    put_strides(d.stride_k, k);
    put_strides(d.stride_v, v);
    put_strides(d.stride_o, dout);
    const Tensor dq = dense_like(q), dk = dense_like(k), dv = dense_like(v), dinitial = initial.defined() && ctx->needs_input_grad(4) ? at::empty_like(initial) : Tensor();
    put_strides(d.stride_dq, dq);
    put_strides(d.stride_dk, dk);
    put_strides(d.stride_dv, dv);
    const Tensor ws = scratch((int64_t)decay_workspace_bytes_fn(&d, 1), q);
    check(decay_backward_fn(&d, in(q), in(k), in(v), floats(log_decay), (const int32_t *)in(offsets), (const float *)in(initial), in(dout),
                            (const float *)in(dfinal), saved.const_data_ptr(), out_of(dq), out_of(dk), out_of(dv), (float *)out_of(dinitial),
                            ws.mutable_data_ptr(), ws.nbytes(), stream(q)));
    return {dq, dk, dv, Tensor(), dinitial, Tensor(), Tensor(), Tensor()};
  }
};

struct RmsNorm : torch::autograd::Function<RmsNorm> {
  static variable_list forward(AutogradContext *ctx, const Tensor &x, const std::optional<Tensor> &weights, const std::optional<Tensor> &added, double eps) {
    const Tensor weight = or_none(weights), residual = or_none(added);
    const int64_t rows = x.size(0), cols = x.size(1);
    const wersa_norm_desc d{rows, (int32_t)cols, dtype_of(x), (float)eps, x.stride(0), residual.defined() ? residual.stride(0) : cols};
    const Tensor y = at::empty({rows, cols}, x.options()), r = residual.defined() ? at::empty({rows, cols}, x.options()) : Tensor(),
                 rstd = at::empty({rows}, x.options().dtype(at::kFloat));
    check(norm_forward_fn(&d, in(x), in(residual), (const float *)in(weight), out_of(r), out_of(y), floats_out(rstd), stream(x)));
    ctx->save_for_backward({r.defined() ? r : x, weight, rstd});
    ctx->set_materialize_grads(false);
    return r.defined() ? variable_list{y, r} : variable_list{y};
  }

  static variable_list backward(AutogradContext *ctx, const variable_list &grads) {
    once();
    const variable_list t = ctx->get_saved_variables();
    const Tensor &r = t[0], &weight = t[1], &rstd = t[2];
    require(r.dim() == 2 && r.stride(1) == 1 && dtype_of(r) >= 0 && (r.size(0) <= 1 || r.stride(0) >= r.size(1)) && holds_floats(rstd, r.size(0)) &&
                (!weight.defined() || holds_floats(weight, r.size(1))),
            "expect the stream, the weight and the statistics as they were saved");
    const int64_t rows = r.size(0), cols = r.size(1);
    const Tensor dy = grads[0].defined() ? grads[0].contiguous() : at::zeros({rows, cols}, r.options());
    const Tensor dr = grads.size() > 1 && grads[1].defined() ? grads[1].contiguous() : Tensor();
    for (const Tensor *x : {&dy, &dr})
      require(!x->defined() || (x->sizes() == r.sizes() && x->dtype() == r.dtype()), "gradients of other shapes or types than the outputs");
    for (const Tensor &x : t) require(!x.defined() || x.device() == dy.device(), "saved tensors on another device");
    const wersa_norm_desc d{rows, (int32_t)cols, dtype_of(r), 0.f, r.stride(0), cols};
    const bool wants = weight.defined() && ctx->needs_input_grad(1);
    const Tensor dx = at::empty({rows, cols}, r.options()), dw = wants ? at::empty_like(weight) : Tensor(),
                 ws = wants ? scratch((int64_t)norm_workspace_bytes_fn(&d), r) : Tensor();
    check(norm_backward_fn(&d, in(r), (const float *)in(weight), floats(rstd), in(dy), in(dr), out_of(dx), (float *)out_of(dw), out_of(ws),
                           wants ? ws.nbytes() : 0, stream(r)));
    // (gradients are asked for by the tensors that there are)
    return {dx, dw, grads.size() > 1 && ctx->needs_input_grad(weight.defined() ? 2 : 1) ? dx : Tensor(), Tensor()};
  }
};

variable_list decay_attention(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &log_decay, const std::optional<Tensor> &initial,
                              const std::optional<Tensor> &offsets, const pybind11::bytes &desc, int64_t saved_bytes) {
  const std::string d = desc;
  pybind11::gil_scoped_release nogil;
  return DecayAttention::apply(q, k, v, log_decay, initial, offsets, d, saved_bytes);
}

variable_list rms_norm(const Tensor &x, const std::optional<Tensor> &weight, const std::optional<Tensor> &residual, double eps) {
  pybind11::gil_scoped_release nogil;
  return RmsNorm::apply(x, weight, residual, eps);
}

}  // namespace

PYBIND11_MODULE(_wersa_torch, m) {
  m.def("bind", [](uintptr_t forward, uintptr_t backward, uintptr_t workspace_bytes, uintptr_t saved_bytes, uintptr_t selected_path) {
    forward_fn = reinterpret_cast<decltype(forward_fn)>(forward);
    backward_fn = reinterpret_cast<decltype(backward_fn)>(backward);
    workspace_bytes_fn = reinterpret_cast<decltype(workspace_bytes_fn)>(workspace_bytes);
    saved_bytes_fn = reinterpret_cast<decltype(saved_bytes_fn)>(saved_bytes);
    selected_path_fn = reinterpret_cast<decltype(selected_path_fn)>(selected_path);
  });
  m.def("attention", &attention);
  m.def("bind_causal", [](const std::vector<uintptr_t> &at) {
    TORCH_CHECK(at.size() == 7, "seven entry points");
    decay_forward_fn = reinterpret_cast<decltype(decay_forward_fn)>(at[0]);
    decay_backward_fn = reinterpret_cast<decltype(decay_backward_fn)>(at[1]);
    decay_workspace_bytes_fn = reinterpret_cast<decltype(decay_workspace_bytes_fn)>(at[2]);
    decay_saved_bytes_fn = reinterpret_cast<decltype(decay_saved_bytes_fn)>(at[3]);
    norm_forward_fn = reinterpret_cast<decltype(norm_forward_fn)>(at[4]);
    norm_backward_fn = reinterpret_cast<decltype(norm_backward_fn)>(at[5]);
    norm_workspace_bytes_fn = reinterpret_cast<decltype(norm_workspace_bytes_fn)>(at[6]);
  });
  m.def("decay_attention", &decay_attention);
  m.def("rms_norm", &rms_norm);
}
