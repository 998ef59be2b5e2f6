// The calls of exact attention that sit on a user's path, marshalled in native code
// as those of MRA-2 are (binding.cpp): the argument checks, the allocations and the
// library call of the forward, and the autograd node of exact_attention. The
// library is bound at run time (the addresses of the libmra_exact.so that
// ops.load_exact opened).
//
// Why native: one sequence of 512 tokens x 12 heads, forward and backward, is 44 us on the
// GPU in four launches and took 203 us a step with the Python autograd function.
#include <cmath>
#include <limits>

#include "binding_rows.h"

namespace {

constexpr const char* kName = "exact_attention";

struct Api {
  decltype(&mra_exact_forward_workspace_bytes) forward_ws;
  decltype(&mra_exact_forward) forward;
  decltype(&mra_exact_backward_workspace_bytes) backward_ws;
  decltype(&mra_exact_backward) backward;
};
Api api{};

// The optional tensors of a call.
struct Extras {
  const at::Tensor *lengths, *key_mask, *q_start, *bias, *buckets;
};

// Every check of the tensors, as ops._exact_problem makes them.
mra_exact_problem_t problem(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, double scale, bool causal,
                            const Extras& x) {
  TORCH_CHECK_VALUE(q.is_cuda() && k.is_cuda() && v.is_cuda(), "tensors must be on a ROCm device");
  TORCH_CHECK_VALUE(q.dim() == 4 && k.dim() == 4 && v.dim() == 4, "q, k, v must have shape [B, heads, n, d]");
  mra_exact_problem_t p{};
  p.dtype = dtype_code(q);
  const int64_t B = q.size(0), H = q.size(1), nq = q.size(2), d = q.size(3), Hkv = k.size(1), nk = k.size(2);
  TORCH_CHECK_VALUE(k.sizes() == at::IntArrayRef({B, Hkv, nk, d}) && v.sizes() == k.sizes() && (Hkv ? H % Hkv : H) == 0,
                    "k, v must share shape [B, H_kv, n_k, d] with q's B and d, H a multiple of H_kv");
  for (const int64_t n : {B, H, nq, d, Hkv, nk})
    TORCH_CHECK_VALUE(n <= std::numeric_limits<int>::max(), "sizes must be below 2^31");
  check_rows(q, q, q.sizes(), "q");
  check_rows(k, q, k.sizes(), "k");
  check_rows(v, q, v.sizes(), "v");
  const at::Device dev = q.device();
  if (x.lengths) check_int(*x.lengths, {B}, "lengths", dev);
  if (x.q_start) check_int(*x.q_start, {B}, "q_start", dev);
  if (x.key_mask) {
    const at::Tensor& m = *x.key_mask;
    TORCH_CHECK_VALUE((m.scalar_type() == at::kBool || m.scalar_type() == at::kByte) &&
                          m.sizes() == at::IntArrayRef({B, nk}) && (nk <= 1 || m.stride(1) == 1) && m.device() == dev,
                      "key_mask must be a bool or uint8 tensor of shape ", tuple_of({B, nk}), " with dense rows", on(dev));
    p.key_mask = static_cast<const uint8_t*>(m.data_ptr());
    p.key_mask_stride = B > 1 ? m.stride(0) : 0;
  }
  TORCH_CHECK_VALUE(!x.bias == !x.buckets, "bias and buckets go together");
  if (x.bias) {
    const at::Tensor &b = *x.bias, &m = *x.buckets;
    TORCH_CHECK_VALUE(b.dim() == 2 && b.size(1) == H &&
                          (b.scalar_type() == q.scalar_type() || b.scalar_type() == at::kFloat) && b.is_contiguous() &&
                          b.device() == dev,
                      "bias must be a contiguous tensor of shape [buckets, ", H, "], float32 or q's dtype,", on(dev));
    TORCH_CHECK_VALUE(m.dim() == 1 && m.numel() % 2 == 1, "buckets must be int32 of odd length (see distance_buckets)");
    check_int(m, m.sizes(), "buckets", dev);
    p.bias = b.data_ptr();
    p.bias_dtype = dtype_code(b);
    p.buckets = (int)b.size(0);
    p.bucket_map = static_cast<const int32_t*>(m.data_ptr());
    p.far = (int)(m.numel() / 2);
  }
  p.B = (int)B;
  p.H = (int)H;
  p.H_kv = (int)Hkv;
  p.n_q = (int)nq;
  p.n_k = (int)nk;
  p.d = (int)d;
  p.scale = (float)scale;
  p.causal = causal;
  p.lengths = x.lengths ? static_cast<const int32_t*>(x.lengths->data_ptr()) : nullptr;
  p.q_start = x.q_start ? static_cast<const int32_t*>(x.q_start->data_ptr()) : nullptr;
  return p;
}

double scale_or(const std::optional<double>& scale, const at::Tensor& q) {
  return scale ? *scale : q.dim() == 4 && q.size(3) > 0 ? 1.0 / std::sqrt((double)q.size(3)) : 1.0;
}

void call_forward(const mra_exact_problem_t& p, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v,
                  const at::Tensor& out, float* lse, const Opt& workspace) {
  const c10::DeviceGuard guard(q.device());
  at::Tensor ws;
  if (given(workspace)) {
    TORCH_CHECK_VALUE(workspace->device() == q.device() && workspace->is_contiguous(),
                      "workspace must be a contiguous tensor", on(q.device()));
    ws = *workspace;
  } else if (const size_t need = api.forward_ws(&p)) {
    ws = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
  }
  const mra_strided_t vq = view(q), vk = view(k), vv = view(v), vo = view(out);
  ok("mra_exact_forward", api.forward(&p, &vq, &vk, &vv, &vo, lse, ws.defined() ? ws.data_ptr() : nullptr,
                                      ws.defined() ? ws.nbytes() : 0, stream_of(q)));
}

// ops.exact_attention_forward
at::Tensor forward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, std::optional<double> scale,
                   bool causal, const Opt& lengths, const Opt& key_mask, const Opt& q_start, const Opt& bias,
                   const Opt& buckets, const Opt& out, const Opt& lse_out, const Opt& workspace) {
  const mra_exact_problem_t p = problem(q, k, v, scale_or(scale, q), causal,
                                        {given(lengths), given(key_mask), given(q_start), given(bias), given(buckets)});
  if (out) check_out(*out, q, "out");
  const at::Tensor z = out ? *out : rows_like(q);
  float* lse = nullptr;
  if (lse_out) {
    TORCH_CHECK_VALUE(lse_out->scalar_type() == at::kFloat && lse_out->sizes() == q.sizes().slice(0, 3) &&
                          lse_out->is_contiguous() && lse_out->device() == q.device(),
                      "lse_out must be a contiguous float32 device tensor of shape ", tuple_of(q.sizes().slice(0, 3)));
    lse = static_cast<float*>(lse_out->data_ptr());
  }
  call_forward(p, q, k, v, z, lse, workspace);
  return z;
}

// ops.exact_attention
struct Exact : torch::autograd::Function<Exact> {
  static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& q, const at::Tensor& k,
                            const at::Tensor& v, const Opt& bias, const Opt& buckets, const Opt& lengths,
                            const Opt& key_mask, const Opt& q_start, double scale, bool causal) {
    const mra_exact_problem_t p = problem(q, k, v, scale, causal,
                                          {given(lengths), given(key_mask), given(q_start), given(bias), given(buckets)});
    const at::Tensor out = rows_like(q);
    const at::Tensor lse = at::empty(q.sizes().slice(0, 3), q.options().dtype(at::kFloat));
    call_forward(p, q, k, v, out, lse.data_ptr<float>(), std::nullopt);
    auto or_none = [](const Opt& t) { return t ? *t : at::Tensor(); };
    ctx->save_for_backward({q, k, v, out, lse, or_none(bias), or_none(buckets), or_none(lengths), or_none(key_mask),
                            or_none(q_start)});
    ctx->saved_data["scale"] = scale;
    ctx->saved_data["causal"] = causal;
    return out;
  }

  // the gradients, with everything allocated here (ops.exact_attention_backward)
  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx,
                                                 torch::autograd::variable_list grads) {
    check_capture(*torch::autograd::get_current_node(), kName);
    const auto t = ctx->get_saved_variables();
    const at::Tensor &q = t[0], &k = t[1], &v = t[2], &out = t[3], &lse = t[4];
    auto opt = [&](int i) { return t[i].defined() ? &t[i] : nullptr; };
    const mra_exact_problem_t p = problem(q, k, v, ctx->saved_data["scale"].toDouble(), ctx->saved_data["causal"].toBool(),
                                          {opt(7), opt(8), opt(9), opt(5), opt(6)});
    const at::Tensor dout = dense_rows(grads[0]) ? grads[0] : grads[0].contiguous();
    check_rows(out, q, q.sizes(), "out");
    check_rows(dout, q, q.sizes(), "dout");
    const c10::DeviceGuard guard(q.device());
    const at::Tensor dq = rows_like(q), dk = rows_like(k), dv = rows_like(v);
    // q, k, v, bias are edges 0 to 3
    const at::Tensor db = opt(5) && ctx->needs_input_grad(3) ? at::empty_like(t[5]) : at::Tensor();
    const size_t need = api.backward_ws(&p);
    at::Tensor ws;
    if (need) ws = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
    const mra_strided_t vq = view(q), vk = view(k), vv = view(v), vo = view(out), vg = view(dout), vdq = view(dq),
                        vdk = view(dk), vdv = view(dv);
    ok("mra_exact_backward",
       api.backward(&p, &vq, &vk, &vv, &vo, &vg, static_cast<const float*>(lse.data_ptr()), &vdq, &vdk, &vdv,
                    db.defined() ? db.data_ptr() : nullptr, need ? ws.data_ptr() : nullptr, need, stream_of(q)));
    const at::Tensor none;
    torch::autograd::variable_list result{dq, dk, dv, db, none, none, none, none, none, none};
    if (at::GradMode::is_enabled()) differentiated_once(result, {q, k, v, t[5], dout}, kName);
    return result;
  }
};

at::Tensor exact_attention(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, std::optional<double> scale,
                           bool causal, const Opt& lengths, const Opt& key_mask, const Opt& q_start, const Opt& bias,
                           const Opt& buckets) {
  return Exact::apply(q, k, v, bias, buckets, lengths, key_mask, q_start, scale_or(scale, q), causal);
}

}  // namespace

PYBIND11_MODULE(_binding_exact, m) {
  m.def("bind", [](const py::dict& a, py::object raiser) {
    bind_one(a, "mra_exact_forward_workspace_bytes", api.forward_ws);
    bind_one(a, "mra_exact_forward", api.forward);
    bind_one(a, "mra_exact_backward_workspace_bytes", api.backward_ws);
    bind_one(a, "mra_exact_backward", api.backward);
    status_error = std::move(raiser);
  });
  // of the backward that runs, or of the one that made z
  m.def("check_capture", [](const std::optional<at::Tensor>& z) {
    check_capture(z ? *z->grad_fn() : *torch::autograd::get_current_node(), kName);
  }, py::arg("z") = py::none());
  m.def("forward", torch::wrap_pybind_function_no_gil(forward));
  m.def("exact_attention", torch::wrap_pybind_function_no_gil(exact_attention));
}
