// The calls of libmra_layer that ops.py offers, marshalled in native code as those of exact
// attention are (exact_binding.cpp): the argument checks, the allocations, the library
// calls and the autograd node of rotary. The library is bound at run time (the addresses of the
// libmra_layer.so that ops.load_layer opened).
#include <cmath>
#include <limits>
#include <tuple>

#include "binding_rows.h"
#include "mra_layer.h"

namespace {

constexpr const char* kName = "rotary";

struct Api {
  decltype(&mra_rotary_forward) rotary_forward;
  decltype(&mra_rotary_backward_workspace_bytes) rotary_backward_ws;
  decltype(&mra_rotary_backward) rotary_backward;
  decltype(&mra_fp4_page_bytes) page_bytes;
  decltype(&mra_fp4_cache_write) cache_write;
  decltype(&mra_fp4_cache_read) cache_read;
  decltype(&mra_fp4_attention_workspace_bytes) attention_ws;
  decltype(&mra_fp4_attention) attention;
};
Api api{};

void check_sizes(at::IntArrayRef sizes) {
  for (const int64_t n : sizes) TORCH_CHECK_VALUE(n <= std::numeric_limits<int>::max(), "sizes must be below 2^31");
}

Opt opt(const at::Tensor& t) { return t.defined() ? Opt(t) : std::nullopt; }

// A result tensor of the caller's. It may be an input, and autograd may know it: what takes part in a graph is refused
// as by torch's own calls with given results, and what is written raises the tensor's version, so
// that a backward which kept the old values is refused there.
void check_graph(const at::Tensor& t, const char* name) {
  TORCH_CHECK_VALUE(!(at::GradMode::is_enabled() && t.requires_grad()), name,
                    " must not require a gradient: none would belong to its new values (torch.no_grad allows it)");
}

void check_result(const at::Tensor& t, const at::Tensor& ref, const char* name) {
  check_out(t, ref, name);
  check_graph(t, name);
}

void written(const at::Tensor& t) {
  if (t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

void written(const Opt& t) {
  if (t) written(*t);
}

// ---- rotary positions and head norms

// What a rotary call has beside its rows.
struct Turn {
  const at::Tensor *freqs, *positions, *q_weight, *k_weight;
  bool interleaved;
  double magnitude, eps;
};

void check_weight(const at::Tensor* w, const at::Tensor& ref, const char* name) {
  if (w == nullptr) return;
  TORCH_CHECK_VALUE((w->scalar_type() == ref.scalar_type() || w->scalar_type() == at::kFloat) && w->dim() == 1 &&
                        w->size(0) == ref.size(3) && w->is_contiguous() && w->device() == ref.device(),
                    name, " must be a contiguous tensor of shape ", tuple_of({ref.size(3)}), ", float32 or q's dtype,",
                    on(ref.device()));
}

// Every check of the tensors. q or k may be undefined (not both), of a backward that one result takes no part in.
mra_rotary_problem_t rotary_problem(const at::Tensor& q, const at::Tensor& k, const Turn& x) {
  const at::Tensor& ref = q.defined() ? q : k;
  for (const at::Tensor* t : {&q, &k}) {
    if (!t->defined()) continue;
    TORCH_CHECK_VALUE(t->is_cuda(), "tensors must be on a ROCm device");
    TORCH_CHECK_VALUE(t->dim() == 4, "q, k must have shape [B, heads, n, d]");
    check_sizes(t->sizes());
  }
  mra_rotary_problem_t p{};
  p.dtype = dtype_code(ref);
  const int64_t B = ref.size(0), n = ref.size(2), d = ref.size(3);
  const at::Device dev = ref.device();
  check_rows(ref, ref, ref.sizes(), q.defined() ? "q" : "k");
  if (q.defined() && k.defined()) {
    TORCH_CHECK_VALUE(k.size(0) == B && k.size(2) == n && k.size(3) == d, "k must share q's B, n and d");
    check_rows(k, ref, k.sizes(), "k");
  }
  if (x.freqs) {
    const at::Tensor& f = *x.freqs;
    TORCH_CHECK_VALUE(f.scalar_type() == at::kDouble && f.dim() == 1 && f.is_contiguous() && f.device() == dev &&
                          f.size(0) % 8 == 0 && 2 * f.size(0) <= d,
                      "freqs must be a contiguous float64 tensor of a multiple of 8, at most d / 2, entries", on(dev));
    p.freqs = f.size(0) ? static_cast<const double*>(f.data_ptr()) : nullptr;
    p.rot = (int)(2 * f.size(0));
  }
  if (x.positions) {
    const at::Tensor& t = *x.positions;
    TORCH_CHECK_VALUE(t.scalar_type() == at::kInt && (t.dim() == 1 || (t.dim() == 2 && t.size(0) == B)) &&
                          t.size(-1) == n && (n <= 1 || t.stride(-1) == 1) && t.device() == dev,
                      "positions must be an int32 tensor of shape ", tuple_of({n}), " or ", tuple_of({B, n}),
                      " with dense rows", on(dev));
    p.positions = static_cast<const int32_t*>(t.data_ptr());
    p.positions_stride = t.dim() == 2 && B > 1 ? t.stride(0) : 0;
  }
  check_weight(x.q_weight, ref, "q_weight");
  check_weight(x.k_weight, ref, "k_weight");
  if (x.q_weight && x.k_weight)
    TORCH_CHECK_VALUE(x.q_weight->scalar_type() == x.k_weight->scalar_type(), "q_weight and k_weight must share their dtype");
  if (const at::Tensor* w = x.q_weight ? x.q_weight : x.k_weight) p.weight_dtype = dtype_code(*w);
  p.q_weight = x.q_weight ? x.q_weight->data_ptr() : nullptr;
  p.k_weight = x.k_weight ? x.k_weight->data_ptr() : nullptr;
  p.B = (int)B;
  p.H = q.defined() ? (int)q.size(1) : 0;
  p.H_kv = k.defined() ? (int)k.size(1) : 0;
  p.n = (int)n;
  p.d = (int)d;
  p.interleaved = x.interleaved;
  p.magnitude = (float)x.magnitude;
  p.eps = (float)x.eps;
  return p;
}

mra_strided_t view_or_none(const at::Tensor& t) { return t.defined() ? view(t) : mra_strided_t{}; }

std::pair<at::Tensor, at::Tensor> turned(const at::Tensor& q, const at::Tensor& k, const Turn& x, const Opt& q_out,
                                         const Opt& k_out) {
  TORCH_CHECK_VALUE(k.defined() || !x.k_weight, "k_weight without k");
  TORCH_CHECK_VALUE(k.defined() || !k_out, "k_out without k");
  const mra_rotary_problem_t p = rotary_problem(q, k, x);
  if (q_out) check_result(*q_out, q, "q_out");
  if (k_out) check_result(*k_out, k, "k_out");
  const c10::DeviceGuard guard(q.device());
  const at::Tensor yq = q_out ? *q_out : rows_like(q), yk = k_out ? *k_out : k.defined() ? rows_like(k) : at::Tensor();
  const mra_strided_t vq = view(q), vk = view_or_none(k), wq = view(yq), wk = view_or_none(yk);
  ok("mra_rotary_forward", api.rotary_forward(&p, &vq, &vk, &wq, &wk, stream_of(q)));
  written(q_out);
  written(k_out);
  return {yq, yk};
}

// ops.rotary_forward
std::tuple<at::Tensor, Opt> rotary_forward(const at::Tensor& q, const Opt& k, const Opt& freqs, const Opt& positions,
                                           bool interleaved, double magnitude, const Opt& q_weight, const Opt& k_weight,
                                           double eps, const Opt& q_out, const Opt& k_out) {
  const auto y = turned(q, k ? *k : at::Tensor(),
                        {given(freqs), given(positions), given(q_weight), given(k_weight), interleaved, magnitude, eps},
                        q_out, k_out);
  return {y.first, opt(y.second)};
}

struct TurnedGrads {
  at::Tensor q, k, q_weight, k_weight;
};

// Gradients for those of the results that are defined.
TurnedGrads turned_back(const at::Tensor& gq, const at::Tensor& gk, const at::Tensor& q, const at::Tensor& k, Turn x,
                        bool need_qw, bool need_kw, const Opt& dq, const Opt& dk) {
  TORCH_CHECK_VALUE(gq.defined() || gk.defined(), "a gradient of either result is needed");
  if (!gq.defined()) x.q_weight = nullptr;
  if (!gk.defined()) x.k_weight = nullptr;
  const mra_rotary_problem_t p = rotary_problem(gq, gk, x);
  auto check_input = [](const at::Tensor& t, const at::Tensor& g, const at::Tensor* w, const char* name) {
    if (w == nullptr) return;
    TORCH_CHECK_VALUE(t.defined(), name, " is needed with its weight");
    check_rows(t, g, g.sizes(), name);
  };
  check_input(q, gq, x.q_weight, "q");
  check_input(k, gk, x.k_weight, "k");
  if (dq) check_result(*dq, gq, "dq");
  if (dk) check_result(*dk, gk, "dk");
  const at::Tensor& ref = gq.defined() ? gq : gk;
  const c10::DeviceGuard guard(ref.device());
  TurnedGrads r;
  if (gq.defined()) r.q = dq ? *dq : rows_like(x.q_weight ? q : gq);
  if (gk.defined()) r.k = dk ? *dk : rows_like(x.k_weight ? k : gk);
  if (x.q_weight && need_qw) r.q_weight = at::empty_like(*x.q_weight);
  if (x.k_weight && need_kw) r.k_weight = at::empty_like(*x.k_weight);
  at::Tensor ws;
  const size_t need = r.q_weight.defined() || r.k_weight.defined() ? api.rotary_backward_ws(&p) : 0;
  if (need) ws = at::empty({(int64_t)need}, ref.options().dtype(at::kByte));
  const mra_strided_t vq = x.q_weight ? view(q) : mra_strided_t{}, vk = x.k_weight ? view(k) : mra_strided_t{},
                      vgq = view_or_none(gq), vgk = view_or_none(gk), vdq = view_or_none(r.q), vdk = view_or_none(r.k);
  ok("mra_rotary_backward",
     api.rotary_backward(&p, &vq, &vk, &vgq, &vgk, &vdq, &vdk, r.q_weight.defined() ? r.q_weight.data_ptr() : nullptr,
                         r.k_weight.defined() ? r.k_weight.data_ptr() : nullptr, need ? ws.data_ptr() : nullptr, need,
                         stream_of(ref)));
  written(dq);
  written(dk);
  return r;
}

// ops.rotary_backward
std::tuple<Opt, Opt, Opt, Opt> rotary_backward(const Opt& dq_out, const Opt& dk_out, const Opt& q, const Opt& k,
                                               const Opt& freqs, const Opt& positions, bool interleaved,
                                               double magnitude, const Opt& q_weight, const Opt& k_weight, double eps,
                                               const Opt& dq, const Opt& dk) {
  auto plain = [](const Opt& t) { return t ? *t : at::Tensor(); };
  TORCH_CHECK_VALUE((dq_out || !dq) && (dk_out || !dk), "dq and dk go with dq_out and dk_out");
  const TurnedGrads g = turned_back(
      plain(dq_out), plain(dk_out), plain(q), plain(k),
      {given(freqs), given(positions), given(q_weight), given(k_weight), interleaved, magnitude, eps}, true, true, dq, dk);
  return {opt(g.q), opt(g.k), opt(g.q_weight), opt(g.k_weight)};
}

// ops.rotary; q and k are kept for the backward where they have a weight
struct Rotary : torch::autograd::Function<Rotary> {
  static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& q, const Opt& k,
                                                const Opt& q_weight, const Opt& k_weight, const Opt& freqs,
                                                const Opt& positions, bool interleaved, double magnitude, double eps) {
    const auto y = turned(q, k ? *k : at::Tensor(),
                          {given(freqs), given(positions), given(q_weight), given(k_weight), interleaved, magnitude, eps},
                          std::nullopt, std::nullopt);
    ctx->set_materialize_grads(false);
    auto or_none = [](const Opt& t) { return t ? *t : at::Tensor(); };
    ctx->save_for_backward({q_weight ? q : at::Tensor(), k_weight ? *k : at::Tensor(), or_none(q_weight),
                            or_none(k_weight), or_none(freqs), or_none(positions)});
    ctx->saved_data["interleaved"] = interleaved;
    ctx->saved_data["magnitude"] = magnitude;
    ctx->saved_data["eps"] = eps;
    torch::autograd::variable_list r{y.first};
    if (y.second.defined()) r.push_back(y.second);
    return r;
  }

  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx,
                                                 torch::autograd::variable_list grads) {
    check_capture(*torch::autograd::get_current_node(), kName);
    const auto t = ctx->get_saved_variables();
    torch::autograd::variable_list result(9);
    // the edges are q, k and the weights that were given, in this order
    size_t edge = 0;
    const bool has_k = grads.size() > 1;
    const bool need_q = ctx->needs_input_grad(edge++), need_k = has_k && ctx->needs_input_grad(edge++);
    const bool need_qw = t[2].defined() && ctx->needs_input_grad(edge++),
               need_kw = t[3].defined() && ctx->needs_input_grad(edge++);
    auto rows = [](const at::Tensor& g) { return !g.defined() || dense_rows(g) ? g : g.contiguous(); };
    const at::Tensor none;
    const at::Tensor gq = need_q || need_qw ? rows(grads[0]) : none,
                     gk = need_k || need_kw ? rows(has_k ? grads[1] : none) : none;
    if (!gq.defined() && !gk.defined()) return result;
    auto at = [&](int i) { return t[i].defined() ? &t[i] : nullptr; };
    const TurnedGrads g = turned_back(gq, gk, t[0], t[1],
                                      {at(4), at(5), at(2), at(3), ctx->saved_data["interleaved"].toBool(),
                                       ctx->saved_data["magnitude"].toDouble(), ctx->saved_data["eps"].toDouble()},
                                      need_qw, need_kw, std::nullopt, std::nullopt);
    result[0] = g.q;
    result[1] = g.k;
    result[2] = g.q_weight;
    result[3] = g.k_weight;
    if (at::GradMode::is_enabled()) {
      // a result's gradient that has a graph last, if any
      const bool first = gq.defined() && (gq.requires_grad() || !gk.defined());
      torch::autograd::variable_list of{t[0], t[1], t[2], t[3]};
      for (const at::Tensor& x : {first ? gk : gq, first ? gq : gk})
        if (x.defined()) of.push_back(x);
      differentiated_once(result, of, kName);
    }
    return result;
  }
};

std::tuple<at::Tensor, Opt> rotary(const at::Tensor& q, const Opt& k, const Opt& freqs, const Opt& positions,
                                   bool interleaved, double magnitude, const Opt& q_weight, const Opt& k_weight,
                                   double eps) {
  const auto y = Rotary::apply(q, k, q_weight, k_weight, freqs, positions, interleaved, magnitude, eps);
  return {y[0], y.size() > 1 ? Opt(y[1]) : std::nullopt};
}

// ---- the cache

mra_fp4_cache_t cache_of(const at::Tensor& data, int64_t page_size, int64_t d, const at::Tensor& table) {
  TORCH_CHECK_VALUE(data.is_cuda(), "tensors must be on a ROCm device");
  check_sizes({page_size, d});
  TORCH_CHECK_VALUE(data.scalar_type() == at::kByte && data.dim() == 3 && data.is_contiguous() &&
                        data.size(2) == (int64_t)api.page_bytes((int)page_size, (int)d),
                    "the cache must be a contiguous uint8 tensor [pages, H_kv, page bytes] (see fp4_cache)");
  TORCH_CHECK_VALUE(table.scalar_type() == at::kInt && table.dim() == 2 && table.is_contiguous() &&
                        table.device() == data.device(),
                    "table must be a contiguous int32 tensor [B, pages of a sequence]", on(data.device()));
  check_sizes(data.sizes());
  check_sizes(table.sizes());
  mra_fp4_cache_t c{};
  c.pages = (int)data.size(0);
  c.H_kv = (int)data.size(1);
  c.d = (int)d;
  c.page_size = (int)page_size;
  c.data = data.data_ptr();
  c.table = static_cast<const int32_t*>(table.data_ptr());
  c.B = (int)table.size(0);
  c.max_pages = (int)table.size(1);
  return c;
}

const int32_t* ints(const Opt& t, int64_t B, const char* name, const at::Device& dev) {
  if (!given(t)) return nullptr;
  check_int(*t, {B}, name, dev);
  return static_cast<const int32_t*>(t->data_ptr());
}

// ops.fp4_cache_write
void cache_write(const at::Tensor& data, int64_t page_size, int64_t d, const at::Tensor& k, const at::Tensor& v,
                 const at::Tensor& table, const Opt& starts, const Opt& counts) {
  const mra_fp4_cache_t c = cache_of(data, page_size, d, table);
  TORCH_CHECK_VALUE(k.is_cuda() && v.is_cuda(), "tensors must be on a ROCm device");
  TORCH_CHECK_VALUE(k.dim() == 4 && k.size(0) == c.B && k.size(1) == c.H_kv && k.size(3) == d && k.sizes() == v.sizes() &&
                        k.device() == data.device(),
                    "k, v must share shape [B, H_kv, n, d] with the table's B and the cache's H_kv and d", on(data.device()));
  const mra_dtype_t dtype = dtype_code(k);
  check_sizes(k.sizes());
  check_rows(k, k, k.sizes(), "k");
  check_rows(v, k, k.sizes(), "v");
  const int32_t *s = ints(starts, c.B, "starts", data.device()), *n = ints(counts, c.B, "counts", data.device());
  const c10::DeviceGuard guard(data.device());
  const mra_strided_t vk = view(k), vv = view(v);
  ok("mra_fp4_cache_write", api.cache_write(&c, &vk, &vv, (int)k.size(2), dtype, s, n, stream_of(data)));
  written(data);
}

// ops.fp4_cache_read
std::tuple<at::Tensor, at::Tensor> cache_read(const at::Tensor& data, int64_t page_size, int64_t d,
                                              const at::Tensor& table, int64_t n, const Opt& starts, const Opt& counts,
                                              at::ScalarType type, const Opt& k_out, const Opt& v_out) {
  const mra_fp4_cache_t c = cache_of(data, page_size, d, table);
  TORCH_CHECK_VALUE(n >= 0, "n must not be negative");
  check_sizes({n});
  const c10::DeviceGuard guard(data.device());
  const std::vector<int64_t> shape{c.B, c.H_kv, n, d};
  at::Tensor out[2];
  const Opt* to[2] = {&k_out, &v_out};
  for (int i = 0; i < 2; ++i) {
    if (given(*to[i])) {
      out[i] = **to[i];
      TORCH_CHECK_VALUE(out[i].sizes() == shape && out[i].scalar_type() == type && out[i].device() == data.device(),
                        i ? "v_out" : "k_out", " must be a tensor of dtype and shape ", tuple_of(shape),
                        on(data.device()));
      check_result(out[i], out[i], i ? "v_out" : "k_out");
    } else {
      out[i] = at::empty(shape, data.options().dtype(type));
    }
  }
  const mra_dtype_t dtype = dtype_code(out[0]);
  const int32_t *s = ints(starts, c.B, "starts", data.device()), *m = ints(counts, c.B, "counts", data.device());
  const mra_strided_t vk = view(out[0]), vv = view(out[1]);
  ok("mra_fp4_cache_read", api.cache_read(&c, &vk, &vv, (int)n, dtype, s, m, stream_of(data)));
  written(k_out);
  written(v_out);
  return {out[0], out[1]};
}

mra_fp4_attention_t attention_problem(const mra_fp4_cache_t& c, const at::Tensor& data, const at::Tensor& q,
                                      const at::Tensor& lengths, const std::optional<double>& scale, bool causal,
                                      const Opt& q_start) {
  TORCH_CHECK_VALUE(q.is_cuda(), "tensors must be on a ROCm device");
  TORCH_CHECK_VALUE(q.dim() == 4 && q.size(0) == c.B && q.size(3) == c.d && q.device() == data.device() &&
                        (c.H_kv ? q.size(1) % c.H_kv : q.size(1)) == 0,
                    "q must have shape [B, H, n_q, d] with the table's B, the cache's d and H a multiple of its H_kv",
                    on(data.device()));
  mra_fp4_attention_t p{};
  p.dtype = dtype_code(q);
  check_sizes(q.sizes());
  check_rows(q, q, q.sizes(), "q");
  check_int(lengths, {c.B}, "lengths", data.device());
  p.H = (int)q.size(1);
  p.n_q = (int)q.size(2);
  p.scale = (float)(scale ? *scale : 1.0 / std::sqrt((double)c.d));
  p.causal = causal;
  p.lengths = static_cast<const int32_t*>(lengths.data_ptr());
  p.q_start = ints(q_start, c.B, "q_start", data.device());
  return p;
}

// ops.fp4_attention_workspace_bytes
size_t attention_workspace(const at::Tensor& data, int64_t page_size, int64_t d, const at::Tensor& q,
                           const at::Tensor& table, const at::Tensor& lengths) {
  const mra_fp4_cache_t c = cache_of(data, page_size, d, table);
  const mra_fp4_attention_t p = attention_problem(c, data, q, lengths, std::nullopt, false, std::nullopt);
  return api.attention_ws(&c, &p);
}

// ops.fp4_cache_attention
at::Tensor attention(const at::Tensor& data, int64_t page_size, int64_t d, const at::Tensor& q, const at::Tensor& table,
                     const at::Tensor& lengths, std::optional<double> scale, bool causal, const Opt& q_start,
                     const Opt& out, const Opt& lse_out, const Opt& workspace) {
  const mra_fp4_cache_t c = cache_of(data, page_size, d, table);
  const mra_fp4_attention_t p = attention_problem(c, data, q, lengths, scale, causal, q_start);
  if (out) check_result(*out, q, "out");
  const c10::DeviceGuard guard(q.device());
  const at::Tensor z = out ? *out : rows_like(q);
  float* lse = nullptr;
  if (lse_out) {
    TORCH_CHECK_VALUE(lse_out->scalar_type() == at::kFloat && lse_out->sizes() == q.sizes().slice(0, 3) &&
                          lse_out->is_contiguous() && lse_out->device() == q.device(),
                      "lse_out must be a contiguous float32 device tensor of shape ", tuple_of(q.sizes().slice(0, 3)));
    check_graph(*lse_out, "lse_out");
    lse = static_cast<float*>(lse_out->data_ptr());
  }
  at::Tensor ws;
  if (given(workspace)) {
    TORCH_CHECK_VALUE(workspace->device() == q.device() && workspace->is_contiguous(),
                      "workspace must be a contiguous tensor", on(q.device()));
    ws = *workspace;
  } else if (const size_t need = api.attention_ws(&c, &p)) {
    ws = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
  }
  const mra_strided_t vq = view(q), vo = view(z);
  ok("mra_fp4_attention", api.attention(&c, &p, &vq, &vo, lse, ws.defined() ? ws.data_ptr() : nullptr,
                                        ws.defined() ? ws.nbytes() : 0, stream_of(q)));
  written(out);
  written(lse_out);
  return z;
}

}  // namespace

PYBIND11_MODULE(_binding_layer, m) {
  m.def("bind", [](const py::dict& a, py::object raiser) {
    bind_one(a, "mra_rotary_forward", api.rotary_forward);
    bind_one(a, "mra_rotary_backward_workspace_bytes", api.rotary_backward_ws);
    bind_one(a, "mra_rotary_backward", api.rotary_backward);
    bind_one(a, "mra_fp4_page_bytes", api.page_bytes);
    bind_one(a, "mra_fp4_cache_write", api.cache_write);
    bind_one(a, "mra_fp4_cache_read", api.cache_read);
    bind_one(a, "mra_fp4_attention_workspace_bytes", api.attention_ws);
    bind_one(a, "mra_fp4_attention", api.attention);
    status_error = std::move(raiser);
  });
  // of the backward that runs, or of the one that made z
  m.def("check_capture", [](const std::optional<at::Tensor>& z) {
    check_capture(z ? *z->grad_fn() : *torch::autograd::get_current_node(), kName);
  }, py::arg("z") = py::none());
  m.def("rotary_forward", torch::wrap_pybind_function_no_gil(rotary_forward));
  m.def("rotary_backward", torch::wrap_pybind_function_no_gil(rotary_backward));
  m.def("rotary", torch::wrap_pybind_function_no_gil(rotary));
  m.def("cache_write", torch::wrap_pybind_function_no_gil(cache_write));
  m.def("cache_read", torch::wrap_pybind_function_no_gil(cache_read));
  m.def("attention", torch::wrap_pybind_function_no_gil(attention));
  m.def("attention_workspace", torch::wrap_pybind_function_no_gil(attention_workspace));
}
