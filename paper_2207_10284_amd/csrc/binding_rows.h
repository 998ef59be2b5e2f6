// What the bindings of strided tensors [B, heads, n, d] share (mra_exact.h, mra_layer.h): their
// checks, and those of an autograd node's backward.
#pragma once

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/accumulate_grad.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>

#include "binding_common.h"
#include "mra_exact.h"

namespace {

using Opt = std::optional<at::Tensor>;

inline const at::Tensor* given(const Opt& t) { return t && t->defined() ? &*t : nullptr; }

inline std::string on(const at::Device& d) { return " on " + d.str(); }

inline mra_strided_t view(const at::Tensor& t) {
  auto st = [&](int i) { return t.size(i) > 1 ? t.stride(i) : 0; };
  return {t.data_ptr(), st(0), st(1), st(2)};
}

inline bool dense_rows(const at::Tensor& t) {
  if (t.numel() == 0) return true;
  const int64_t per = 16 / t.element_size();
  const mra_strided_t v = view(t);
  return t.stride(3) == 1 && reinterpret_cast<uintptr_t>(v.data) % 16 == 0 && v.stride_b % per == 0 &&
         v.stride_h % per == 0 && v.stride_n % per == 0;
}

inline void check_rows(const at::Tensor& t, const at::Tensor& ref, at::IntArrayRef shape, const char* name) {
  TORCH_CHECK_VALUE(t.is_cuda(), "tensors must be on a ROCm device");
  TORCH_CHECK_VALUE(t.sizes() == shape && t.scalar_type() == ref.scalar_type() && t.device() == ref.device(), name,
                    " must be a torch.", ref.scalar_type() == at::kFloat ? "float32" : "bfloat16", " tensor of shape ",
                    tuple_of(shape), on(ref.device()));
  TORCH_CHECK_VALUE(dense_rows(t), name, " must have dense rows, 16-byte aligned");
}

// A result tensor of the caller's: like ref, and no two of its rows the same memory.
inline void check_out(const at::Tensor& t, const at::Tensor& ref, const char* name) {
  check_rows(t, ref, ref.sizes(), name);
  const mra_strided_t v = view(t);
  TORCH_CHECK_VALUE(t.numel() == 0 || ((t.size(0) == 1 || v.stride_b) && (t.size(1) == 1 || v.stride_h) &&
                                       (t.size(2) == 1 || v.stride_n)),
                    name, " must not be broadcast");
}

inline at::Tensor rows_like(const at::Tensor& t) {
  at::Tensor o = at::empty_like(t);
  return dense_rows(o) ? o : at::empty(t.sizes(), t.options());
}

inline void check_int(const at::Tensor& t, at::IntArrayRef shape, const char* name, const at::Device& dev) {
  TORCH_CHECK_VALUE(t.scalar_type() == at::kInt && t.sizes() == shape && t.is_contiguous() && t.device() == dev, name,
                    " must be a contiguous int32 tensor of shape ", tuple_of(shape), on(dev));
}

// A leaf's accumulator belongs to the stream on which the leaf entered the oldest graph that is
// alive: of eager work, the default stream. The engine would have it wait for the stream of a backward that a HIP
// graph captures, which the default stream cannot: the capture fails in the engine, where that can end
// the process. So such a backward is refused before it enqueues anything. (Leaves further up are not in sight.)
inline void check_capture(const torch::autograd::Node& node, const char* name) {
  for (size_t i = 0; i < node.num_outputs(); ++i) {
    const torch::autograd::Edge& e = node.next_edge(i);
    if (!node.task_should_compute_output(i)) continue;   // of a backward for other inputs
    if (dynamic_cast<torch::autograd::AccumulateGrad*>(e.function.get()) == nullptr) continue;
    const auto stream = e.function->stream();
    // 0: the default stream, which does not capture itself
    if (!stream || stream->id() != 0 || c10::hip::getCurrentHIPStream(stream->device_index()).id() == 0) continue;
    TORCH_CHECK(c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None,
                "a graph captures the backward of ", name, " while an eager graph of one of its inputs is alive, "
                "whose gradient belongs to the default stream; drop the outputs of that graph first");
  }
}

// Gradients taken with a graph of their own, which does not reach through them: where the output's
// gradient (the last of `of`) has one, a node whose backward raises stands between them and
// what they depend on; where it is a constant they are constants too, and a warning says so.
inline void differentiated_once(torch::autograd::variable_list& grads, const torch::autograd::variable_list& of,
                                const char* name) {
  if (!of.back().requires_grad()) {
    TORCH_WARN("the gradients of ", name, " are not differentiable: these are constants of the graph");
    return;
  }
  const auto error = std::make_shared<torch::autograd::Error>(
      std::string("the gradients of ") + name + " are not differentiable: trying to differentiate twice",
      torch::autograd::collect_next_edges(of));
  for (at::Tensor& t : grads)
    if (t.defined()) torch::autograd::set_history(t, error);
}

}  // namespace
