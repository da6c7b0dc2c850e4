// What the marshalling of the training-step operators for torch tensors shares.
#pragma once
#include <ATen/cuda/CUDAContext.h>
#include <c10/cuda/CUDAGuard.h>
#include <torch/extension.h>

#include <initializer_list>
#include <optional>

#include "ones_train.h"

namespace {

using at::Tensor;
using MaybeTensor = std::optional<Tensor>;

inline int kind_of(at::ScalarType t) {
    return t == at::kFloat ? ONES_F32 : t == at::kBFloat16 ? ONES_BF16 : t == at::kHalf ? ONES_F16 : -1;
}

// Results have no graph: who asks for a gradient (or sends a tangent) through here would get none, without a word.
inline void no_graph(std::initializer_list<const Tensor*> ts) {
    for (const Tensor* t : ts)
        TORCH_CHECK_VALUE(!(t->requires_grad() && at::GradMode::is_enabled()) && !t->_fw_grad(0).defined(),
                          "an input requires a gradient, but this function is not differentiable: use its form with `_autograd` "
                          "(layer_norm, linear_cross_entropy, qk_norm, attention), or call it under torch.no_grad()");
}
inline const Tensor* given(const MaybeTensor& t, const Tensor& other) { return t ? &*t : &other; }

inline void* ptr(const MaybeTensor& t) { return t ? t->data_ptr() : nullptr; }
inline void* stream() { return at::cuda::getCurrentCUDAStream().stream(); }
inline Tensor bytes(size_t n, const Tensor& like) { return at::empty({(int64_t)n}, like.options().dtype(at::kByte)); }
inline Tensor fresh(at::IntArrayRef shape, const Tensor& like, at::ScalarType type) { return at::empty(shape, like.options().dtype(type)); }

inline py::object result(int rc, py::object v) { return rc ? py::int_(rc) : std::move(v); }

}  // namespace

void add_attention(py::module_& m);  // the functions of ones_attention.h
