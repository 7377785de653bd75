// What the bindings to torch tensors (losses_binding.cpp, rollouts_binding.cpp) share: one module, _losses.so.
#pragma once

#include <torch/extension.h>

#include <optional>
#include <string>
#include <tuple>

#include "../../include/lbfgsb.h"

namespace py = pybind11;
using at::Tensor;
using Maybe = std::optional<Tensor>;

void add_rollouts(py::module_& m);

inline int type_code(at::ScalarType d) {
    return d == at::kFloat ? LBFGSB_F32 : (d == at::kBFloat16 ? (int)LBFGSB_BF16 : (d == at::kHalf ? (int)LBFGSB_F16 : -1));
}
inline int logit_type(const Tensor& t, const char* name) {
    const int type = type_code(t.scalar_type());
    if (type < 0 || !t.is_cuda() || t.dim() != 2 || (t.stride(1) != 1 && t.size(1) != 1))
        throw py::type_error(std::string(name) + " must be a 2-d float32/bfloat16/float16 CUDA tensor with unit column stride");
    return type;
}

inline int64_t row_stride(const Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }

// the address of a contiguous 1-d tensor of `numel` entries
template <typename T = float>
T* vec(const Tensor& t, const char* name, int64_t numel, const at::Device& dev, at::ScalarType type = at::kFloat) {
    if (t.scalar_type() != type || t.device() != dev || !t.is_contiguous())
        throw py::type_error(std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor on " + dev.str());
    if (t.dim() != 1 || t.size(0) != numel)
        throw py::value_error(std::string(name) + " must be 1-d with " + std::to_string(numel) + " entries, got " + std::to_string(t.numel()) +
                              " in " + std::to_string(t.dim()) + " dimensions");
    return (T*)t.data_ptr();
}
template <typename T = float>
T* maybe(const Maybe& t, const char* name, int64_t numel, const at::Device& dev) {
    return t ? vec<T>(*t, name, numel, dev) : nullptr;
}
inline void* address(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
inline size_t bytes(const Tensor& t) { return t.defined() ? (size_t)t.numel() : 0; }
// After a call that went well: torch learns that the caller's tensor has been written to, so that a way back which kept it is
// refused, as after any operation in place.  (Tensors of inference mode have no count and nobody's way back keeps them.)
inline void written(const Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
