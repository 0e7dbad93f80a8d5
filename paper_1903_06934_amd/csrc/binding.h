// What the Python bindings of include/mitrain.h (binding.cpp) and include/mistep.h
// (binding_step.cpp) share, two sources of one module.
#pragma once

#include <stdint.h>
#include <optional>
#include <string>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/utils/pybind.h>

#include "mitrain.h"

namespace binding {

namespace py = pybind11;
using at::Tensor;
using Maybe = std::optional<Tensor>;

void bind_step(py::module_ &m);

inline py::object *raise_status;  // raises the error of (status, function)

inline void call(int status, const char *name)
{
    if (status != MICONV_OK)
        (*raise_status)(status, name);
}

[[noreturn]] inline void refuse(const char *name, const std::string &what)
{
    throw py::value_error(std::string(name) + what);
}

// ------------------------------------------------------------------- tensors
inline int type_of(const Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return MITRAIN_F32;
    case at::kBFloat16: return MITRAIN_BF16;
    case at::kHalf: return MITRAIN_F16;
    default: return -1;
    }
}

inline bool here(const Tensor &t)
{
    return t.is_cuda() && t.get_device() == c10::hip::current_device();
}

struct Rows {
    int64_t rows, cols, ld;
};

// A tensor of rows: its rows' elements side by side in the last dimension, one
// stride over the dimensions before it.
inline Rows rows_of(const Tensor &t, const char *name)
{
    const int64_t dims = t.dim();
    if (!dims)
        refuse(name, " must have at least one dimension");
    Rows r{1, t.size(dims - 1), 0};
    for (int64_t i = 0; i < dims - 1; i++)
        r.rows *= t.size(i);
    if (r.cols > 1 && t.stride(dims - 1) != 1)
        refuse(name, ": the elements of a row must lie side by side");
    r.ld = r.cols;
    if (r.rows > 1) {
        int64_t span = -1;  // the stride that the next outer dimension needs
        for (int64_t i = dims - 2; i >= 0; i--) {
            if (t.size(i) == 1)
                continue;
            if (span < 0)
                r.ld = span = t.stride(i);
            else if (t.stride(i) != span)
                refuse(name, ": one stride must cover the rows");
            span *= t.size(i);
        }
        if (r.ld < r.cols)
            refuse(name, ": rows must not overlap");
    }
    return r;
}

inline int float_rows(const Tensor &t, const char *name, Rows *r)
{
    const int type = type_of(t);
    if (type < 0 || !here(t))
        refuse(name, " must be a float32, bfloat16 or float16 tensor on the current device");
    *r = rows_of(t, name);
    return type;
}

// The row stride of t, which has x's type, rows and columns.
inline int64_t like(const Tensor &t, const char *name, const Tensor &x, const Rows &rx)
{
    if (t.scalar_type() != x.scalar_type() || !here(t))
        refuse(name, " must be of the input's type, on the current device");
    const Rows r = rows_of(t, name);
    if (r.rows != rx.rows || r.cols != rx.cols)
        refuse(name, " must have the input's rows and columns");
    return r.ld;
}

template <class T = void>
T *vector(const Maybe &m, const char *name, int64_t n, at::ScalarType type)
{
    if (!m)
        return nullptr;
    if (m->numel() != n || m->scalar_type() != type || !m->is_contiguous() || !here(*m))
        refuse(name, " must be a contiguous tensor of " + std::to_string(n) + " elements of " +
                         c10::toString(type) + " on the current device");
    return (T *)m->data_ptr();
}

inline Tensor empty(at::IntArrayRef sizes, const Tensor &x, at::ScalarType type)
{
    return at::empty(sizes, x.options().dtype(type));
}

// A tensor that a call has written, as torch's own calls in place count it: one
// that autograd has saved before is reported when it is used.
inline void written(const Tensor &t)
{
    if (!t.is_inference())
        t.unsafeGetTensorImpl()->bump_version();
}

inline void written(const Maybe &m)
{
    if (m)
        written(*m);
}

// Small results of one type (floats, if it is not said) side by side in one buffer: its
// allocation takes the host longer than the views.  Only of one type: tensors of several
// types in one storage cannot be saved together.
struct Results {
    Tensor floats;
    int64_t used = 0;

    Results(int64_t n, const Tensor &x, at::ScalarType type = at::kFloat)
        : floats(empty({n}, x, type))
    {
    }

    Tensor next(at::IntArrayRef sizes)
    {
        Tensor t = at::detail::make_tensor<c10::TensorImpl>(
            c10::Storage(floats.storage()), floats.key_set(), floats.dtype());
        t.unsafeGetTensorImpl()->set_storage_offset(used);
        t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
        used += t.numel();
        return t;
    }
};

// The caller's workspace, or one of the size that is needed.
struct Workspace {
    Maybe own;
    void *p = nullptr;
    size_t bytes = 0;

    Workspace(const Maybe &given, size_t need, at::Device device)
    {
        if (!given && need)
            own = at::empty({(int64_t)need}, at::TensorOptions(device).dtype(at::kByte));
        const Maybe &w = given ? given : own;
        if (w) {
            if (!w->is_contiguous() || !here(*w))
                refuse("ws", " must be a contiguous tensor on the current device");
            p = w->data_ptr();
            bytes = w->nbytes();
        }
    }
};

inline Maybe workspace(size_t need, at::Device device)
{
    if (!need)
        return std::nullopt;
    return at::empty({(int64_t)need}, at::TensorOptions(device).dtype(at::kByte));
}

inline hipStream_t stream() { return c10::hip::getCurrentHIPStream().stream(); }

}  // namespace binding
