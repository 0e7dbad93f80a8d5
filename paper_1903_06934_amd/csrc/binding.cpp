// Python binding of include/mitrain.h: argument marshalling only, on torch's
// tensors and current stream, in C++ because the smallest calls' kernels take
// less time than a Python function's checks (four rows of layer norm: 4 us of
// kernel behind 20 us of ctypes marshalling), and lists of some hundred
// gradients far less (288 tensors: 0.1 ms behind 0.3 ms).  mitrain.py has the
// documentation; it hands over the library's functions once (load).
#include <stdint.h>
#include <string.h>
#include <algorithm>
#include <array>
#include <optional>
#include <string>
#include <tuple>
#include <vector>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include "mitrain.h"

namespace py = pybind11;
using at::Tensor;
using Maybe = std::optional<Tensor>;

namespace {

struct Library {
    decltype(&::layernorm_fwd_workspace_size) layernorm_fwd_ws;
    decltype(&::layernorm_bwd_workspace_size) layernorm_bwd_ws;
    decltype(&::layernorm_fwd) layernorm_fwd;
    decltype(&::layernorm_bwd) layernorm_bwd;
    decltype(&::logprob_fwd_workspace_size) logprob_fwd_ws;
    decltype(&::logprob_fwd) logprob_fwd;
    decltype(&::logprob_bwd) logprob_bwd;
    decltype(&::grad_workspace_size) grad_ws;
    decltype(&::grad_norm) grad_norm;
    decltype(&::grad_clip) grad_clip;
} lib;
py::object *raise_status;  // raises the error of (status, function)

void load(const std::array<uintptr_t, 10> &functions, py::object raise)
{
    memcpy(&lib, functions.data(), sizeof(lib));
    static_assert(sizeof(lib) == 10 * sizeof(uintptr_t), "one address each");
    raise_status = new py::object(std::move(raise));
}

void call(int status, const char *name)
{
    if (status != MICONV_OK)
        (*raise_status)(status, name);
}

[[noreturn]] void refuse(const char *name, const std::string &what)
{
    throw py::value_error(std::string(name) + what);
}

// ------------------------------------------------------------------- tensors
int type_of(const Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return MITRAIN_F32;
    case at::kBFloat16: return MITRAIN_BF16;
    case at::kHalf: return MITRAIN_F16;
    default: return -1;
    }
}

bool here(const Tensor &t)
{
    return t.is_cuda() && t.get_device() == c10::hip::current_device();
}

struct Rows {
    int64_t rows, cols, ld;
};

// A tensor of rows: its rows' elements side by side in the last dimension, one
// stride over the dimensions before it.
Rows rows_of(const Tensor &t, const char *name)
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

int float_rows(const Tensor &t, const char *name, Rows *r)
{
    const int type = type_of(t);
    if (type < 0 || !here(t))
        refuse(name, " must be a float32, bfloat16 or float16 tensor on the current device");
    *r = rows_of(t, name);
    return type;
}

// The row stride of t, which has x's type, rows and columns.
int64_t like(const Tensor &t, const char *name, const Tensor &x, const Rows &rx)
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

Tensor empty(at::IntArrayRef sizes, const Tensor &x, at::ScalarType type)
{
    return at::empty(sizes, x.options().dtype(type));
}

// A tensor that a call has written, as torch's own calls in place count it: one
// that autograd has saved before is reported when it is used.
void written(const Tensor &t)
{
    if (!t.is_inference())
        t.unsafeGetTensorImpl()->bump_version();
}

void written(const Maybe &m)
{
    if (m)
        written(*m);
}

// Small float results side by side in one buffer: its allocation takes the host
// longer than the views.  Only floats: tensors of several types in one storage
// cannot be saved together.
struct Results {
    Tensor floats;
    int64_t used = 0;

    Results(int64_t n, const Tensor &x) : floats(empty({n}, x, at::kFloat)) {}

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

Maybe workspace(size_t need, at::Device device)
{
    if (!need)
        return std::nullopt;
    return at::empty({(int64_t)need}, at::TensorOptions(device).dtype(at::kByte));
}

hipStream_t stream() { return c10::hip::getCurrentHIPStream().stream(); }

// ---------------------------------------------------------------- layer norm
Maybe layernorm_workspace(bool backward, const Tensor &x)
{
    Rows r;
    const int type = float_rows(x, "x", &r);
    return workspace((backward ? lib.layernorm_bwd_ws : lib.layernorm_fwd_ws)(type, r.rows, r.cols),
                     x.device());
}

std::tuple<Tensor, Tensor, Tensor> layernorm_forward(const Tensor &x, const Maybe &w,
                                                     const Maybe &b, double eps, const Maybe &y_,
                                                     const Maybe &mean_, const Maybe &rstd_,
                                                     const Maybe &ws)
{
    Rows r;
    const int type = float_rows(x, "x", &r);
    const at::ScalarType wt = w ? w->scalar_type() : b ? b->scalar_type() : x.scalar_type();
    const void *wp = vector(w, "w", r.cols, wt), *bp = vector(b, "b", r.cols, wt);
    const Tensor y = y_ ? *y_ : empty(x.sizes(), x, x.scalar_type());
    const int64_t ldy = like(y, "y", x, r);
    Tensor mean, rstd;
    if (mean_ && rstd_) {
        mean = *mean_;
        rstd = *rstd_;
    } else {
        Results out(2 * r.rows, x);
        mean = mean_ ? *mean_ : out.next({r.rows});
        rstd = rstd_ ? *rstd_ : out.next({r.rows});
    }
    const Workspace s(ws, lib.layernorm_fwd_ws(type, r.rows, r.cols), x.device());
    call(lib.layernorm_fwd(type, w ? type_of(*w) : b ? type_of(*b) : type, r.rows, r.cols,
                           x.data_ptr(), r.ld, wp, bp, (float)eps, y.data_ptr(), ldy,
                           vector<float>(mean, "mean", r.rows, at::kFloat),
                           vector<float>(rstd, "rstd", r.rows, at::kFloat), s.p, s.bytes,
                           stream()),
         "layernorm_fwd");
    written(y);
    written(mean);
    written(rstd);
    return {y, mean, rstd};
}

std::tuple<Maybe, Maybe, Maybe> layernorm_backward(const Tensor &dy, const Tensor &x,
                                                   const Tensor &mean, const Tensor &rstd,
                                                   const Maybe &w, Maybe dx, Maybe dw, Maybe db,
                                                   bool with_input, bool with_weight,
                                                   bool with_bias, const Maybe &ws)
{
    Rows r;
    const int type = float_rows(x, "x", &r);
    const int64_t lddy = like(dy, "dy", x, r);
    const Maybe &given = w ? w : dw ? dw : db;
    const at::ScalarType wt = given ? given->scalar_type() : at::kFloat;
    int64_t lddx = r.cols;
    if (!with_input)
        dx = std::nullopt;
    else if (!dx)
        dx = empty(x.sizes(), x, x.scalar_type());
    if (dx)
        lddx = like(*dx, "dx", x, r);
    if (!with_weight)
        dw = std::nullopt;
    else if (!dw)
        dw = empty({r.cols}, x, wt);
    if (!with_bias)
        db = std::nullopt;
    else if (!db)
        db = empty({r.cols}, x, wt);
    const Workspace s(ws, lib.layernorm_bwd_ws(type, r.rows, r.cols), x.device());
    call(lib.layernorm_bwd(type, given ? type_of(*given) : MITRAIN_F32, r.rows, r.cols,
                           dy.data_ptr(), lddy, x.data_ptr(), r.ld,
                           vector<float>(mean, "mean", r.rows, at::kFloat),
                           vector<float>(rstd, "rstd", r.rows, at::kFloat),
                           vector(w, "w", r.cols, wt), dx ? dx->data_ptr() : nullptr, lddx,
                           vector(dw, "dw", r.cols, wt), vector(db, "db", r.cols, wt), s.p,
                           s.bytes, stream()),
         "layernorm_bwd");
    written(dx);
    written(dw);
    written(db);
    return {dx, dw, db};
}

// --------------------------------------------------------- log probabilities
Maybe logprob_workspace(const Tensor &logits, int top)
{
    Rows r;
    const int type = float_rows(logits, "logits", &r);
    top = (int)std::min<int64_t>(top, r.cols);
    return workspace(lib.logprob_fwd_ws(type, r.rows, r.cols, top), logits.device());
}

std::tuple<Maybe, Tensor, Tensor, Tensor, Maybe, Maybe>
logprob_forward(const Tensor &z, const Maybe &targets, int top, double scale, Maybe logp,
                Maybe lse, Maybe entropy, Maybe stats, Maybe top_logp, Maybe top_index,
                const Maybe &ws)
{
    Rows r;
    const int type = float_rows(z, "logits", &r);
    top = (int)std::min<int64_t>(top, r.cols);  // a row has no more tokens
    const auto *tp = vector<long long>(targets, "targets", r.rows, at::kLong);
    const at::IntArrayRef shape = z.sizes().slice(0, z.dim() - 1);
    const auto last = [&](int64_t n) {
        at::DimVector v(shape.begin(), shape.end());
        v.push_back(n);
        return v;
    };
    if (top < 0)
        call(MICONV_ERR_SHAPE, "logprob_fwd");
    const bool new_logp = targets && !logp, new_top = top && !top_logp;
    const int64_t floats = (stats ? 0 : 2) + !lse + !entropy + new_logp + (new_top ? top : 0);
    if (floats) {
        Results out(r.rows * floats, z);
        if (!stats)
            stats = out.next(last(2));
        if (!lse)
            lse = out.next(shape);
        if (!entropy)
            entropy = out.next(shape);
        if (new_logp)
            logp = out.next(shape);
        if (new_top)
            top_logp = out.next(last(top));
    }
    if (top && !top_index)
        top_index = empty(last(top), z, at::kLong);
    const Workspace s(ws, lib.logprob_fwd_ws(type, r.rows, r.cols, top), z.device());
    call(lib.logprob_fwd(type, r.rows, r.cols, z.data_ptr(), r.ld, tp, (float)scale, top,
                         vector<float>(logp, "logp", r.rows, at::kFloat),
                         vector<float>(lse, "lse", r.rows, at::kFloat),
                         vector<float>(entropy, "entropy", r.rows, at::kFloat),
                         vector<float>(stats, "stats", 2 * r.rows, at::kFloat),
                         vector<float>(top_logp, "top_logp", r.rows * top, at::kFloat),
                         vector<long long>(top_index, "top_index", r.rows * top, at::kLong), s.p,
                         s.bytes, stream()),
         "logprob_fwd");
    for (const Maybe *t : {&logp, &lse, &entropy, &stats, &top_logp, &top_index})
        written(*t);
    return {logp, *lse, *entropy, *stats, top_logp, top_index};
}

Tensor logprob_backward(const Tensor &z, const Tensor &stats, const Maybe &targets,
                        const Maybe &dlogp, const Maybe &entropy, const Maybe &dentropy,
                        double scale, const Maybe &dlogits)
{
    Rows r;
    const int type = float_rows(z, "logits", &r);
    const Tensor dz = dlogits ? *dlogits : empty(z.sizes(), z, z.scalar_type());
    const int64_t ldd = like(dz, "dlogits", z, r);
    call(lib.logprob_bwd(type, r.rows, r.cols, z.data_ptr(), r.ld,
                         vector<long long>(targets, "targets", r.rows, at::kLong), (float)scale,
                         vector<float>(stats, "stats", 2 * r.rows, at::kFloat),
                         vector<float>(dlogp, "dlogp", r.rows, at::kFloat),
                         vector<float>(entropy, "entropy", r.rows, at::kFloat),
                         vector<float>(dentropy, "dentropy", r.rows, at::kFloat), dz.data_ptr(),
                         ldd, stream()),
         "logprob_bwd");
    written(dz);
    return dz;
}

// ------------------------------------------------------------------ clipping
struct List {
    // Of a generator's tensors this is the only holder: until the launches are
    // enqueued, so that neither workspace nor results are given their memory.
    py::object fast;
    std::vector<void *> p;
    std::vector<long long> count;
    std::vector<int> type;
    std::optional<at::Device> device;

    List(const py::handle &tensors, const char *name)
        : fast(py::reinterpret_steal<py::object>(
              PySequence_Fast(tensors.ptr(), "a list of tensors is wanted")))
    {
        if (!fast)
            throw py::error_already_set();
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast.ptr());
        int current = -1;  // asked for once, where there is a device tensor
        p.reserve(n);
        count.reserve(n);
        type.reserve(n);
        for (Py_ssize_t i = 0; i < n; i++) {
            PyObject *o = PySequence_Fast_GET_ITEM(fast.ptr(), i);
            if (!THPVariable_Check(o))
                refuse(name, " must hold tensors");
            const Tensor &t = THPVariable_Unpack(o);
            const int k = type_of(t);
            if (current < 0 && t.is_cuda())
                current = c10::hip::current_device();
            if (k < 0 || !t.is_cuda() || t.get_device() != current || !t.is_contiguous())
                refuse(name, " must hold contiguous float32, bfloat16 or float16 tensors on the "
                             "current device");
            p.push_back(t.data_ptr());
            count.push_back(t.numel());
            type.push_back(k);
        }
        device = at::Device(at::kCUDA, n ? current : c10::hip::current_device());
    }
    int n() const { return (int)p.size(); }
    const Tensor &operator[](int i) const
    {
        return THPVariable_Unpack(PySequence_Fast_GET_ITEM(fast.ptr(), i));
    }
    size_t need() const { return lib.grad_ws(n(), count.data(), type.data()); }
};

Maybe grad_workspace(const py::object &grads)
{
    const List g(grads, "grads");
    return workspace(g.need(), *g.device);
}

Tensor one_float(const Maybe &norm, const List &g)
{
    if (norm)
        vector(norm, "norm", 1, at::kFloat);
    return norm ? *norm : at::empty({1}, at::TensorOptions(*g.device).dtype(at::kFloat));
}

Tensor gradient_norm(const py::object &grads, const Maybe &norm_, const Maybe &ws)
{
    const List g(grads, "grads");
    const Tensor norm = one_float(norm_, g);
    const Workspace s(ws, g.need(), *g.device);
    call(lib.grad_norm(g.n(), g.p.data(), g.count.data(), g.type.data(), (float *)norm.data_ptr(),
                       s.p, s.bytes, stream()),
         "grad_norm");
    written(norm);
    return norm;
}

Tensor gradient_clip(const py::object &grads, double max_norm, const py::object &out,
                     const Maybe &norm_, const Maybe &ws)
{
    const List g(grads, "grads");
    std::optional<List> o;
    if (!out.is_none()) {
        o.emplace(out, "out");
        if (o->count != g.count || o->type != g.type)
            refuse("out", " must hold a tensor of each gradient's type and size");
    }
    const Tensor norm = one_float(norm_, g);
    const Workspace s(ws, g.need(), *g.device);
    call(lib.grad_clip(g.n(), g.p.data(), g.count.data(), g.type.data(), (float)max_norm,
                       o ? o->p.data() : g.p.data(), (float *)norm.data_ptr(), s.p, s.bytes,
                       stream()),
         "grad_clip");
    written(norm);
    for (int i = 0; i < g.n(); i++)
        written((o ? *o : g)[i]);
    return norm;
}

}  // namespace

PYBIND11_MODULE(_mitrain, m)
{
    m.def("load", &load);
    m.def("rows", [](const Tensor &t) {
        const Rows r = rows_of(t, "x");
        return std::make_tuple(r.rows, r.cols, r.ld);
    });
    m.def("layernorm_workspace", &layernorm_workspace);
    m.def("layernorm_fwd", &layernorm_forward);
    m.def("layernorm_bwd", &layernorm_backward);
    m.def("logprob_workspace", &logprob_workspace);
    m.def("logprob_fwd", &logprob_forward);
    m.def("logprob_bwd", &logprob_backward);
    m.def("grad_workspace", &grad_workspace);
    m.def("grad_norm", &gradient_norm);
    m.def("grad_clip", &gradient_clip);
}
