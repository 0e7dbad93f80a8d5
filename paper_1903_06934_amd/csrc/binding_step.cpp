// Python binding of include/mistep.h: argument marshalling only, as binding.cpp.
// mistep.py has the documentation; it hands over the library's functions once
// (load_step).
#include <math.h>
#include <string.h>
#include <array>
#include <tuple>

#include <torch/csrc/autograd/python_variable.h>

#include "binding.h"
#include "mistep.h"

using namespace binding;

namespace {

struct Library {
    decltype(&::dropout_fwd) dropout_fwd;
    decltype(&::dropout_bwd) dropout_bwd;
    decltype(&::residual_norm_fwd_workspace_size) norm_fwd_ws;
    decltype(&::residual_norm_bwd_workspace_size) norm_bwd_ws;
    decltype(&::residual_norm_fwd) norm_fwd;
    decltype(&::residual_norm_bwd) norm_bwd;
    decltype(&::policy_loss_workspace_size) policy_ws;
    decltype(&::policy_loss) policy;
    decltype(&::preference_loss_workspace_size) preference_ws;
    decltype(&::preference_loss) preference;
} step_lib;

void load_step(const std::array<uintptr_t, 10> &functions)
{
    memcpy(&step_lib, functions.data(), sizeof(step_lib));
    static_assert(sizeof(step_lib) == 10 * sizeof(uintptr_t), "one address each");
}

// The numbers of a dropout; step is a number or a device tensor that holds one.
struct Numbers {
    unsigned long long seed;
    unsigned layer, step = 0;
    const long long *step_at = nullptr;

    Numbers(uint64_t seed_, uint32_t layer_, const py::object &s) : seed(seed_), layer(layer_)
    {
        if (THPVariable_Check(s.ptr())) {
            step_at = vector<long long>(THPVariable_Unpack(s.ptr()), "step", 1, at::kLong);
        } else {
            if (!PyIndex_Check(s.ptr()))
                refuse("step", " must be a whole number, or a device tensor of one");
            const auto n = py::reinterpret_steal<py::object>(PyNumber_Index(s.ptr()));
            if (!n)
                throw py::error_already_set();
            step = (unsigned)PyLong_AsUnsignedLongLongMask(n.ptr());  // modulo 2^32
        }
    }
};

// --------------------------------------------------------------------- dropout
Tensor dropout_forward(const Tensor &x, double p, uint64_t seed, uint32_t layer,
                       const py::object &step, const Maybe &residual, const Maybe &y_)
{
    Rows r;
    const int type = float_rows(x, "x", &r);
    const int64_t ldr = residual ? like(*residual, "residual", x, r) : 0;
    const Tensor y = y_ ? *y_ : empty(x.sizes(), x, x.scalar_type());
    const int64_t ldy = like(y, "y", x, r);
    const Numbers n(seed, layer, step);
    call(step_lib.dropout_fwd(type, r.rows, r.cols, x.data_ptr(), r.ld,
                              residual ? residual->data_ptr() : nullptr, ldr, p, n.seed, n.layer,
                              n.step, n.step_at, y.data_ptr(), ldy, stream()),
         "dropout_fwd");
    written(y);
    return y;
}

Tensor dropout_backward(const Tensor &dy, double p, uint64_t seed, uint32_t layer,
                        const py::object &step, const Maybe &dx_)
{
    Rows r;
    const int type = float_rows(dy, "dy", &r);
    const Tensor dx = dx_ ? *dx_ : empty(dy.sizes(), dy, dy.scalar_type());
    const int64_t lddx = like(dx, "dx", dy, r);
    const Numbers n(seed, layer, step);
    call(step_lib.dropout_bwd(type, r.rows, r.cols, dy.data_ptr(), r.ld, p, n.seed, n.layer,
                              n.step, n.step_at, dx.data_ptr(), lddx, stream()),
         "dropout_bwd");
    written(dx);
    return dx;
}

// ------------------------------------------------------------ residual branches
// Of so many bytes each, two results share an allocation (four rows of 2048 16-bit
// elements: 16 KiB).  Larger ones do not: one would keep the other's memory.
constexpr size_t kSmall = 64 << 10;

Maybe norm_workspace(bool backward, const Tensor &x)
{
    Rows r;
    const int type = float_rows(x, "x", &r);
    return workspace((backward ? step_lib.norm_bwd_ws : step_lib.norm_fwd_ws)(type, r.rows, r.cols),
                     x.device());
}

std::tuple<Tensor, Tensor, Tensor, Tensor>
norm_forward(const Tensor &x, const Tensor &residual, const Maybe &w, const Maybe &b, double eps,
             double p, uint64_t seed, uint32_t layer, const py::object &step, const Maybe &total_,
             const Maybe &y_, const Maybe &mean_, const Maybe &rstd_, const Maybe &ws)
{
    Rows r;
    const int type = float_rows(x, "x", &r);
    const int64_t ldr = like(residual, "residual", x, r);
    const at::ScalarType wt = w ? w->scalar_type() : b ? b->scalar_type() : x.scalar_type();
    const void *wp = vector(w, "w", r.cols, wt), *bp = vector(b, "b", r.cols, wt);
    Tensor total, y;
    if (!total_ && !y_ && x.nbytes() <= kSmall) {
        Results out(2 * x.numel(), x, x.scalar_type());
        total = out.next(x.sizes());
        y = out.next(x.sizes());
    } else {
        total = total_ ? *total_ : empty(x.sizes(), x, x.scalar_type());
        y = y_ ? *y_ : empty(x.sizes(), x, x.scalar_type());
    }
    const int64_t ldt = like(total, "total", x, r), ldy = like(y, "y", x, r);
    Tensor mean, rstd;
    if (mean_ && rstd_) {
        mean = *mean_;
        rstd = *rstd_;
    } else {
        Results out(2 * r.rows, x);
        mean = mean_ ? *mean_ : out.next({r.rows});
        rstd = rstd_ ? *rstd_ : out.next({r.rows});
    }
    const Numbers n(seed, layer, step);
    const Workspace s(ws, step_lib.norm_fwd_ws(type, r.rows, r.cols), x.device());
    call(step_lib.norm_fwd(type, w ? type_of(*w) : b ? type_of(*b) : type, r.rows, r.cols,
                           x.data_ptr(), r.ld, residual.data_ptr(), ldr, p, n.seed, n.layer, n.step,
                           n.step_at, wp, bp, (float)eps, total.data_ptr(), ldt, y.data_ptr(), ldy,
                           vector<float>(mean, "mean", r.rows, at::kFloat),
                           vector<float>(rstd, "rstd", r.rows, at::kFloat), s.p, s.bytes,
                           stream()),
         "residual_norm_fwd");
    for (const Tensor &t : {total, y, mean, rstd})
        written(t);
    return {total, y, mean, rstd};
}

std::tuple<Maybe, Maybe, Maybe, Maybe>
norm_backward(const Tensor &dy, const Tensor &total, const Tensor &mean, const Tensor &rstd,
              const Maybe &w, const Maybe &dtotal, double p, uint64_t seed, uint32_t layer,
              const py::object &step, Maybe dx, Maybe dresidual, Maybe dw, Maybe db,
              bool with_input, bool with_weight, bool with_bias, const Maybe &ws)
{
    Rows r;
    const int type = float_rows(total, "total", &r);
    const int64_t lddy = like(dy, "dy", total, r);
    const int64_t lddt = dtotal ? like(*dtotal, "dtotal", total, r) : 0;
    const Maybe &given = w ? w : dw ? dw : db;
    const at::ScalarType wt = given ? given->scalar_type() : at::kFloat;
    const bool drops = !(p <= 0.5 / 65536);  // else dx and dresidual are one
    if (!with_input) {
        dx = dresidual = std::nullopt;
    } else {
        if (!dresidual)
            dresidual = empty(total.sizes(), total, total.scalar_type());
        if (!dx && drops)
            dx = empty(total.sizes(), total, total.scalar_type());
    }
    const int64_t lddx = dx ? like(*dx, "dx", total, r) : 0;
    const int64_t lddr = dresidual ? like(*dresidual, "dresidual", total, r) : 0;
    if (!with_weight)
        dw = std::nullopt;
    else if (!dw)
        dw = empty({r.cols}, total, wt);
    if (!with_bias)
        db = std::nullopt;
    else if (!db)
        db = empty({r.cols}, total, wt);
    const Numbers n(seed, layer, step);
    const Workspace s(ws, step_lib.norm_bwd_ws(type, r.rows, r.cols), total.device());
    call(step_lib.norm_bwd(type, given ? type_of(*given) : MITRAIN_F32, r.rows, r.cols,
                           dy.data_ptr(), lddy, total.data_ptr(), r.ld,
                           vector<float>(mean, "mean", r.rows, at::kFloat),
                           vector<float>(rstd, "rstd", r.rows, at::kFloat),
                           vector(w, "w", r.cols, wt), dtotal ? dtotal->data_ptr() : nullptr, lddt,
                           p, n.seed, n.layer, n.step, n.step_at,
                           dresidual ? dresidual->data_ptr() : nullptr, lddr,
                           dx ? dx->data_ptr() : nullptr, lddx, vector(dw, "dw", r.cols, wt),
                           vector(db, "db", r.cols, wt), s.p, s.bytes, stream()),
         "residual_norm_bwd");
    for (const Maybe *t : {&dx, &dresidual, &dw, &db})
        written(*t);
    return {dx || !with_input ? dx : dresidual, dresidual, dw, db};
}

// ---------------------------------------------------------------------- losses
// The tokens' mask, of bool or uint8.
const unsigned char *mask_of(const Maybe &mask, int64_t n)
{
    if (!mask)
        return nullptr;
    return vector<unsigned char>(mask, "mask", n,
                                 mask->scalar_type() == at::kBool ? at::kBool : at::kByte);
}

struct Sequences {
    int64_t n = 0;
    const long long *starts = nullptr;

    explicit Sequences(const Maybe &t)
    {
        if (!t)
            return;
        n = t->numel() - 1;
        if (n < 0)
            refuse("starts", " must have at least one element");
        starts = vector<long long>(t, "starts", n + 1, at::kLong);
    }
};

// The tokens' log probabilities, which all other tensors go by.
int64_t tokens_of(const Tensor &logp)
{
    vector<float>(logp, "logp", logp.numel(), at::kFloat);
    return logp.numel();
}

Maybe policy_workspace(const Tensor &logp, const Maybe &starts)
{
    return workspace(step_lib.policy_ws(tokens_of(logp), Sequences(starts).n), logp.device());
}

std::tuple<Tensor, Maybe, Maybe>
policy(const Tensor &logp, const Tensor &old_logp, const Tensor &advantages, bool by_sequence,
       const Maybe &ref_logp, const Maybe &entropy, const Maybe &mask, const Maybe &starts,
       double clip_low, double clip_high, double dual_clip, int kl, double kl_weight,
       double entropy_weight, int mean, double count, double scale, bool with_grad,
       const Maybe &stats_, Maybe dlogp, Maybe dentropy, const Maybe &ws)
{
    const int64_t n = tokens_of(logp);
    const Sequences q(starts);
    const Tensor stats = stats_ ? *stats_ : empty({6}, logp, at::kFloat);
    if (!with_grad) {
        dlogp = dentropy = std::nullopt;
    } else {
        if (!dlogp)
            dlogp = empty(logp.sizes(), logp, at::kFloat);
        if (!dentropy && entropy)
            dentropy = empty(logp.sizes(), logp, at::kFloat);
    }
    const auto floats = [&](const Maybe &t, const char *name) {
        return vector<float>(t, name, n, at::kFloat);
    };
    const Workspace s(ws, step_lib.policy_ws(n, q.n), logp.device());
    call(step_lib.policy(n, q.n, floats(logp, "logp"), floats(old_logp, "old_logp"),
                         floats(ref_logp, "ref_logp"), floats(entropy, "entropy"),
                         vector<float>(advantages, "advantages", by_sequence ? q.n : n, at::kFloat),
                         by_sequence, mask_of(mask, n), q.starts, clip_low, clip_high, dual_clip,
                         kl, kl_weight, entropy_weight, mean, count, scale,
                         vector<float>(stats, "stats", 6, at::kFloat), floats(dlogp, "dlogp"),
                         floats(dentropy, "dentropy"), s.p, s.bytes, stream()),
         "policy_loss");
    written(stats);
    written(dlogp);
    written(dentropy);
    return {stats, dlogp, dentropy};
}

// Pairs of sequences.
int64_t pairs_of(const Sequences &q)
{
    if (q.n % 2)
        refuse("starts", " must be of an even number of sequences");
    return q.n / 2;
}

Maybe preference_workspace(const Tensor &logp, const Tensor &starts)
{
    return workspace(step_lib.preference_ws(tokens_of(logp), pairs_of(Sequences(starts))),
                     logp.device());
}

std::tuple<Tensor, Tensor, Maybe>
preference(const Tensor &logp, const Maybe &ref_logp, const Tensor &starts, double beta, int form,
           double smoothing, double margin, bool length_mean, const Maybe &mask, double scale,
           bool with_grad, Maybe stats, Maybe rewards, Maybe dlogp, const Maybe &ws)
{
    const int64_t n = tokens_of(logp);
    const Sequences q(starts);
    const int64_t pairs = pairs_of(q);
    if (!stats || !rewards) {
        Results out(5 + q.n, logp);
        if (!stats)
            stats = out.next({5});
        if (!rewards)
            rewards = out.next({q.n});
    }
    if (!with_grad)
        dlogp = std::nullopt;
    else if (!dlogp)
        dlogp = empty(logp.sizes(), logp, at::kFloat);
    const Workspace s(ws, step_lib.preference_ws(n, pairs), logp.device());
    call(step_lib.preference(n, pairs, vector<float>(logp, "logp", n, at::kFloat),
                             vector<float>(ref_logp, "ref_logp", n, at::kFloat), mask_of(mask, n),
                             q.starts, beta, form, smoothing, margin, length_mean, scale,
                             vector<float>(stats, "stats", 5, at::kFloat),
                             vector<float>(rewards, "rewards", q.n, at::kFloat),
                             vector<float>(dlogp, "dlogp", n, at::kFloat), s.p, s.bytes, stream()),
         "preference_loss");
    written(stats);
    written(rewards);
    written(dlogp);
    return {*stats, *rewards, dlogp};
}

}  // namespace

void binding::bind_step(py::module_ &m)
{
    m.def("load_step", &load_step);
    m.def("dropout_fwd", &dropout_forward);
    m.def("dropout_bwd", &dropout_backward);
    m.def("residual_norm_workspace", &norm_workspace);
    m.def("residual_norm_fwd", &norm_forward);
    m.def("residual_norm_bwd", &norm_backward);
    m.def("policy_workspace", &policy_workspace);
    m.def("policy_loss", &policy);
    m.def("preference_workspace", &preference_workspace);
    m.def("preference_loss", &preference);
}
