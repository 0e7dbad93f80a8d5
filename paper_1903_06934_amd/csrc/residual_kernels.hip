// The end of a residual branch, forward and backward (include/mistep.h): total =
// residual + dropout(x) and the layer norm of total, by the kernels of
// norm_rows.h, which hold a row between its sum and its norm, or between its
// norm's gradient and the branch's.
#include "norm_rows.h"

namespace miconv {

namespace {

template <class T, class TW>
hipError_t branch_fwd(int xtype, const ResidualFwdArgs &a, hipStream_t stream)
{
    if (!a.rows)
        return hipSuccess;
    const RowPlan p = row_plan(xtype, a.rows, a.cols, true);
    if (p.nv)
        return fwd_in_registers<T, TW>(p, a, stream);
    // Rows that go by pieces: the sum first, then the norm of what it wrote.
    const hipError_t e =
        launch_dropout(xtype, DropoutArgs{a.rows, a.cols, a.x, a.residual, a.total, a.drop}, stream);
    if (e != hipSuccess)
        return e;
    NormFwdArgs n = a;
    n.x = a.total;
    return launch_norm_fwd(xtype, sizeof(TW) == 4, n, stream);
}

}  // namespace

hipError_t launch_residual_fwd(int xtype, bool w32, const ResidualFwdArgs &a, hipStream_t stream)
{
    if (xtype == 0)
        return branch_fwd<float, float>(xtype, a, stream);
    if (xtype == 1)
        return w32 ? branch_fwd<__bf16, float>(xtype, a, stream)
                   : branch_fwd<__bf16, __bf16>(xtype, a, stream);
    return w32 ? branch_fwd<_Float16, float>(xtype, a, stream)
               : branch_fwd<_Float16, _Float16>(xtype, a, stream);
}

hipError_t launch_residual_bwd(int xtype, bool w32, const ResidualBwdArgs &a, hipStream_t stream)
{
    if (xtype == 0)
        return bwd<float, float>(xtype, a, stream);
    if (xtype == 1)
        return w32 ? bwd<__bf16, float>(xtype, a, stream) : bwd<__bf16, __bf16>(xtype, a, stream);
    return w32 ? bwd<_Float16, float>(xtype, a, stream)
               : bwd<_Float16, _Float16>(xtype, a, stream);
}

}  // namespace miconv
