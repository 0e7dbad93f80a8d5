// The end of a residual branch, forward and backward (include/mistep.h): total =
// residual + dropout(x) and the layer norm of total, by the kernels of
// norm_rows.h, which hold a row between its sum and its norm, or between its
// norm's gradient and the branch's.
//
// Forward x and the residual are read, total and y written; backward dy, total and the
// stream's gradient are read, that of the branch and of the residual written, which are
// one tensor where nothing is dropped.  Bound by memory (16384 x 4096 bf16: forward 94.1
// us for 537 MB, 5.7 TB/s, the sum and the norm by launches of their own 64.7 and 47;
// backward 138 for 671 MB, 4.9 TB/s, and 34 MB of partial sums), rows of few elements a
// thread by the loads they wait for (12544 x 513 fp32 backward 25.7 us, a copy of as many
// bytes 21), few rows by latencies (4 x 2048 bf16 forward 4.0).
// total is rounded to its type before its statistics are taken, so that the backward
// pass, which reads it, has the same numbers.
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
