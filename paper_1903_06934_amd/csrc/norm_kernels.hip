// Layer norm of rows (include/mitrain.h); the kernels are in norm_rows.h.
#include "norm_rows.h"

namespace miconv {

size_t norm_fwd_ws(int xtype, long long rows, long long cols)
{
    if (row_plan(xtype, rows, cols, true).nv)
        return 0;
    return (size_t)rows * piece_plan(xtype, rows, cols, true).splits * sizeof(Moments);
}

size_t norm_bwd_ws(int xtype, long long rows, long long cols)
{
    const RowPlan p = row_plan(xtype, rows, cols, false);
    const size_t part = 2 * (size_t)cols * sizeof(float);
    if (!rows)
        return 0;
    if (p.nv)
        return bwd_blocks(p, rows) * part;
    const int n = row_chunks(xtype, rows, cols);  // one writes dw and db itself
    return up16((size_t)rows * piece_plan(xtype, rows, cols, false).splits * 2 * sizeof(float)) +
           (n > 1 ? n * part : 0);
}

hipError_t launch_norm_fwd(int xtype, bool w32, const NormFwdArgs &a, hipStream_t stream)
{
    if (xtype == 0)
        return fwd<float, float>(xtype, a, stream);
    if (xtype == 1)
        return w32 ? fwd<__bf16, float>(xtype, a, stream) : fwd<__bf16, __bf16>(xtype, a, stream);
    return w32 ? fwd<_Float16, float>(xtype, a, stream)
               : fwd<_Float16, _Float16>(xtype, a, stream);
}

hipError_t launch_norm_bwd(int xtype, bool w32, const NormBwdArgs &a, hipStream_t stream)
{
    if (xtype == 0)
        return bwd<float, float>(xtype, a, stream);
    if (xtype == 1)
        return w32 ? bwd<__bf16, float>(xtype, a, stream) : bwd<__bf16, __bf16>(xtype, a, stream);
    return w32 ? bwd<_Float16, float>(xtype, a, stream)
               : bwd<_Float16, _Float16>(xtype, a, stream);
}

}  // namespace miconv
