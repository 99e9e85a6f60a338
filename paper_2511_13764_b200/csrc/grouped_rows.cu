// Instantiations of the grouped kernel, in a file of their own so that they compile side by side.
#include "grouped.cuh"

namespace nk {

GroupedFunction grouped_rows_kernel(bool a_mn, GroupedOut out) {
    if (out == GRP_OUT_H) return a_mn ? grouped_kernel<GRP_ROWS, true, GRP_OUT_H> : grouped_kernel<GRP_ROWS, false, GRP_OUT_H>;
    if (a_mn)
        return out == GRP_OUT_F32 ? grouped_kernel<GRP_ROWS, true, GRP_OUT_F32>
               : out == GRP_OUT_BF16 ? grouped_kernel<GRP_ROWS, true, GRP_OUT_BF16> : grouped_kernel<GRP_ROWS, true, GRP_OUT_F16>;
    return out == GRP_OUT_F32 ? grouped_kernel<GRP_ROWS, false, GRP_OUT_F32>
           : out == GRP_OUT_BF16 ? grouped_kernel<GRP_ROWS, false, GRP_OUT_BF16> : grouped_kernel<GRP_ROWS, false, GRP_OUT_F16>;
}

}  // namespace nk
