// Instantiations of the grouped kernel, in a file of their own so that they compile side by side.
#include "grouped.cuh"

namespace nk {

GroupedFunction grouped_weights_kernel(GroupedOut out, bool sums) {
    if (out == GRP_OUT_F32) return grouped_kernel<GRP_WEIGHTS, true, GRP_OUT_F32, true>;
    if (sums) return out == GRP_OUT_BF16 ? grouped_kernel<GRP_WEIGHTS, true, GRP_OUT_BF16, true> : grouped_kernel<GRP_WEIGHTS, true, GRP_OUT_F16, true>;
    return out == GRP_OUT_BF16 ? grouped_kernel<GRP_WEIGHTS, true, GRP_OUT_BF16, false> : grouped_kernel<GRP_WEIGHTS, true, GRP_OUT_F16, false>;
}

}  // namespace nk
