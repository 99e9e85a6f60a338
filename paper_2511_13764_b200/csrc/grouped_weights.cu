// Instantiations of the grouped kernel, in a file of their own so that they compile side by side.
#include "grouped.cuh"

namespace nk {

GroupedFunction grouped_weights_kernel(GroupedOut out) {
    return out == GRP_OUT_F32 ? grouped_kernel<GRP_WEIGHTS, true, GRP_OUT_F32>
           : out == GRP_OUT_BF16 ? grouped_kernel<GRP_WEIGHTS, true, GRP_OUT_BF16> : grouped_kernel<GRP_WEIGHTS, true, GRP_OUT_F16>;
}

}  // namespace nk
