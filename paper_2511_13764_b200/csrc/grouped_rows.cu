// Instantiations of the grouped kernel, in a file of their own so that they compile side by side.
#include "grouped.cuh"

namespace nk {

template <bool A_MN>
static GroupedFunction of(GroupedOut out, bool sums) {
    if (out == GRP_OUT_H) return grouped_kernel<GRP_ROWS, A_MN, GRP_OUT_H, false>;      // (one chunk: nk_lora.cu)
    if (out == GRP_OUT_F32) return grouped_kernel<GRP_ROWS, A_MN, GRP_OUT_F32, true>;
    if (sums) return out == GRP_OUT_BF16 ? grouped_kernel<GRP_ROWS, A_MN, GRP_OUT_BF16, true> : grouped_kernel<GRP_ROWS, A_MN, GRP_OUT_F16, true>;
    return out == GRP_OUT_BF16 ? grouped_kernel<GRP_ROWS, A_MN, GRP_OUT_BF16, false> : grouped_kernel<GRP_ROWS, A_MN, GRP_OUT_F16, false>;
}

GroupedFunction grouped_rows_kernel(bool a_mn, GroupedOut out, bool sums) { return a_mn ? of<true>(out, sums) : of<false>(out, sums); }

}  // namespace nk
