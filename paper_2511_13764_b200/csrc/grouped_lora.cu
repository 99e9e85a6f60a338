// Instantiations of the grouped kernel, in a file of their own so that they compile side by side.
#include "grouped.cuh"

namespace nk {

LoraFunction grouped_lora_kernel(bool a_mn, GroupedOut out) {
    if (a_mn)
        return out == GRP_OUT_F32 ? grouped_kernel<GRP_LORA, true, GRP_OUT_F32, true>
               : out == GRP_OUT_BF16 ? grouped_kernel<GRP_LORA, true, GRP_OUT_BF16, true> : grouped_kernel<GRP_LORA, true, GRP_OUT_F16, true>;
    return out == GRP_OUT_F32 ? grouped_kernel<GRP_LORA, false, GRP_OUT_F32, true>
           : out == GRP_OUT_BF16 ? grouped_kernel<GRP_LORA, false, GRP_OUT_BF16, true> : grouped_kernel<GRP_LORA, false, GRP_OUT_F16, true>;
}

}  // namespace nk
