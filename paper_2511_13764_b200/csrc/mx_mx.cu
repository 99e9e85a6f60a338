// The kernels of nk_mx for MXF4 operands.
#include "mx.cuh"

namespace nk {

template <int OUT>
static MxFunction of_mode(MxMode mode) {
    return mode == MX_SUMS ? mx_kernel<false, OUT, MX_SUMS> : mode == MX_CUT ? mx_kernel<false, OUT, MX_CUT> : mx_kernel<false, OUT, MX_WHOLE_TILES>;
}
MxFunction mx_kernel_mx(MxOut out, MxMode mode) {
    return out == MX_OUT_F32 ? of_mode<MX_OUT_F32>(mode) : out == MX_OUT_BF16 ? of_mode<MX_OUT_BF16>(mode) : of_mode<MX_OUT_F16>(mode);
}

}  // namespace nk
