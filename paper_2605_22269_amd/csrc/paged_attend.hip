// The kernels of an attention call over rows of the payload type.
#include "paged_attend_dev.h"

namespace mukv {

hipError_t launch_paged_attend(const PagedAttendArgs &a, int D, int dtype, hipStream_t st) {
    return dtype == MUKV_BF16 ? launch_by_dim<uint16_t, false, false>(a, D, st) : launch_by_dim<float, false, false>(a, D, st);
}
hipError_t launch_paged_weights(const PagedAttendArgs &a, int D, bool bf16, hipStream_t st) {
    return bf16 ? launch_weights_by_dim<uint16_t, false>(a, D, st) : launch_weights_by_dim<float, false>(a, D, st);
}

} // namespace mukv
