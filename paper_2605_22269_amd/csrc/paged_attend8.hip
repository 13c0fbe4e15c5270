// The kernels of an attention call over rows in 8 bits.
#include "paged_attend_dev.h"

namespace mukv {

hipError_t launch_paged_attend8(const PagedAttendArgs &a, int D, int dtype, hipStream_t st) {
    return dtype == MUKV_BF16 ? launch_by_dim<uint16_t, true, false>(a, D, st) : launch_by_dim<float, true, false>(a, D, st);
}
hipError_t launch_paged_weights8(const PagedAttendArgs &a, int D, bool bf16, hipStream_t st) {
    return bf16 ? launch_weights_by_dim<uint16_t, true>(a, D, st) : launch_weights_by_dim<float, true>(a, D, st);
}

} // namespace mukv
