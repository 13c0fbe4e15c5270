// Attention over rows that groups of sequences share: the kernels for any shape that leave or take results.
#include "paged_attend_dev.h"

namespace mukv {

hipError_t launch_shared_attend(const PagedAttendArgs &a, int D, int dtype, bool eight, hipStream_t st) {
    if (eight) return dtype == MUKV_BF16 ? launch_by_dim<uint16_t, true, true>(a, D, st) : launch_by_dim<float, true, true>(a, D, st);
    return dtype == MUKV_BF16 ? launch_by_dim<uint16_t, false, true>(a, D, st) : launch_by_dim<float, false, true>(a, D, st);
}

} // namespace mukv
