// The kernel for prompts that leaves or takes results of shared rows, over rows in 8 bits.
#include "paged_flash_dev.h"

namespace mukv {

hipError_t launch_shared_flash8(const PagedAttendArgs &a, int D, hipStream_t st) { return launch_flash_by_dim<true, true>(a, D, st); }

} // namespace mukv
