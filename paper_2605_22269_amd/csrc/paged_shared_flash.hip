// The kernel for prompts that leaves or takes results of shared rows, over rows of the payload type.
#include "paged_flash_dev.h"

namespace mukv {

hipError_t launch_shared_flash(const PagedAttendArgs &a, int D, hipStream_t st) { return launch_flash_by_dim<false, true>(a, D, st); }

} // namespace mukv
