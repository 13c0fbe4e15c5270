// The kernel for prompts over rows in 8 bits.
#include "paged_flash_dev.h"

namespace mukv {

hipError_t launch_paged_flash8(const PagedAttendArgs &a, int D, hipStream_t st) { return launch_flash_by_dim<true, false>(a, D, st); }

} // namespace mukv
