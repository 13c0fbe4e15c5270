// The kernel for prompts over rows of the payload type.
#include "paged_flash_dev.h"

namespace mukv {

hipError_t launch_paged_flash(const PagedAttendArgs &a, int D, hipStream_t st) { return launch_flash_by_dim<false, false>(a, D, st); }

} // namespace mukv
