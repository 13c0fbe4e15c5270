// Between the C ABI of the paged cache and its kernels.
#pragma once

#include "mukv_internal.h"
#include "paged_plan.h"

namespace mukv {

// Rows to rotate, copy and place: up to three tensors [token][head][D].  Strides in bytes.
struct RopeArgs {
    struct Rows {
        const unsigned char *x;
        unsigned char *out; // or null: into the pages
        int64_t token, head, out_token, out_head;
        int heads;
    } q, k, v; // q, k rotated; k, v into the pages
    PagedView view;
    const double *inv_freq;
    const int32_t *axis, *positions;
    int n_tokens, D, n_rot, n_axes;
    bool rotate, neighbours, inverse;
};
hipError_t launch_rope(const RopeArgs &a, int dtype, hipStream_t st);

} // namespace mukv
