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
// k and v to pages of 8 bits; read: from them to k.out and v.out
hipError_t launch_rows8(const RopeArgs &a, int dtype, bool read, hipStream_t st);

// What a chunk of a tile's rows leaves for whoever joins them: per query, what its exponents subtracted and the sum of its weights, and its
// unnormalised output.
struct ChunkRecords {
    float *stats;  // [record][queries][2]
    float *values; // [record][queries][D]
    float *sums;   // [record][queries]: of weights that the values were not multiplied by as they are, before their rounding (paged_flash_dev.h,
                   // where the weights of rows are asked for)
};

// What attention over shared rows leaves for the call's other launch, over the sequences' own.  Chunks of a tile are not joined there but
// left as they are, for the other launch has more workgroups to read them than the shared rows have tiles: a place per chunk and query
// (of tiles with one chunk: per query) with the unnormalised output and, of its weights, what their exponents subtract, their sum as the
// output was multiplied by them and their sum as they were.
struct SharedResults {
    enum { kNone, kLeave, kTake };
    int mode;
    int n_groups;
    const int32_t *offsets; // of the groups' tokens; tokens before the first and behind the last are no group's.  Null: all are some group's
    int32_t *heads;         // [n_tokens * Hq][4]: chunks (kPlanChunks at most: PlanShape::left), the first one's place, places from one to the next
    float *values;          // [place][D]
    float *stats;           // [place][4]
    int single;             // place of query 0 of tiles with one chunk
    int *fit;               // whether the groups' offsets ascend: otherwise nothing is left, and nothing may be taken
};

struct PagedAttendArgs {
    PagedView view;
    PlanShape plan;
    const unsigned char *q; // strides in bytes
    int64_t q_token, q_head;
    void *out;     // [n_tokens][Hq][D]
    int *counts;   // [kPlanRecords], zero between calls
    ChunkRecords records; // room for the plan's
    float *pairs;  // [n_tokens * Hq][2]: what a query's weights' exponents subtract, 1 / their sum (0: no row seen); or null
    float scale_log2e;
    int causal;
    // with pairs: weights_out[b][g][j] = decay * weights_in[b][g][j] + what row j received; weights_in may be null
    const float *weights_in;
    float *weights_out;
    int64_t weights_seq, weights_head; // strides in elements
    int weights_rows;                  // rows a head has room for
    float decay;
    SharedResults shared;
};
hipError_t launch_paged_attend(const PagedAttendArgs &a, int D, int dtype, hipStream_t st);
hipError_t launch_paged_flash(const PagedAttendArgs &a, int D, hipStream_t st);
// the same over rows in 8 bits
hipError_t launch_paged_attend8(const PagedAttendArgs &a, int D, int dtype, hipStream_t st);
hipError_t launch_paged_flash8(const PagedAttendArgs &a, int D, hipStream_t st);
// what rows receive, by a.pairs
hipError_t launch_paged_weights(const PagedAttendArgs &a, int D, bool bf16, hipStream_t st);
hipError_t launch_paged_weights8(const PagedAttendArgs &a, int D, bool bf16, hipStream_t st);
// the same with results left or taken
hipError_t launch_shared_attend(const PagedAttendArgs &a, int D, int dtype, bool eight, hipStream_t st);
hipError_t launch_shared_flash(const PagedAttendArgs &a, int D, hipStream_t st);
hipError_t launch_shared_flash8(const PagedAttendArgs &a, int D, hipStream_t st);

struct EvictArgs {
    PagedView view; // of layer 0
    int64_t stride_layer, scale_layer; // bytes; of the scales, where rows are in 8 bits
    const float *w_in;
    float *w_out;
    int64_t w_layer, w_seq, w_head; // elements
    int w_rows, budget, n_sink, n_recent;
    const int32_t *into; // [n_seqs][into_width], or null: in place
    int into_width;
    int32_t *kept, *lengths_out; // [layer][n_seqs][Hkv][budget], [n_seqs]
};
hipError_t launch_paged_evict(const EvictArgs &a, int n_layers, int row_bytes, int device, hipStream_t st);

} // namespace mukv
