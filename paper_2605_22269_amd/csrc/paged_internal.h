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

// Which kernel takes an attention call follows from types and sizes that the host knows (paged_attend.hip): 0 that for any shape, otherwise
// the one for prompts, with tiles of so many queries.  new_hint: new tokens of a sequence, as far as that is known.
int paged_prompt_tile(const PagedView &v, int dtype, int D, int64_t new_hint);
PlanShape paged_plan(int dtype, int prompt_tile, bool causal);
constexpr int kPlanChunks = 64;     // most chunks of a sequence
constexpr int kPlanRecords = 2048;  // most that any plan has: the counts at a workspace's start

// What a chunk of a tile's rows leaves for whoever joins them: per query, what its exponents subtracted and the sum of its weights, and its
// unnormalised output.
struct ChunkRecords {
    float *stats;  // [record][queries][2]
    float *values; // [record][queries][D]
    float *sums;   // [record][queries]: of weights that the values were not multiplied by as they are, before their rounding (paged_flash.hip,
                   // where the weights of rows are asked for)
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
};
hipError_t launch_paged_attend(const PagedAttendArgs &a, int D, int dtype, hipStream_t st);
hipError_t launch_paged_flash(const PagedAttendArgs &a, int D, hipStream_t st);

struct EvictArgs {
    PagedView view; // of layer 0
    int64_t stride_layer; // bytes
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
