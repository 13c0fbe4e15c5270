// C ABI of the conversation's paged cache (declared in include/mukv.h): argument validation and dispatch.  Nothing here is kept
// between calls.
#include <cmath>

#include "paged_internal.h"

using mukv::DeviceScope;
using mukv::PagedView;
using mukv::RopeArgs;

namespace {

bool aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int elem_size(int dtype) { return dtype == MUKV_BF16 ? 2 : 4; }
int finished(hipError_t e) { return e == hipSuccess ? MUKV_OK : MUKV_ERR_HIP; }

// Strides of `count` places: not negative, whole pieces of 16 bytes, and so small that bytes stay within 63 bits.  That of a single
// place is never walked and may be anything.
int check_stride(int64_t stride, int64_t count, int esz) {
    if (count <= 1) return MUKV_OK;
    if (stride < 0) return MUKV_ERR_INVALID_ARG;
    if (stride * esz % 16 || stride > (INT64_MAX >> 4) / count) return MUKV_ERR_UNSUPPORTED;
    return MUKV_OK;
}

int64_t in_bytes(int64_t stride, int64_t count, int esz) { return count > 1 ? stride * esz : 0; }

// empty: no row is ever looked at, and empty tensors need not have an address
int check_pages(const mukv_paged *p, bool empty = false) {
    if (!p || (!empty && (!p->k_pages || !p->v_pages))) return MUKV_ERR_INVALID_ARG;
    if (p->n_layers < 1 || p->n_pages < 1 || p->page_rows < (empty ? 0 : 1) || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->device_id < 0)
        return MUKV_ERR_INVALID_ARG;
    if (p->dtype != MUKV_BF16 && p->dtype != MUKV_F32) return MUKV_ERR_INVALID_ARG;
    if (p->n_q_heads % p->n_kv_heads) return MUKV_ERR_SHAPE;
    if (p->head_dim < 16 || p->head_dim > 128 || (p->head_dim & (p->head_dim - 1))) return MUKV_ERR_UNSUPPORTED;
    if (p->n_q_heads / p->n_kv_heads > 1024 || p->n_q_heads > 65535) return MUKV_ERR_UNSUPPORTED;
    const int esz = elem_size(p->dtype);
    const int64_t strides[4] = {p->stride_layer, p->stride_page, p->stride_head, p->stride_row};
    const int64_t counts[4] = {p->n_layers, p->n_pages, p->n_kv_heads, p->page_rows};
    for (int i = 0; i < 4; ++i)
        if (const int rc = check_stride(strides[i], counts[i], esz)) return rc;
    if (!aligned(p->k_pages) || !aligned(p->v_pages)) return MUKV_ERR_UNSUPPORTED;
    return MUKV_OK;
}

bool packed_nothing(const mukv_seqs *s) { return s && !s->table && s->n_tokens == 0; }

int check_seqs(const mukv_paged *p, const mukv_seqs *s, bool may_be_packed, bool has_tokens) {
    if (!s) return MUKV_ERR_INVALID_ARG;
    if (s->n_seqs < 1) return MUKV_ERR_INVALID_ARG;
    if (s->n_seqs > 65536) return MUKV_ERR_UNSUPPORTED;
    if (has_tokens) {
        if (s->n_tokens < 0 || s->max_new < 0) return MUKV_ERR_INVALID_ARG;
        if (!s->offsets && s->n_tokens % s->n_seqs) return MUKV_ERR_SHAPE;
        if ((int64_t)s->n_tokens * p->n_q_heads > 0x7ff00000) return MUKV_ERR_UNSUPPORTED;
    }
    if (!s->table) {
        if (!may_be_packed) return MUKV_ERR_INVALID_ARG;
        return s->offsets ? MUKV_OK : MUKV_ERR_INVALID_ARG;
    }
    if (!s->lengths || s->table_width < 1) return MUKV_ERR_INVALID_ARG;
    if (p->page_rows > 1 << 24 || (int64_t)s->table_width * p->page_rows > 0x7ff00000 || (int64_t)s->table_width * s->n_seqs > 0x7fffffff)
        return MUKV_ERR_UNSUPPORTED; // row and entry numbers are 32-bit in the kernels
    return MUKV_OK;
}

PagedView view_of(const mukv_paged &p, int layer, const mukv_seqs &s) {
    const int esz = elem_size(p.dtype);
    PagedView v;
    v.k = static_cast<unsigned char *>(p.k_pages) + layer * in_bytes(p.stride_layer, p.n_layers, esz);
    v.v = static_cast<unsigned char *>(p.v_pages) + layer * in_bytes(p.stride_layer, p.n_layers, esz);
    v.stride_page = in_bytes(p.stride_page, p.n_pages, esz);
    v.stride_head = in_bytes(p.stride_head, p.n_kv_heads, esz);
    v.stride_row = in_bytes(p.stride_row, p.page_rows, esz);
    v.table = s.table;
    v.lengths = s.lengths;
    v.offsets = s.offsets;
    v.n_pages = p.n_pages;
    v.page_rows = p.page_rows;
    v.n_seqs = s.n_seqs;
    v.table_width = s.table_width;
    v.n_tokens = s.n_tokens;
    v.per_seq = s.n_tokens / s.n_seqs;
    v.Hq = p.n_q_heads;
    v.Hkv = p.n_kv_heads;
    v.G = p.n_q_heads / p.n_kv_heads;
    return v;
}

// [token][head][head_dim] with strides
int check_rows(const void *x, const mukv_strides *st, int n_tokens, int n_heads, int esz) {
    if (!x || !st) return MUKV_ERR_INVALID_ARG;
    if (const int rc = check_stride(st->token, n_tokens, esz)) return rc;
    if (const int rc = check_stride(st->head, n_heads, esz)) return rc;
    return aligned(x) ? MUKV_OK : MUKV_ERR_UNSUPPORTED;
}
RopeArgs::Rows rows_in(const void *x, const mukv_strides *st, void *out, const mukv_strides *out_st, int tokens, int heads, int esz) {
    RopeArgs::Rows r = {};
    if (!x) return r;
    r.x = static_cast<const unsigned char *>(x);
    r.token = in_bytes(st->token, tokens, esz);
    r.head = in_bytes(st->head, heads, esz);
    r.out = static_cast<unsigned char *>(out);
    if (out) {
        r.out_token = in_bytes(out_st->token, tokens, esz);
        r.out_head = in_bytes(out_st->head, heads, esz);
    }
    r.heads = heads;
    return r;
}

int check_rope(const mukv_rope_table *r, bool have_positions, int head_dim) {
    if (!r || !r->inv_freq || !have_positions) return MUKV_ERR_INVALID_ARG;
    if (r->n_rot < 1 || r->n_axes < 1 || r->n_axes > 16 || (r->inverse != 0 && r->inverse != 1)) return MUKV_ERR_INVALID_ARG;
    if (r->pairing != MUKV_ROPE_HALVES && r->pairing != MUKV_ROPE_NEIGHBOURS) return MUKV_ERR_INVALID_ARG;
    if (r->n_rot > head_dim) return MUKV_ERR_SHAPE;
    if (r->n_rot % 16 || r->n_rot > 512) return MUKV_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(r->inv_freq) & 7) return MUKV_ERR_UNSUPPORTED;
    return MUKV_OK;
}
void set_rope(RopeArgs &a, const mukv_rope_table *r, const int32_t *positions) {
    a.rotate = r != nullptr;
    if (!r) return;
    a.inv_freq = r->inv_freq;
    a.axis = r->axis;
    a.positions = positions;
    a.n_rot = r->n_rot;
    a.n_axes = r->n_axes;
    a.neighbours = r->pairing == MUKV_ROPE_NEIGHBOURS;
    a.inverse = r->inverse != 0;
}

// Which kernel takes an attention call, and its workspace: counts, records, then (with weights) the prompt kernel's sums and a pair per query.
struct Space {
    mukv::PlanShape plan;
    int64_t stats, values, sums, pairs, bytes; // offsets; the counts are at 0
};
Space space_of(const mukv_paged &p, const mukv_seqs &s, bool causal, bool with_weights) {
    const int64_t hint = s.max_new > 0 ? s.max_new : mukv::div_up(s.n_tokens, s.n_seqs);
    Space x;
    const int tile = mukv::paged_prompt_tile(view_of(p, 0, s), p.dtype, p.head_dim, hint);
    x.plan = mukv::paged_plan(p.dtype, tile, causal);
    const int64_t rows = (int64_t)x.plan.records * x.plan.queries;
    x.stats = 4 * mukv::kPlanRecords;
    x.values = x.stats + 8 * rows;
    x.sums = x.values + 4 * rows * p.head_dim;
    x.pairs = x.sums + (with_weights && tile ? 4 * rows : 0);
    x.bytes = x.pairs + (with_weights ? 8 * (int64_t)s.n_tokens * p.n_q_heads : 0);
    return x;
}

int check_weights(const mukv_row_weights *w) {
    if (!w->out || w->rows < 1 || w->stride_layer < 0 || w->stride_seq < 0 || w->stride_head < 0) return MUKV_ERR_INVALID_ARG;
    if (!(w->decay >= 0.f) || !(w->decay <= 3.4e38f)) return MUKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(w->in) & 3) || (reinterpret_cast<uintptr_t>(w->out) & 3)) return MUKV_ERR_UNSUPPORTED;
    return MUKV_OK;
}

} // namespace

extern "C" {

int mukv_rope(const mukv_rope_table *rope, const void *x, const mukv_strides *x_strides, const int32_t *positions,
              int32_t n_tokens, int32_t n_heads, int32_t head_dim, int32_t dtype, void *out,
              const mukv_strides *out_strides, int32_t device_id, void *stream) {
    if (n_tokens < 0 || n_heads < 1 || head_dim < 1 || device_id < 0) return MUKV_ERR_INVALID_ARG;
    if (dtype != MUKV_BF16 && dtype != MUKV_F32) return MUKV_ERR_INVALID_ARG;
    const int esz = elem_size(dtype);
    if (const int rc = check_rope(rope, n_tokens == 0 || positions, head_dim)) return rc;
    if (head_dim * esz % 16 || head_dim > 1024 || n_heads > 65535) return MUKV_ERR_UNSUPPORTED;
    if (n_tokens == 0) return MUKV_OK;
    if (const int rc = check_rows(x, x_strides, n_tokens, n_heads, esz)) return rc;
    if (const int rc = check_rows(out, out_strides, n_tokens, n_heads, esz)) return rc;
    RopeArgs a = {};
    a.q = rows_in(x, x_strides, out, out_strides, n_tokens, n_heads, esz);
    a.n_tokens = n_tokens;
    a.D = head_dim;
    set_rope(a, rope, positions);
    DeviceScope dev(device_id);
    if (!dev.ok) return MUKV_ERR_HIP;
    return finished(mukv::launch_rope(a, dtype, reinterpret_cast<hipStream_t>(stream)));
}

int mukv_paged_append(const mukv_paged *pages, int32_t layer, const mukv_seqs *seqs, const void *k,
                      const mukv_strides *k_strides, const void *v, const mukv_strides *v_strides, const void *q,
                      const mukv_strides *q_strides, void *q_out, const mukv_strides *q_out_strides,
                      const mukv_rope_table *rope, const int32_t *positions, void *stream) {
    if (const int rc = check_pages(pages)) return rc;
    if (layer < 0 || layer >= pages->n_layers) return MUKV_ERR_INVALID_ARG;
    if (const int rc = check_seqs(pages, seqs, false, true)) return rc;
    const int esz = elem_size(pages->dtype), T = seqs->n_tokens;
    if (rope)
        if (const int rc = check_rope(rope, T == 0 || positions, pages->head_dim)) return rc;
    if (T == 0) return MUKV_OK; // (empty tensors need not have an address)
    if ((q != nullptr) != (q_out != nullptr)) return MUKV_ERR_INVALID_ARG;
    if (const int rc = check_rows(k, k_strides, T, pages->n_kv_heads, esz)) return rc;
    if (const int rc = check_rows(v, v_strides, T, pages->n_kv_heads, esz)) return rc;
    if (q) {
        if (const int rc = check_rows(q, q_strides, T, pages->n_q_heads, esz)) return rc;
        if (const int rc = check_rows(q_out, q_out_strides, T, pages->n_q_heads, esz)) return rc;
    }
    RopeArgs a = {};
    a.q = rows_in(q, q_strides, q_out, q_out_strides, T, pages->n_q_heads, esz);
    a.k = rows_in(k, k_strides, nullptr, nullptr, T, pages->n_kv_heads, esz);
    a.v = rows_in(v, v_strides, nullptr, nullptr, T, pages->n_kv_heads, esz);
    a.view = view_of(*pages, layer, *seqs);
    a.n_tokens = T;
    a.D = pages->head_dim;
    set_rope(a, rope, positions);
    DeviceScope dev(pages->device_id);
    if (!dev.ok) return MUKV_ERR_HIP;
    return finished(mukv::launch_rope(a, pages->dtype, reinterpret_cast<hipStream_t>(stream)));
}

int mukv_stream_capture(void *stream, uint64_t *id_out) {
    if (!id_out) return MUKV_ERR_INVALID_ARG;
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    unsigned long long id = 0;
    const hipError_t e = hipStreamGetCaptureInfo(reinterpret_cast<hipStream_t>(stream), &status, &id);
    *id_out = e == hipSuccess && status == hipStreamCaptureStatusActive ? id : 0;
    return finished(e);
}

static_assert(MUKV_PAGED_CLEAR == 4 * mukv::kPlanRecords, "the counts");
int mukv_paged_workspace_size(const mukv_paged *pages, const mukv_seqs *seqs, int32_t with_weights, int64_t *bytes_out) {
    if (!bytes_out || (with_weights != 0 && with_weights != 1)) return MUKV_ERR_INVALID_ARG;
    if (const int rc = check_pages(pages, packed_nothing(seqs))) return rc;
    if (const int rc = check_seqs(pages, seqs, true, true)) return rc;
    *bytes_out = space_of(*pages, *seqs, true, with_weights != 0).bytes;
    return MUKV_OK;
}

int mukv_paged_attend(const mukv_paged *pages, int32_t layer, const mukv_seqs *seqs, const void *q,
                      const mukv_strides *q_strides, int32_t causal, void *out, const mukv_row_weights *weights,
                      void *workspace, int64_t workspace_bytes, void *stream) {
    if (const int rc = check_pages(pages, packed_nothing(seqs))) return rc;
    if (layer < 0 || layer >= pages->n_layers || (causal != 0 && causal != 1)) return MUKV_ERR_INVALID_ARG;
    if (const int rc = check_seqs(pages, seqs, true, true)) return rc;
    if (weights)
        if (const int rc = check_weights(weights)) return rc;
    const int T = seqs->n_tokens, D = pages->head_dim, esz = elem_size(pages->dtype);
    if (T == 0 && (!weights || !seqs->table)) return MUKV_OK; // (packed, no sequence has a row that could have a weight)
    const mukv_strides dense = {0, D, (int64_t)D * pages->n_q_heads};
    const mukv_strides *qs = q_strides ? q_strides : &dense;
    if (T > 0) { // (empty tensors need not have an address)
        if (const int rc = check_rows(q, qs, T, pages->n_q_heads, esz)) return rc;
        if (!out) return MUKV_ERR_INVALID_ARG;
        if (!aligned(out)) return MUKV_ERR_UNSUPPORTED;
    }
    if (!workspace) return MUKV_ERR_INVALID_ARG;
    const Space x = space_of(*pages, *seqs, causal != 0, weights != nullptr);
    if (workspace_bytes < x.bytes) return MUKV_ERR_CAPACITY;
    if (!aligned(workspace)) return MUKV_ERR_UNSUPPORTED;
    mukv::PagedAttendArgs a = {};
    a.view = view_of(*pages, layer, *seqs);
    a.plan = x.plan;
    a.q = static_cast<const unsigned char *>(q);
    a.q_token = in_bytes(qs->token, T, esz);
    a.q_head = in_bytes(qs->head, pages->n_q_heads, esz);
    a.out = out;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    a.counts = reinterpret_cast<int *>(ws);
    a.records.stats = reinterpret_cast<float *>(ws + x.stats);
    a.records.values = reinterpret_cast<float *>(ws + x.values);
    a.records.sums = reinterpret_cast<float *>(ws + x.sums);
    a.pairs = weights ? reinterpret_cast<float *>(ws + x.pairs) : nullptr;
    a.scale_log2e = (float)(1.4426950408889634 / std::sqrt((double)D));
    a.causal = causal;
    if (weights) {
        a.weights_in = weights->in;
        a.weights_out = weights->out;
        a.weights_seq = weights->stride_seq;
        a.weights_head = weights->stride_head;
        a.weights_rows = weights->rows;
        a.decay = weights->decay;
    }
    DeviceScope dev(pages->device_id);
    if (!dev.ok) return MUKV_ERR_HIP;
    return finished(mukv::launch_paged_attend(a, D, pages->dtype, reinterpret_cast<hipStream_t>(stream)));
}

int mukv_paged_evict(const mukv_paged *pages, const mukv_seqs *seqs, const mukv_row_weights *weights, int32_t budget,
                     int32_t n_sink, int32_t n_recent, const int32_t *into_table, int32_t into_width,
                     int32_t *kept_out, int32_t *lengths_out, void *stream) {
    if (const int rc = check_pages(pages)) return rc;
    if (const int rc = check_seqs(pages, seqs, false, false)) return rc;
    if (!weights || !weights->in || !kept_out || !lengths_out) return MUKV_ERR_INVALID_ARG;
    mukv_row_weights w = *weights;
    w.decay = 0.f; // not read
    if (const int rc = check_weights(&w)) return rc;
    if (budget < 1 || n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > budget) return MUKV_ERR_INVALID_ARG;
    if (into_table && into_width < 1) return MUKV_ERR_INVALID_ARG;
    const int64_t lists = (int64_t)pages->n_layers * seqs->n_seqs * pages->n_kv_heads;
    if (lists > 0x7fffffff || (int64_t)into_width * seqs->n_seqs > 0x7fffffff || budget > 1 << 30) return MUKV_ERR_UNSUPPORTED;
    mukv::EvictArgs a = {};
    mukv_seqs s = *seqs;
    s.offsets = nullptr;
    s.n_tokens = s.max_new = 0;
    const int esz = elem_size(pages->dtype);
    a.view = view_of(*pages, 0, s);
    a.stride_layer = in_bytes(pages->stride_layer, pages->n_layers, esz);
    a.w_in = w.in;
    a.w_out = w.out;
    a.w_layer = w.stride_layer;
    a.w_seq = w.stride_seq;
    a.w_head = w.stride_head;
    a.w_rows = w.rows;
    a.budget = budget;
    a.n_sink = n_sink;
    a.n_recent = n_recent;
    a.into = into_table;
    a.into_width = into_width;
    a.kept = kept_out;
    a.lengths_out = lengths_out;
    DeviceScope dev(pages->device_id);
    if (!dev.ok) return MUKV_ERR_HIP;
    return finished(mukv::launch_paged_evict(a, pages->n_layers, pages->head_dim * esz, pages->device_id, reinterpret_cast<hipStream_t>(stream)));
}

} // extern "C"
