// Where the rows of a paged cache live: plain C++, the same on the device and on the host (where the tests walk through it).
#pragma once

#include <stdint.h>

#if defined(__HIP__)
#define MUKV_HD __host__ __device__ __forceinline__
#else
#define MUKV_HD inline
#endif

namespace mukv {

// One layer of a paged cache and the sequences that lie in it.  Strides in bytes.
struct PagedView {
    unsigned char *k, *v; // the layer's
    int64_t stride_page, stride_head, stride_row;
    const int32_t *table, *lengths, *offsets;
    int n_pages, page_rows, n_seqs, table_width, n_tokens, per_seq; // per_seq: new tokens each, where there are no offsets
    int Hq, Hkv, G;
};

// The new tokens of sequence b: first and number, both inside 0 .. n_tokens whatever the offsets say.
MUKV_HD void tokens_of(const PagedView &v, int b, int *first, int *count) {
    int lo = b * v.per_seq, hi = lo + v.per_seq;
    if (v.offsets) {
        lo = v.offsets[b];
        hi = v.offsets[b + 1];
    }
    lo = lo < 0 ? 0 : lo > v.n_tokens ? v.n_tokens : lo;
    hi = hi < lo ? lo : hi > v.n_tokens ? v.n_tokens : hi;
    *first = lo;
    *count = hi - lo;
}

// Rows the table has room for.
MUKV_HD int64_t room_of(const PagedView &v) { return (int64_t)v.table_width * v.page_rows; }

// Length of sequence b as its tokens count it, and the rows of it that exist (a table of more than 2^31-1 rows is refused on the host).
MUKV_HD int length_of(const PagedView &v, int b, int n_new) {
    if (!v.table) return n_new; // packed: the tokens' own rows
    const int n = v.lengths[b];
    return n < 0 ? 0 : n;
}
MUKV_HD int rows_of(const PagedView &v, int first_token, int length) {
    const int room = v.table ? (int)room_of(v) : first_token < v.page_rows ? v.page_rows - first_token : 0;
    return length < room ? length : room;
}

// The entry of the table that names row j's page; j inside 0 .. room_of.
MUKV_HD int64_t entry_of(const PagedView &v, int b, int j) { return (int64_t)b * v.table_width + (int)((unsigned)j / (unsigned)v.page_rows); }

// Byte offset of row j (KV head 0) on page `page`, which the caller has found to be one of the pages.
MUKV_HD int64_t offset_of(const PagedView &v, int page, int j) {
    return (int64_t)page * v.stride_page + (int64_t)((unsigned)j % (unsigned)v.page_rows) * v.stride_row;
}
MUKV_HD bool is_page(const PagedView &v, int page) { return (unsigned)page < (unsigned)v.n_pages; }

} // namespace mukv
