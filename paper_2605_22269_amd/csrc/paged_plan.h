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

// ---- how an attention call is shared out ----
// A tile is `queries` (token, head of the KV group) pairs of one sequence; a unit is a tile, a KV head and a chunk of the sequence's
// rows, a whole number of blocks of `rows` each.  Every workgroup works the plan out for itself from lengths and offsets, so nothing
// about them has to be known on the host.
struct PlanShape {
    int queries, rows; // of a tile, of a block
    int target;        // units that are wanted; tiles come on top, since each has one unit at least
    int most;          // chunks of a sequence
};
MUKV_HD int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct SeqShape {
    int first, n_new, length, rows; // its first new token, how many, its length as its tokens count it, rows that exist
    int tiles, blocks;
};
MUKV_HD SeqShape shape_of(const PagedView &v, const PlanShape &p, int b) {
    SeqShape s;
    tokens_of(v, b, &s.first, &s.n_new);
    s.length = length_of(v, b, s.n_new);
    s.rows = rows_of(v, s.first, s.length);
    s.tiles = (int)div_up((int64_t)s.n_new * v.G, p.queries);
    s.blocks = s.rows > 0 ? (int)div_up(s.rows, p.rows) : 1; // (without rows a tile still has zeros to write)
    return s;
}
// Blocks of all tiles, what the chunks share out.
MUKV_HD double blocks_of(const PagedView &v, const SeqShape &s) { return (double)s.tiles * v.Hkv * s.blocks; }
// Blocks of a chunk, given those of the whole call.
MUKV_HD int chunk_of(const PlanShape &p, double all_blocks) {
    const int64_t per = div_up((int64_t)all_blocks, p.target);
    return per < 1 ? 1 : per > 0x40000000 ? 0x40000000 : (int)per;
}
MUKV_HD int chunk_of(const PlanShape &p, const SeqShape &s, int per) { // of one sequence: as many chunks, all about the same
    const int least = (int)div_up(s.blocks, p.most);
    return (int)div_up(s.blocks, div_up(s.blocks, per > least ? per : least));
}
MUKV_HD int chunks_of(const PlanShape &p, const SeqShape &s, int per) { return (int)div_up(s.blocks, chunk_of(p, s, per)); }
// Workgroups that cover every unit, and records: sum over sequences of tiles * ceil(blocks / per) is at most target + tiles, and where
// there are two chunks or more, at most twice target.
MUKV_HD int64_t units_bound(const PagedView &v, const PlanShape &p) {
    const int64_t with = v.n_seqs < v.n_tokens ? v.n_seqs : v.n_tokens;
    const int64_t tiles = ((int64_t)v.n_tokens * v.G / p.queries + with) * v.Hkv;
    const int64_t room = v.table ? room_of(v) : v.n_tokens; // (packed: a sequence has no more rows than there are tokens)
    int64_t chunks = div_up(room, p.rows);
    chunks = chunks > p.most ? p.most : chunks < 1 ? 1 : chunks;
    return tiles * chunks < tiles + p.target ? tiles * chunks : tiles + p.target;
}
MUKV_HD int records_bound(const PlanShape &p) { return 2 * p.target; }

} // namespace mukv
