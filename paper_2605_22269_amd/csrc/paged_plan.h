// Where the rows of a paged cache live: plain C++, the same on the device and on the host (where the tests walk through it).
#pragma once

#include <math.h>
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

// Whether sequence b's offsets ascend.  Where all of a call's do, no token is two sequences' (brought inside 0 .. n_tokens they still ascend), which
// units_bound reckons with: otherwise a tile's chunks could be more than there are workgroups, and those that ran would wait in the counts
// for the next call.
MUKV_HD bool offsets_fit(const PagedView &v, int b) { return !v.offsets || v.offsets[b] <= v.offsets[b + 1]; }

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
    int queries, rows; // of a tile, of a block: powers of two, 1 << log_queries and 1 << log_rows
    int log_queries, log_rows;
    int records;       // chunks that there is room for, of tiles with more than one
    int most;          // chunks of a tile
    int places;        // workgroups that are resident at once
    int start;         // what a unit costs before its first block, in blocks; 0: rows are all that has to move (chunk_by_room)
    float join, record; // what joining a chunk of a tile costs, and a chunk of any tile, in blocks
    int causal;
};
MUKV_HD int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
// (Numbers here stay so far below 2^31 that 32 bits hold the sums; a division of 64 bits is a quarter of a microsecond of instructions.)
MUKV_HD int div_up32(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1u) / (unsigned)b); }

struct SeqShape {
    int first, n_new, length, rows; // its first new token, how many, its length as its tokens count it, rows that exist
    int tiles, blocks;
};
MUKV_HD SeqShape shape_of(const PagedView &v, const PlanShape &p, int b) {
    SeqShape s;
    tokens_of(v, b, &s.first, &s.n_new);
    s.length = length_of(v, b, s.n_new);
    s.rows = rows_of(v, s.first, s.length);
    s.tiles = (s.n_new * v.G + p.queries - 1) >> p.log_queries;
    s.blocks = s.rows > 0 ? (int)(((unsigned)s.rows + p.rows - 1) >> p.log_rows) : 1; // (without rows a tile still has zeros to write)
    return s;
}

// Of all sequences: tiles (times KV heads), their blocks, those of them that are seen, and the most that a tile has.
struct PlanSums { // (32 bits: 10^-5 of a sum may be missing, which the room for records allows for)
    float tiles, blocks, seen, longest;
};
MUKV_HD PlanSums sums_of(const PagedView &v, const PlanShape &p, const SeqShape &s) {
    PlanSums x;
    x.tiles = (float)s.tiles * (float)v.Hkv;
    x.blocks = x.tiles * (float)s.blocks;
    const float late = p.causal ? 0.5f * (float)s.n_new / (float)p.rows : 0.f; // under the mask a tile misses half of the new rows in the mean
    x.seen = x.tiles * (late < (float)s.blocks - 1.f ? (float)s.blocks - late : 1.f);
    x.longest = s.tiles > 0 ? (float)s.blocks : 0.f;
    return x;
}
// What the call takes, in blocks, if the longest tile's rows are `chunks` chunks (1e30: there is no room for them).  Units of about
// the same size run `places` at a time.
MUKV_HD float cost_of(const PlanShape &p, const PlanSums &x, bool one_sequence, int chunks) {
    const float per = ceilf(x.longest / (float)chunks);
    float units = x.tiles;
    if (chunks > 1) {
        units = one_sequence ? x.tiles * (float)chunks : x.blocks / per + x.tiles;
        if (units * 1.001f > (float)p.records || (float)chunks > x.longest) return 1e30f;
    }
    const float rounds = ceilf(units / (float)p.places) * (x.seen / units + (float)p.start), last = per + (float)p.start;
    return (rounds > last ? rounds : last) + (chunks > 1 ? p.join * (float)chunks + p.record * units : 0.f);
}
constexpr int kWhole = 0x40000000; // blocks of a chunk: more than any tile has
// Blocks of a chunk where rows are all that has to move (start: 0).  Few tiles: eight blocks, which is enough to hide how a unit starts,
// or less where that leaves compute units without one; many: whole, unless they differ much, when the long ones are cut to half
// the mean.  (us a launch, blocks of 128 rows a chunk: 8 users of 8000 rows, 28/4 heads, 8 blocks 26.9, 4 28.1, 2 37; 64 users of
// 2000, 64/8 heads, whole 93, 8 blocks 104; 64 users of 200 to 12000, 30 blocks 199, 15 188, 8 187.)
// Room: the sum of ceil(blocks / per) over tiles with two chunks or more is at most twice that of blocks / per.
MUKV_HD int chunk_by_room(const PlanShape &p, const PlanSums &x) {
    const float least = ceilf(x.blocks * (2.002f / (float)p.records));
    float per;
    if (x.tiles < 256.f) {
        per = ceilf(x.blocks * (1.f / 256.f));
        per = per < 8.f ? per : 8.f;
    } else {
        if (x.longest * x.tiles <= 1.5f * x.blocks) return kWhole;
        per = ceilf(0.5f * x.blocks / x.tiles);
        per = per > 8.f ? per : 8.f;
    }
    per = per > least ? per : least;
    return per < 1.f ? 1 : per > (float)kWhole ? kWhole : (int)per;
}
MUKV_HD int chunk_of(const PlanShape &p, const SeqShape &s, int per) { // of one sequence: as many chunks, all about the same
    if (per >= s.blocks) return s.blocks;
    const int least = div_up32(s.blocks, p.most);
    return div_up32(s.blocks, div_up32(s.blocks, per > least ? per : least));
}
MUKV_HD int chunks_of(const PlanShape &p, const SeqShape &s, int per) {
    if (per >= s.blocks) return 1;
    return div_up32(s.blocks, chunk_of(p, s, per));
}
// ---- even shares ----
// One sequence whose tiles are about as many as there are compute units: chunks of a tile do not come out even (172 tiles in four chunks
// each are three rounds of 256 with a third of the last one empty).  There all steps of all tiles (a step is one block of rows of a tile and
// KV head, heads outermost) are one line, and `workers` workgroups take a stretch each, of one step more or less: the end of a
// tile, whole ones, the beginning of another.  There are no more workers than steps; 32 bits hold a line of up to kMostSteps.
constexpr uint32_t kMostSteps = 1u << 22;
MUKV_HD int steps_of_tile(const PagedView &v, const PlanShape &p, const SeqShape &s, int tile) {
    const int n_queries = s.n_new * v.G, end = (tile + 1) << p.log_queries, last_q = (end < n_queries ? end : n_queries) - 1;
    int rows = s.rows;
    if (p.causal) { // up to the last one that a query of the tile sees
        const int seen = s.length - s.n_new + last_q / v.G + 1;
        rows = seen < rows ? seen : rows;
    }
    return rows > 0 ? (int)(((unsigned)rows + p.rows - 1) >> p.log_rows) : 1;
}
MUKV_HD uint32_t stretch_of(uint32_t worker, uint32_t workers, uint32_t line) { return line * worker / workers; } // where its stretch begins
MUKV_HD uint32_t worker_at(uint32_t step, uint32_t workers, uint32_t line) { return ((step + 1) * workers - 1) / line; }
// The records of a tile start at this one: worker_at of its first step and its number (a tile's last worker is the next one's first at most).
MUKV_HD int record_of(uint32_t first_worker, int tile) { return (int)first_worker + tile; }
MUKV_HD float cost_of_shares(const PlanShape &p, float tiles, float line, float workers) {
    return ceilf(line / workers) + (float)p.start * (1.f + tiles / workers) + p.join * (1.f + workers / tiles) + p.record * (workers + tiles);
}
// Workgroups that cover every unit.
MUKV_HD int64_t units_bound(const PagedView &v, const PlanShape &p) {
    const int64_t with = v.n_seqs < v.n_tokens ? v.n_seqs : v.n_tokens;
    const int64_t tiles = ((int64_t)v.n_tokens * v.G / p.queries + with) * v.Hkv;
    const int64_t room = v.table ? room_of(v) : v.n_tokens; // (packed: a sequence has no more rows than there are tokens)
    int64_t chunks = div_up(room, p.rows);
    chunks = chunks > p.most ? p.most : chunks < 1 ? 1 : chunks;
    // with start: all units are within the records if any tile has two chunks; without: tiles of one chunk come on top
    const int64_t split = p.start ? (tiles > p.records ? tiles : p.records) : tiles + p.records;
    return tiles * chunks < split ? tiles * chunks : split;
}

} // namespace mukv
