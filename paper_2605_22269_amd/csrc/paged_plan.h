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

// Of a cache in 8 bits: where the powers of two of one layer's rows are, a byte each.
struct ScaleView {
    unsigned char *k, *v;
    int64_t stride_page, stride_head, stride_row;
};

// One layer of a paged cache and the sequences that lie in it.  Strides in bytes.
struct PagedView {
    unsigned char *k, *v; // the layer's
    int64_t stride_page, stride_head, stride_row;
    const int32_t *table, *lengths, *offsets;
    int n_pages, page_rows, n_seqs, table_width, n_tokens, per_seq; // per_seq: new tokens each, where there are no offsets
    int Hq, Hkv, G;
    ScaleView scales; // rows in 8 bits
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
MUKV_HD int64_t scale_offset_of(const PagedView &v, int page, int j) { // of its scales
    return (int64_t)page * v.scales.stride_page + (int64_t)((unsigned)j % (unsigned)v.page_rows) * v.scales.stride_row;
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
    int units = 0; // units there are workgroups for, where a tile has two chunks or more (0: as many as records)
    bool left = false; // chunks are left for another launch, which has room for those of a tile up to `most` (as where units is set)
};
MUKV_HD int most_units(const PlanShape &p) { return p.units ? p.units : p.records; }
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
        if (units * 1.001f > (float)most_units(p) || (float)chunks > x.longest) return 1e30f;
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
// Whether a tile is in no more than p.most stretches, where that matters (what is left of shared rows is read again by their number, and by a launch
// that holds what each is multiplied by): a tile of a line of equal ones meets the starts of workers / tiles stretches, rounded up, and one
// more, and may begin inside another.  tiles: those that there are, of which a group that has few of a call's tokens has few.
MUKV_HD bool shares_fit(const PlanShape &p, uint32_t tiles, uint32_t workers) {
    return !(p.left || p.units) || tiles * (uint32_t)(p.most - 2) >= workers;
}
// Workgroups that cover every unit.
MUKV_HD int64_t tiles_bound(const PagedView &v, const PlanShape &p) {
    const int64_t with = v.n_seqs < v.n_tokens ? v.n_seqs : v.n_tokens;
    return ((int64_t)v.n_tokens * v.G / p.queries + with) * v.Hkv;
}
MUKV_HD int64_t units_bound(const PagedView &v, const PlanShape &p) {
    // (without offsets all have as many tokens; workgroups without a unit are not free: 200 users' tokens over 10 to 400 rows, 64/8 heads of 128 in
    // 8 bits, 58.0 us a call with room for 2048 chunks, 50.1 for half of them, 44.9 without offsets and 39.8 with the tiles that there are)
    const int64_t tiles = v.offsets ? tiles_bound(v, p) : (int64_t)v.n_seqs * v.Hkv * div_up((int64_t)v.per_seq * v.G, p.queries);
    const int64_t room = v.table ? room_of(v) : v.n_tokens; // (packed: a sequence has no more rows than there are tokens)
    int64_t chunks = div_up(room, p.rows);
    chunks = chunks > p.most ? p.most : chunks < 1 ? 1 : chunks;
    // with start: all units are within the records if any tile has two chunks; without: a tile's chunks are less than one more than its blocks by
    // those of a chunk, of which there are at most records / 2.002 (chunk_by_room)
    const int64_t split = p.start ? (tiles > most_units(p) ? tiles : most_units(p)) : tiles + p.records / 2 + 1;
    return tiles * chunks < split ? tiles * chunks : split;
}

// ---- which kernel takes a call, and its plan: by types and sizes that the host knows ----
constexpr int kPlanChunks = 64;     // most chunks of a sequence
constexpr int kPlanRecords = 2048;  // most that any plan has: the counts at a workspace's start
constexpr int kPQ = 16;             // queries of a tile of the kernel for any shape
// An attention call's kernel: 0 that for any shape, otherwise the one for prompts, with tiles of so many queries.  new_hint: new tokens of a sequence,
// as far as that is known.  (Times: us a call, 28/4 heads of 128, what the rule takes marked.)
// The kernel for any shape reads a sequence's rows once for every 16 queries of a KV head, the one for prompts once for 128 or 256, but its
// units are large and start slowly: it takes calls with more queries than that (any / prompts in tiles of 128 / of 256: one user, 16 tokens
// over 8000 rows 19.5* / 34 / 50, over 32000 59* / 58 / 87, 32 tokens over 8000 28.6* / 35 / 51, 64 tokens over 8000 52 / 36 / 52*, over 1000
// 14.0 / 19.5* / 28.8; 8 users over 8000 rows, 4 tokens 31.5* / 42 / 61, 8 tokens 55 / 42* / 61, 16 tokens 89 / 43* / 62).
// Tiles of 128 or of 256 queries: the wide ones read operands for twice the products, so they are faster where there is enough to
// do for every compute unit, and slower where a tile is half empty or the last tiles' rows are what the call waits for (128 / 256: 6
// users, 16 tokens over 3000 to 9000 rows 39* / 56; 300 tokens 14.6* / 20.2; 2000 tokens 55* / 71; 8192 tokens 650 / 493*; 1568 over 6272 rows
// 277 / 238*; 8 users, 64 tokens over 8000 rows 135 / 101*).  What a table has room for stands in for the rows that are there, which the
// host does not know: one user's 64 tokens over 8000 rows are the case above where that takes the slower tile.
inline int paged_prompt_tile(const PagedView &v, bool bf16, int D, int64_t new_hint) {
    if (!bf16 || D < 64) return 0;
    const int64_t queries = new_hint * v.G; // of a sequence and KV head
    if (queries < 48 || (int64_t)v.n_tokens * v.Hq < 1500) return 0;
    const int64_t room = v.table ? room_of(v) : new_hint, tiles = div_up(queries, 256) * v.n_seqs * v.Hkv;
    return queries <= 128 || (tiles <= 256 && room <= 4096) ? 128 : 256;
}

inline PlanShape paged_plan(bool bf16, int prompt_tile, bool causal, bool eight) {
    PlanShape p;
    p.causal = causal;
    p.most = kPlanChunks;
    if (prompt_tile) {
        p.queries = prompt_tile;
        p.rows = 64; // a step of the workgroup
        p.records = 704;
        p.places = 256;
        p.start = 3;
        p.join = 0.8f;
        p.record = 0.06f;
    } else {
        p.queries = kPQ;
        p.rows = bf16 || eight ? 128 : 64; // a block of every wave
        p.records = 2048;
        p.places = 512;
        p.start = 0;
        p.join = p.record = 0.f;
    }
    p.log_queries = p.queries == 256 ? 8 : p.queries == 128 ? 7 : 4;
    p.log_rows = p.rows == 128 ? 7 : 6;
    return p;
}

// Which kernel takes rows that groups share, and its plan: chunks are left, not joined, so that tiles are better small and many units cheap.
// us a call, single tokens over 20 to 900 rows of their own too, what the rule takes marked (any / prompts in tiles of 128 / of 256): 8 users over
// 6272 rows, 28/4 heads of 128, 27.1* / 32.1 / 37.7; 16 over 500 20.7* / 26.1 / 29.6; 48 users in three rooms of 2113 to 6272 44.9 / 39.9* / 46.7;
// 64 in eight rooms 62.5 / 46.7* / 57.2; 64 users of 100 to 3000 rows, 64/8 heads, over 10000 rows in 8 bits 153 / 86.7* / 90.9, over 40000
// 470 / 173 / 151*; 718 tokens of prompts over 6272, 28/4 heads, 305 / 126 / 106*.
// Workgroups without a unit still have to start, after all that have one.  Few tiles: no more units than places, or one group's tiles
// shared out step by step, which leaves no place without work either (the last two cases above: 153 and 110 with 704 units).
inline PlanShape shared_plan(const PagedView &groups, bool bf16, int D, int64_t new_hint, bool eight) {
    const int64_t queries = new_hint * groups.G, tiles256 = div_up(queries, 256) * groups.n_seqs * groups.Hkv;
    int tile = 0;
    if (bf16 && D >= 64 && queries >= 48 && (int64_t)groups.n_tokens * groups.Hq >= 1000)
        tile = queries > 128 && tiles256 * div_up(room_of(groups), 64) > 24 * 256 ? 256 : 128;
    PlanShape p = paged_plan(bf16, tile, false, eight);
    p.left = true;
    if (!tile) return p;
    p.join = 0.2f; // (the other launch's, shared by more workgroups)
    p.record = 0.02f;
    const int64_t tiles = tiles_bound(groups, p);
    if (tiles > p.places / 2) return p;
    p.units = p.places + 8;
    p.records = p.places + 8 + (int)tiles;
    return p;
}
// Workgroups that share a list's rows, `per` at a time, where weights of rows are worked out.  They go round: a table is often wider than its
// sequences.  A round is at most 2^20 rows, so that the number of a workgroup's next row behind a sequence of 2^31 - 2^20 of them, the most there are,
// is still one of 32 bits.
MUKV_HD int weight_groups(int64_t rows, int per, int64_t lists) {
    int64_t most = 8192 / lists;
    if (most < 16) most = 16;
    if (most > (1 << 20) / per) most = (1 << 20) / per;
    const int64_t groups = div_up(rows, per);
    return (int)(groups < most ? groups : most);
}
// Whether one sequence's tiles may be shared out evenly: to look at that takes the kernel a microsecond, so not where it gains nothing:
// few tiles, which come out even in chunks, more than twice the compute units, or few rows (us a launch without / with, 28/4 heads of 128:
// 200 tokens over 20000 rows 89 / 93, 300 alone 14.5 / 15.6, 1000 29.8 / 31.0, 2000 55.0 / 57.3; the gains are at the kernel).
inline bool may_share(const PagedView &v, const PlanShape &p) {
    if (p.units) return v.n_seqs == 1; // shared rows of one group
    const int64_t tiles = div_up((int64_t)v.n_tokens * v.G, p.queries) * v.Hkv, room = v.table ? room_of(v) : v.n_tokens;
    return v.n_seqs == 1 && tiles > 64 && tiles <= p.records - p.places && room >= 4096;
}

} // namespace mukv
