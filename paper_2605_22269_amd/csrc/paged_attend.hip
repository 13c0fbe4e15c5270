// Which kernel takes an attention call, and those for rows of the payload type.
#include "paged_attend_dev.h"

namespace mukv {

// Which kernel takes a call, by what is known on the host; us a call, 28/4 heads of 128, what the rule takes marked.
// The kernel for any shape reads a sequence's rows once for every 16 queries of a KV head, the one for prompts once for 128 or 256, but its
// units are large and start slowly: it takes calls with more queries than that (any / prompts in tiles of 128 / of 256: one user, 16 tokens
// over 8000 rows 19.5* / 34 / 50, over 32000 59* / 58 / 87, 32 tokens over 8000 28.6* / 35 / 51, 64 tokens over 8000 52 / 36 / 52*, over 1000
// 14.0 / 19.5* / 28.8; 8 users over 8000 rows, 4 tokens 31.5* / 42 / 61, 8 tokens 55 / 42* / 61, 16 tokens 89 / 43* / 62).
// Tiles of 128 or of 256 queries: the wide ones read operands for twice the products, so they are faster where there is enough to
// do for every compute unit, and slower where a tile is half empty or the last tiles' rows are what the call waits for (128 / 256: 6
// users, 16 tokens over 3000 to 9000 rows 39* / 56; 300 tokens 14.6* / 20.2; 2000 tokens 55* / 71; 8192 tokens 650 / 493*; 1568 over 6272 rows
// 277 / 238*; 8 users, 64 tokens over 8000 rows 135 / 101*).  What a table has room for stands in for the rows that are there, which the
// host does not know: one user's 64 tokens over 8000 rows are the case above where that takes the slower tile.
int paged_prompt_tile(const PagedView &v, int dtype, int D, int64_t new_hint) {
    if (dtype != MUKV_BF16 || D < 64) return 0;
    const int64_t queries = new_hint * v.G; // of a sequence and KV head
    if (queries < 48 || (int64_t)v.n_tokens * v.Hq < 1500) return 0;
    const int64_t room = v.table ? room_of(v) : new_hint, tiles = div_up(queries, 256) * v.n_seqs * v.Hkv;
    return queries <= 128 || (tiles <= 256 && room <= 4096) ? 128 : 256;
}

PlanShape paged_plan(int dtype, int prompt_tile, bool causal, bool eight) {
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
        p.rows = dtype == MUKV_BF16 || eight ? 128 : 64; // a block of every wave
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
// us a call, what the rule takes marked (any / prompts in tiles of 128 / of 256): 8 users over 6272 rows, 28/4 heads of 128, 27.3* / 31.8 / 41.6; 16 over
// 500 18.1* / 20.9 / 27.1; 48 users in three rooms of 2113 to 6272 45.7 / 40.5* / 55.2; 64 in eight rooms 57.3 / 42.7* / 60.5; 64 users, 64/8 heads,
// over 10000 rows in 8 bits 111 / 57* / 65, over 40000 408 / 175 / 171*; 718 tokens over 6272, 28/4 heads, 303 / 127 / 118*.
// Workgroups without a unit still have to start, after all that have one.  Few tiles: no more units than places, or one group's tiles
// shared out step by step, which leaves no place without work either (the last two cases above: 171.6 and 121.8 with 704 units).
PlanShape shared_plan(const PagedView &groups, int dtype, int D, int64_t new_hint, bool eight) {
    const int64_t queries = new_hint * groups.G, tiles256 = div_up(queries, 256) * groups.n_seqs * groups.Hkv;
    int tile = 0;
    if (dtype == MUKV_BF16 && D >= 64 && queries >= 48 && (int64_t)groups.n_tokens * groups.Hq >= 1000)
        tile = queries > 128 && tiles256 * div_up(room_of(groups), 64) > 24 * 256 ? 256 : 128;
    PlanShape p = paged_plan(dtype, tile, false, eight);
    if (!tile) return p;
    p.join = 0.2f; // (the other launch's, shared by more workgroups)
    p.record = 0.02f;
    const int64_t tiles = tiles_bound(groups, p);
    if (tiles > p.places / 2) return p;
    p.units = p.places + 8;
    p.records = p.places + 8 + (int)tiles;
    return p;
}

hipError_t launch_paged_attend(const PagedAttendArgs &a, int D, int dtype, hipStream_t st) {
    return dtype == MUKV_BF16 ? launch_by_dim<uint16_t, false, false>(a, D, st) : launch_by_dim<float, false, false>(a, D, st);
}
hipError_t launch_paged_weights(const PagedAttendArgs &a, int D, bool bf16, hipStream_t st) {
    return bf16 ? launch_weights_by_dim<uint16_t, false>(a, D, st) : launch_weights_by_dim<float, false>(a, D, st);
}

} // namespace mukv
