"""Chunks whose results are left for a call's other launch, which has room for 64 of a tile: the plans of calls over shared rows as the host makes
them, shared out on the host as the workgroups do.  Groups may hold few of the call's tokens, and their rows may be long."""
from test_paged_shared_plan import run

SOURCE = r'''
#include <cstdio>
#include <random>
#include <vector>
#include "paged_plan.h"
using namespace mukv;
#define CHECK(c) do { if (!(c)) { printf("line %d, trial %d: %s\n", __LINE__, trial, #c); return 1; } } while (0)
int main() {
    std::mt19937 rng(23);
    auto in = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    int shared_out = 0, free_units = 0, by_chunks = 0;
    for (int trial = 0; trial < 40000; ++trial) {
        PagedView v = {};
        v.n_seqs = in(0, 3) ? 1 : in(2, 9);
        v.Hkv = in(1, 3); v.G = in(1, 9); v.Hq = v.G * v.Hkv;
        v.n_tokens = in(1, in(0, 3) ? 4000 : 200);
        v.page_rows = 64; v.table_width = in(0, 3) ? in(1500, 6500) : in(1, 300); v.n_pages = 1;
        std::vector<int> off(v.n_seqs + 1), len(v.n_seqs), table(v.n_seqs);
        const int most = in(0, 3) ? 60 : 4000;
        int at = in(0, 2) ? 0 : in(0, v.n_tokens), longest = 0;
        for (int b = 0; b <= v.n_seqs; ++b) {
            off[b] = at;
            const int n = in(0, most);
            at = at + n < v.n_tokens ? at + n : v.n_tokens;
        }
        for (int b = 0; b < v.n_seqs; ++b) {
            len[b] = in(0, 9) ? (int)room_of(v) - in(0, (int)room_of(v) / 4) : in(-3, 100);
            longest = off[b + 1] - off[b] > longest ? off[b + 1] - off[b] : longest;
        }
        v.table = table.data(); v.lengths = len.data(); v.offsets = off.data(); v.per_seq = v.n_tokens / v.n_seqs;
        const int64_t hint = in(0, 2) ? (longest > 0 ? longest : 1) : div_up(v.n_tokens, v.n_seqs);
        const int dims[3] = {64, 128, 32};
        const PlanShape p = shared_plan(v, in(0, 5) != 0, dims[in(0, 2)], hint, in(0, 1) != 0);
        CHECK(p.most <= kPlanChunks && p.records <= kPlanRecords && p.causal == 0);
        PlanSums all = {0, 0, 0, 0};
        for (int b = 0; b < v.n_seqs; ++b) {
            const PlanSums x = sums_of(v, p, shape_of(v, p, b));
            all.tiles += x.tiles; all.blocks += x.blocks; all.seen += x.seen;
            if (x.longest > all.longest) all.longest = x.longest;
        }
        int best = 1, per = chunk_by_room(p, all);
        if (p.start) { // the least cost, as the lanes find it
            for (int c = 2; c <= p.most; ++c)
                if (cost_of(p, all, v.n_seqs == 1, c) < cost_of(p, all, v.n_seqs == 1, best)) best = c;
            per = best == 1 ? kWhole : div_up32((int)all.longest, best);
        }
        int64_t units = 0, records = 0;
        for (int b = 0; b < v.n_seqs; ++b) {
            const SeqShape s = shape_of(v, p, b);
            const int n = chunks_of(p, s, per);
            CHECK(n >= 1 && n <= kPlanChunks);
            by_chunks += n == kPlanChunks;
            units += (int64_t)s.tiles * v.Hkv * n;
            records += n > 1 ? (int64_t)s.tiles * v.Hkv * n : 0;
        }
        CHECK(units <= units_bound(v, p) && records <= p.records);
        // one group's tiles may be a line, of which as many workgroups take a stretch as there are places for
        if (!p.start || !may_share(v, p)) continue;
        const SeqShape s = shape_of(v, p, 0);
        const uint32_t workers = (uint32_t)(p.places < units_bound(v, p) ? p.places : units_bound(v, p));
        const int64_t tiles = (int64_t)s.tiles * v.Hkv;
        if (tiles < 1 || tiles + workers > p.records || tiles * s.blocks > kMostSteps || !shares_fit(p, (uint32_t)tiles, workers)) continue;
        if (!(cost_of_shares(p, all.tiles, all.seen, (float)workers) < cost_of(p, all, true, best))) continue;
        uint32_t head = 0;
        for (int t = 0; t < s.tiles; ++t) head += (uint32_t)steps_of_tile(v, p, s, t);
        const uint32_t line = head * (uint32_t)v.Hkv;
        if (line < workers) continue;
        ++shared_out;
        free_units += p.units == 0;
        uint32_t start = 0;
        for (int g = 0; g < v.Hkv; ++g)
            for (int t = 0; t < s.tiles; ++t) {
                const uint32_t n = (uint32_t)steps_of_tile(v, p, s, t), first = worker_at(start, workers, line), last = worker_at(start + n - 1, workers, line);
                CHECK(last - first + 1 <= kPlanChunks);
                CHECK(record_of(first, g * s.tiles + t) + (int)(last - first) < p.records);
                start += n;
            }
        CHECK(start == line);
    }
    printf("%s\n", shared_out > 500 && free_units > 100 && by_chunks > 100 ? "ok" : "too few");
    if (!(shared_out > 500 && free_units > 100 && by_chunks > 100)) printf("%d %d %d\n", shared_out, free_units, by_chunks);
    return 0;
}
'''


def test_no_tile_is_left_in_more_chunks_than_are_taken(tmp_path):
    run(tmp_path, SOURCE)
