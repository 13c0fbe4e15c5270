"""The plan of an attention call, walked through on the host: every tile, KV head and block of rows is somebody's exactly once, within the
workgroups and records that the host reckons with; rows, entries and tokens stay inside their arrays whatever lengths and offsets say."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <tuple>
#include <vector>
#include "paged_plan.h"
using namespace mukv;
#define CHECK(c) do { if (!(c)) { printf("line %d, trial %d: %s\n", __LINE__, trial, #c); return 1; } } while (0)
int main() {
    std::mt19937 rng(7);
    auto in = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    for (int trial = 0; trial < 3000; ++trial) {
        PagedView v = {};
        PlanShape p;
        const int kinds[3][7] = {{16, 128, 2048, 64, 512, 0, 0}, {16, 64, 2048, 64, 512, 0, 0}, {in(0, 1) ? 256 : 128, 64, 704, 64, 256, 3, 1}};
        const int *k = kinds[in(0, 2)];
        p.queries = k[0]; p.rows = k[1]; p.records = k[2]; p.most = k[3]; p.places = k[4]; p.start = k[5]; p.join = 0.8f * k[6]; p.record = 0.06f * k[6]; p.causal = in(0, 1);
        for (p.log_queries = 0; 1 << p.log_queries < p.queries;) ++p.log_queries;
        for (p.log_rows = 0; 1 << p.log_rows < p.rows;) ++p.log_rows;
        v.n_seqs = in(1, in(0, 3) ? 5 : 150);
        v.page_rows = in(1, 70); v.table_width = in(1, in(0, 4) ? 40 : 3000); v.n_pages = in(1, 500);
        v.G = in(1, 9); v.Hkv = in(1, 8); v.Hq = v.G * v.Hkv;
        const bool packed = in(0, 3) == 0, wild = in(0, 2) == 0, even = !packed && in(0, 2) == 0;
        std::vector<int> table((size_t)v.n_seqs * v.table_width), len(v.n_seqs), off(v.n_seqs + 1);
        int T = 0, each = in(0, 4);
        for (int b = 0; b < v.n_seqs; ++b) {
            off[b] = T;
            T += even ? each : in(0, 3) ? in(0, 4) : in(0, 900);
            len[b] = in(0, 5) ? in(0, v.table_width * v.page_rows) : in(0, 3);
            if (wild && in(0, 3) == 0) len[b] = in(0, 1) ? 0x7fffffff : -0x7fffffff - 1;
        }
        off[v.n_seqs] = T;
        v.n_tokens = T;
        v.per_seq = T / v.n_seqs;
        if (wild) for (int b = 0; b <= v.n_seqs; ++b) if (in(0, 9) == 0) off[b] = in(0, 1) ? in(-5, 2 * T) : (int)rng();
        v.table = packed ? nullptr : table.data(); v.lengths = len.data(); v.offsets = even ? nullptr : off.data();
        if (packed) { v.page_rows = T > 0 ? T : 1; v.n_pages = 1; }
        PlanSums all = {0, 0, 0, 0};
        for (int b = 0; b < v.n_seqs; ++b) {
            const PlanSums x = sums_of(v, p, shape_of(v, p, b));
            all.tiles += x.tiles; all.blocks += x.blocks; all.seen += x.seen;
            if (x.longest > all.longest) all.longest = x.longest;
        }
        int per = chunk_by_room(p, all);
        if (p.start) { // the least cost, as the lanes find it
            int best = 1;
            for (int c = 2; c <= p.most; ++c)
                if (cost_of(p, all, v.n_seqs == 1, c) < cost_of(p, all, v.n_seqs == 1, best)) best = c;
            per = best == 1 ? kWhole : div_up32((int)all.longest, best);
        }
        int64_t units = 0, records = 0, tokens = 0;
        for (int b = 0; b < v.n_seqs; ++b) {
            const SeqShape s = shape_of(v, p, b);
            CHECK(s.first >= 0 && s.n_new >= 0 && (int64_t)s.first + s.n_new <= v.n_tokens);
            CHECK(s.length >= 0 && s.rows >= 0 && s.rows <= s.length);
            if (packed) CHECK((int64_t)s.first + s.rows <= v.page_rows);
            if (!packed) CHECK(s.rows <= room_of(v));
            for (int j : {0, s.rows / 2, s.rows - 1})
                if (j >= 0 && j < s.rows && !packed) {
                    const int64_t e = entry_of(v, b, j);
                    CHECK(e >= (int64_t)b * v.table_width && e < (int64_t)(b + 1) * v.table_width);
                    v.stride_page = 1 << 20; v.stride_row = 16;
                    CHECK(offset_of(v, v.n_pages - 1, j) == (int64_t)(v.n_pages - 1) * (1 << 20) + 16 * (j % v.page_rows));
                }
            CHECK((int64_t)s.tiles * p.queries >= (int64_t)s.n_new * v.G && (int64_t)(s.tiles - 1) * p.queries < (int64_t)s.n_new * v.G);
            const int n = chunks_of(p, s, per), c = chunk_of(p, s, per);
            CHECK(c >= 1 && n >= 1 && n <= p.most && (int64_t)n * c >= s.blocks && (int64_t)(n - 1) * c < s.blocks);
            units += (int64_t)s.tiles * v.Hkv * n;
            if (n > 1) records += (int64_t)s.tiles * v.Hkv * n;
            tokens += s.n_new;
        }
        if (tokens <= v.n_tokens) { // (offsets out of order can name a token twice: the bound is for those that do not)
            CHECK(units <= units_bound(v, p));
        }
        CHECK(records <= p.records);
    }
    printf("ok\n");
    return 0;
}
'''


def test_every_unit_is_somebodys(tmp_path):
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2605_22269_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr[-2000:]
