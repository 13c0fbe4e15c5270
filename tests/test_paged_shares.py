"""Even shares of one sequence's tiles, walked through on the host as the workgroups do: every step of every tile and KV head is somebody's
exactly once, a tile's chunks are numbered in their order, and no two tiles share a record."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <vector>
#include "paged_plan.h"
using namespace mukv;
#define CHECK(c) do { if (!(c)) { printf("line %d, trial %d: %s\n", __LINE__, trial, #c); return 1; } } while (0)
int main() {
    std::mt19937 rng(11);
    auto in = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    int walked = 0;
    for (int trial = 0; trial < 2000; ++trial) {
        PagedView v = {};
        PlanShape p = {};
        p.log_queries = in(7, 8); p.queries = 1 << p.log_queries; p.log_rows = 6; p.rows = 64; p.records = 704; p.most = 64; p.places = 256; p.start = 3;
        p.join = 0.8f; p.record = 0.06f; p.causal = in(0, 1);
        v.n_seqs = 1; v.G = in(1, 9); v.Hkv = in(1, 8); v.Hq = v.G * v.Hkv;
        v.page_rows = in(1, 128); v.table_width = in(1, 200); v.n_pages = 1;
        const int n_new = in(1, in(0, 3) ? 3000 : 90);
        int table = 0, length = in(0, 9) ? n_new + in(0, 12000) : in(-5, 100), off[2] = {0, n_new};
        v.table = &table; v.lengths = &length; v.offsets = off; v.n_tokens = n_new; v.per_seq = n_new;
        const SeqShape s = shape_of(v, p, 0);
        const uint32_t workers = in(0, 2) ? 256 : (uint32_t)in(1, 256), tiles = (uint32_t)(s.tiles * v.Hkv);
        if (tiles + workers > (uint32_t)p.records || (int64_t)tiles * s.blocks > kMostSteps) continue;
        std::vector<int> first(s.tiles + 1, 0);
        for (int t = 0; t < s.tiles; ++t) {
            const int n = steps_of_tile(v, p, s, t);
            CHECK(n >= 1 && n <= s.blocks);
            first[t + 1] = first[t] + n;
        }
        const uint32_t head = (uint32_t)first[s.tiles], line = head * (uint32_t)v.Hkv;
        if (line < workers) continue; // shared out by chunks
        ++walked;
        std::vector<char> seen(line, 0);
        std::map<int, int> owner;                        // of a record: its tile
        std::map<int, std::pair<int, int>> next;         // of a tile: chunks met, chunks
        for (uint32_t w = 0; w < workers; ++w)
            for (uint32_t at = stretch_of(w, workers, line), end = stretch_of(w + 1, workers, line); at < end;) {
                CHECK(worker_at(at, workers, line) == w && end <= line);
                const uint32_t g = at / head, step = at - g * head;
                int t = 0;
                while ((uint32_t)first[t + 1] <= step) ++t;
                const int n = first[t + 1] - first[t], lo = (int)step - first[t], hi = (uint32_t)(n - lo) < end - at ? n : lo + (int)(end - at);
                const uint32_t start = g * head + (uint32_t)first[t], w0 = worker_at(start, workers, line);
                const int chunks = (int)(worker_at(start + n - 1, workers, line) - w0) + 1, chunk = (int)(w - w0), id = (int)g * s.tiles + t;
                CHECK(chunk >= 0 && chunk < chunks && hi > lo);
                auto &x = next.insert({id, {0, chunks}}).first->second;
                CHECK(x.first++ == chunk && x.second == chunks);
                const int r = record_of(w0, id) + chunk;
                CHECK(r >= 0 && r < p.records && owner.insert({r, id}).second);
                for (int i = lo; i < hi; ++i) CHECK(seen[start + i]++ == 0);
                at += hi - lo;
            }
        for (uint32_t i = 0; i < line; ++i) CHECK(seen[i] == 1);
        CHECK(next.size() == tiles);
        for (auto &x : next) CHECK(x.second.first == x.second.second);
    }
    printf("%s\n", walked > 1000 ? "ok" : "too few");
    return 0;
}
'''


def test_every_step_is_somebodys(tmp_path):
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2605_22269_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr[-2000:]
