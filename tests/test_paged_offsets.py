"""Offsets against the rule: what the plan reckons with holds wherever offsets_fit says so of every sequence, whatever they are otherwise."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include <cstdio>
#include <random>
#include <vector>
#include "paged_plan.h"
using namespace mukv;
#define CHECK(c) do { if (!(c)) { printf("line %d, trial %d: %s\n", __LINE__, trial, #c); return 1; } } while (0)
int64_t units_of(const PagedView &v, const PlanShape &p) {
    PlanSums all = {0, 0, 0, 0};
    for (int b = 0; b < v.n_seqs; ++b) {
        const PlanSums x = sums_of(v, p, shape_of(v, p, b));
        all.tiles += x.tiles; all.blocks += x.blocks; all.seen += x.seen;
        if (x.longest > all.longest) all.longest = x.longest;
    }
    int per = chunk_by_room(p, all);
    if (p.start) {
        int best = 1;
        for (int c = 2; c <= p.most; ++c)
            if (cost_of(p, all, v.n_seqs == 1, c) < cost_of(p, all, v.n_seqs == 1, best)) best = c;
        per = best == 1 ? kWhole : div_up32((int)all.longest, best);
    }
    int64_t units = 0;
    for (int b = 0; b < v.n_seqs; ++b) {
        const SeqShape s = shape_of(v, p, b);
        units += (int64_t)s.tiles * v.Hkv * chunks_of(p, s, per);
    }
    return units;
}
int main() {
    std::mt19937 rng(3);
    auto in = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    int fits = 0, too_many = 0, trial = 0;
    for (; trial < 20000; ++trial) {
        PagedView v = {};
        PlanShape p = {};
        const bool prompt = in(0, 1);
        p.log_queries = prompt ? in(7, 8) : 4; p.queries = 1 << p.log_queries; p.log_rows = prompt ? 6 : 7; p.rows = 1 << p.log_rows;
        p.records = prompt ? 704 : 2048; p.most = 64; p.places = prompt ? 256 : 512; p.start = prompt ? 3 : 0;
        p.join = prompt ? 0.8f : 0.f; p.record = prompt ? 0.06f : 0.f; p.causal = in(0, 1);
        v.n_seqs = in(1, in(0, 3) ? 5 : 130); v.n_tokens = in(0, in(0, 2) ? 60 : 2000); v.G = in(1, 9); v.Hkv = in(1, 8); v.Hq = v.G * v.Hkv;
        v.page_rows = 16; v.table_width = in(1, 400); v.n_pages = 1; v.per_seq = v.n_tokens / v.n_seqs;
        int table = 0;
        std::vector<int> len(v.n_seqs), off(v.n_seqs + 1);
        const int kind = in(0, 3);
        for (int b = 0; b <= v.n_seqs; ++b) off[b] = kind == 0 ? (int)rng() : kind == 1 ? in(-2, v.n_tokens + 2) : kind == 2 ? (b % 2 ? v.n_tokens : 0) : in(0, v.n_tokens);
        if (in(0, 1)) for (int b = 1; b <= v.n_seqs; ++b) if (off[b] < off[b - 1]) off[b] = off[b - 1];
        for (int b = 0; b < v.n_seqs; ++b) len[b] = in(0, in(0, 2) ? 300 : v.table_width * 16);
        v.table = &table; v.lengths = len.data(); v.offsets = off.data();
        bool fit = true;
        for (int b = 0; b < v.n_seqs; ++b) fit = fit && offsets_fit(v, b);
        const int64_t units = units_of(v, p), bound = units_bound(v, p);
        CHECK(units >= 0 && bound >= 0);
        if (fit || v.n_seqs == 1) CHECK(units <= bound); // (one sequence's tokens are brought inside, and that is all)
        fits += fit;
        too_many += units > bound;
    }
    // a call that would leave counts behind: three sequences, the last one's tile 13 would have two of its three chunks
    PagedView v = {};
    PlanShape p = {16, 128, 4, 7, 2048, 64, 512, 0, 0.f, 0.f, 1};
    int table = 0, len[3] = {128, 50, 384}, off[4] = {0, 32, 0, 32};
    v.n_seqs = 3; v.n_tokens = 32; v.G = v.Hq = 8; v.Hkv = 1; v.page_rows = 16; v.table_width = 24; v.n_pages = 1;
    v.table = &table; v.lengths = len; v.offsets = off;
    CHECK(units_of(v, p) == 64 && units_bound(v, p) == 57);
    CHECK(offsets_fit(v, 0) && !offsets_fit(v, 1) && offsets_fit(v, 2));
    off[1] = off[2] = 0;
    CHECK(offsets_fit(v, 0) && offsets_fit(v, 1) && offsets_fit(v, 2) && units_of(v, p) <= units_bound(v, p));
    printf("%s\n", fits > 1000 && too_many > 100 ? "ok" : "too few");
    return 0;
}
'''


def test_units_stay_within_the_workgroups_wherever_offsets_fit(tmp_path):
    src, exe = tmp_path / "offsets.cpp", tmp_path / "offsets"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2605_22269_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr[-2000:]
