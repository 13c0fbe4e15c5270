"""The plan of attention over shared rows, whose chunks are left where the next launch finds them: places for all of them, workgroups for every
unit, no tile in more chunks than are read again."""
import os
import subprocess

import test_paged_plan
import test_paged_shares

ROOT = test_paged_plan.ROOT


def run(tmp_path, source):
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(source)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2605_22269_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr[-2000:]


def replaced(source, *pairs):
    for old, new in pairs:
        assert source.count(old) == 1, old
        source = source.replace(old, new)
    return source


def test_units_and_records_are_as_many_as_the_host_reckons_with(tmp_path):
    run(tmp_path, replaced(
        test_paged_plan.SOURCE,
        ("const int *k = kinds[in(0, 2)];", "const int *k = kinds[2];"),
        ("p.causal = in(0, 1);", "p.causal = 0;"),
        ("const bool packed = in(0, 3) == 0,", "const bool packed = false,"),
        ("        PlanSums all = {0, 0, 0, 0};", """        p.join = 0.2f, p.record = 0.02f;
        if (tiles_bound(v, p) <= p.places / 2) { p.units = p.places + 8; p.records = p.places + 8 + (int)tiles_bound(v, p); }
        PlanSums all = {0, 0, 0, 0};"""),
        ("        if (tokens <= v.n_tokens) {", "        if (tokens <= v.n_tokens && p.units) CHECK(units <= (tiles_bound(v, p) > p.units ? tiles_bound(v, p) : p.units));\n        if (tokens <= v.n_tokens) {")))


def test_no_tile_is_in_more_stretches_than_are_read_again(tmp_path):
    run(tmp_path, replaced(
        test_paged_shares.SOURCE,
        ("p.causal = in(0, 1);", "p.causal = 0;"),
        ("in(0, 3) ? 3000 : 90)", "in(0, 1) ? 1500 : 60)"),
        ("in(0, 9) ? n_new + in(0, 12000) : in(-5, 100)", "in(0, 9) ? in(0, 1) ? in(1, 3000) : in(3000, 200000) : in(-5, 100)"),
        ("v.page_rows = in(1, 128); v.table_width = in(1, 200);", "v.page_rows = 128; v.table_width = in(1, 2000);"),
        ("        const uint32_t workers = in(0, 2) ? 256 : (uint32_t)in(1, 256),", "        p.units = 264; p.records = 264 + (int)tiles_bound(v, p);\n        const uint32_t workers = 256,"),
        ("        if (line < workers) continue;", "        if (line < workers || !shares_fit(p, tiles, workers)) continue;"),
        ("                CHECK(chunk >= 0 && chunk < chunks && hi > lo);", "                CHECK(chunk >= 0 && chunk < chunks && hi > lo && chunks <= p.most);"),
        ("walked > 1000", "walked > 500")))
