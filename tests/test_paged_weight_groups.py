"""How rows are dealt to the workgroups that work out their weights, as they go round: every row is somebody's once, and no number passes 32 bits."""
from test_paged_shared_plan import run

SOURCE = r'''
#include <climits>
#include <cstdio>
#include <random>
#include <vector>
#include "paged_plan.h"
using namespace mukv;
#define CHECK(c) do { if (!(c)) { printf("line %d, trial %d: %s\n", __LINE__, trial, #c); return 1; } } while (0)
int main() {
    std::mt19937 rng(3);
    auto in = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    const int64_t most_rows = 0x7ff00000; // of a sequence: more are refused
    for (int trial = 0; trial < 4000; ++trial) {
        const int pers[4] = {32, 64, 128, 256}, per = pers[in(0, 3)];
        const int64_t lists = in(0, 1) ? 1 : in(1, in(0, 1) ? 64 : 65536);
        const int64_t rows = in(0, 3) ? in(0, 40000) : most_rows - in(0, 1) * (int64_t)in(0, 3000000);
        const int groups = weight_groups(rows, per, lists);
        CHECK(groups >= 0 && (groups >= 1) == (rows > 0));
        // a workgroup's next rows follow its last ones, groups * per on
        CHECK(rows == 0 || rows - 1 + (int64_t)groups * per <= INT_MAX);
        if (rows > 100000) continue;
        std::vector<char> seen(rows, 0);
        for (int w = 0; w < groups; ++w)
            for (int r0 = w * per; r0 < rows; r0 += groups * per)
                for (int r = r0; r < r0 + per && r < rows; ++r) CHECK(seen[r]++ == 0);
        for (char s : seen) CHECK(s == 1);
    }
    printf("ok\n");
    return 0;
}
'''


def test_rows_are_dealt_within_32_bits(tmp_path):
    run(tmp_path, SOURCE)
