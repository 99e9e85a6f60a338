"""Where the tiles of scales of grouped rows lie (csrc/mx_format.cuh), compiled here by the C++ compiler with a trap on overflow of whole numbers: every
tile belongs to one group at most and has the rows that 64-bit arithmetic gives it, up to the largest number of rows that a plan accepts."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_13764_b200", "csrc")

PROGRAM = r"""
#define __host__
#define __device__
#include "mx_format.cuh"
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (rows %lld, groups %d, group %d, tile %lld)\n", __LINE__, #x, rows, groups, g, tile); return 1; } } while (0)
static unsigned long long state = 1;
static unsigned next() { state = state * 6364136223846793005ull + 1442695040888963407ull; return static_cast<unsigned>(state >> 33); }
static int check(long long rows, int groups) {
    static int off[1026];
    int g = 0;
    long long tile = 0;
    // loads: all rows in the first group, in the last, even ones, any
    for (int kind = 0; kind < 4; ++kind) {
        for (g = 0; g <= groups; ++g)
            off[g] = kind == 0 ? (g ? static_cast<int>(rows) : 0) : kind == 1 ? (g == groups ? static_cast<int>(rows) : 0)
                     : kind == 2 ? static_cast<int>(rows * g / groups) : static_cast<int>(next() % (rows + 1));
        if (kind == 3)
            for (int a = 1; a <= groups; ++a)
                for (int b = a; b > 0 && off[b - 1] > off[b]; --b) { const int t = off[b]; off[b] = off[b - 1]; off[b - 1] = t; }
        const long long tiles = rows / 128 + groups;
        for (int n = 0; n < 4000; ++n) {
            // the first and the last tiles, and some between
            tile = n < 1200 ? n : n < 2400 ? tiles - 1 - (n - 1200) : static_cast<long long>(next()) % tiles;
            if (tile < 0 || tile >= tiles) continue;
            int owners = 0;
            for (g = 0; g < groups; ++g) {
                const long long first = off[g] / 128 + g, at = tile - first, mine = static_cast<long long>(off[g + 1]) - off[g];
                const long long want = at < 0 || at * 128 >= mine ? 0 : mine - at * 128 < 128 ? mine - at * 128 : 128;
                CHECK(nk::mx_group_tile(off[g], g) == first);
                CHECK(nk::mx_tile_rows(static_cast<int>(at), static_cast<int>(mine)) == want);
                owners += want > 0;
            }
            CHECK(owners <= 1);
        }
    }
    return 0;
}
int main() {
    const long long most = (1ll << 31) - 4097;
    for (long long rows : {1ll, 127ll, 128ll, 129ll, 5000ll, 1000000ll, most - 131072, most})
        for (int groups : {1, 2, 37, 1024})
            if (check(rows, groups)) return 1;
    return 0;
}
"""


def test_a_tile_has_its_groups_rows(tmp_path):
    compiler = shutil.which("g++") or shutil.which("c++")
    if not compiler:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "tiles.cpp", tmp_path / "tiles"
    src.write_text(PROGRAM)
    subprocess.check_call([compiler, "-std=c++17", "-O1", "-ftrapv", "-Wall", "-I", CSRC, str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stdout or out.returncode
