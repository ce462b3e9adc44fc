"""The list of cut row tiles of the attention over the paged cache (csrc/prefix_split.h), on the
host: each row tile that the CTAs' ranges cut has an entry of its own inside the list, and a
block of the joining launch that reads it."""
import shutil
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2608_11742_gb300" / "csrc"

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "prefix_split.h"
using namespace rps::prefix;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (%d row tiles, %d SMs)\n", __LINE__, #x, row_tiles, sms); return 1; } } while (0)

int main(int argc, char **argv) {
    std::mt19937 g(std::atoi(argv[1]));
    const auto rnd = [&](int lo, int hi) { return lo + static_cast<int>(g() % static_cast<unsigned>(hi - lo + 1)); };
    long cut_tiles = 0;
    for (int row_tiles = 1; row_tiles <= 400; row_tiles += row_tiles < 140 || row_tiles > 175 ? rnd(1, 9) : 1)
        for (int sms : {1, 7, 132, 148, 150, 151, 152, 153, 159, 160, 188})
            for (int trial = 0; trial < 12; ++trial) {
                // row tiles alike, of random lengths, or with some that have no key tile
                std::vector<Tiles> t(row_tiles);
                const Tiles one{rnd(0, 30), rnd(0, 30)};
                for (auto &x : t) {
                    x = trial % 3 ? Tiles{rnd(0, 4), rnd(0, 40)} : one;
                    if (trial % 4 == 1 && rnd(0, 5) == 0) x = Tiles{0, 0};
                    if (trial % 4 == 2 && &x - t.data() > row_tiles - 10) x.own += 300;
                }
                int64_t work = 0, most = 0;
                for (auto &x : t) work += cost_of(x), most += x.shared + x.own;
                if (!work) continue;
                const int ctas = static_cast<int>(std::min<int64_t>({sms, kMaxCtas, row_tiles * (most + 2)}));
                const int n = static_cast<int>(std::min<int64_t>(ctas, std::max<int64_t>(1, work / kWidest)));
                const Ranges ranges = make_ranges(work, n);
                const CutList list = cut_list(row_tiles, ctas);
                CHECK(list.blocks >= 1 && list.blocks <= kMaxCtas);  // entries of the workspace
                std::vector<int> entry(list.blocks, 0);
                int64_t start = 0;
                for (int k = 0; k < row_tiles; ++k) {
                    int parts = 0, first = -1;
                    for (int c = 0; c < n; ++c) {
                        const int lo = reach(t[k], range_start(ranges, c) - start), hi = reach(t[k], range_start(ranges, c + 1) - start);
                        if (hi <= lo) continue;
                        if (!parts++) first = c;
                    }
                    start += cost_of(t[k]);
                    if (parts < 2) continue;
                    const int at = list.by_tile ? k : first;
                    CHECK(at < list.blocks);        // a block joins it
                    CHECK(entry[at]++ == 0);        // and no other
                    ++cut_tiles;
                }
            }
    if (cut_tiles < 10000) { std::printf("%ld cut row tiles\n", cut_tiles); return 1; }
    std::printf("ok\n");
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("join")
    src, exe = d / "join.cpp", d / "join"
    src.write_text(PROGRAM)
    subprocess.run([gxx, "-std=c++17", "-O2", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    return exe


@pytest.mark.parametrize("seed", range(3))
def test_every_cut_row_tile_is_joined(program, seed):
    out = subprocess.run([str(program), str(seed)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr
