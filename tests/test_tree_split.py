"""The cut of the attention of drafted tokens (csrc/tree_split.h), on the host: every key
tile of every unit is taken exactly once, the parts of a cut unit are on neighbouring CTAs,
and the bits of the keys that a query sees are those of the definition."""
import shutil
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2608_11742_gb300" / "csrc"

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <tuple>
#include <vector>
#include "tree_split.h"
using namespace rps::tree;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (trial %d)\n", __LINE__, #x, trial); return 1; } } while (0)

int main(int argc, char **argv) {
    std::mt19937 g(std::atoi(argv[1]));
    const auto rnd = [&](int lo, int hi) { return lo + static_cast<int>(g() % static_cast<unsigned>(hi - lo + 1)); };
    for (int trial = 0; trial < 60; ++trial) {
        const int groups[] = {1, 2, 3, 7, 8, 33, 64, 65, 128}, pages[] = {16, 32, 64, 128, 256};
        const int n_seq = rnd(1, 12), n_q = rnd(0, 2) ? rnd(1, 40) : rnd(1, 300), heads = rnd(1, 4), page = pages[rnd(0, 4)];
        const int width = rnd(1, 2000 / page + 2);
        const Shape s = make_shape(n_seq, n_q, heads, groups[rnd(0, 8)], page, 1000, width, rnd(0, 1));
        CHECK(s.tokens >= 1 && s.tokens * s.group <= kRows && s.tokens <= n_q);
        std::vector<Seq> seq(n_seq);
        for (auto &x : seq) {
            x = used_seq(s, rnd(0, 4) ? rnd(-1, width * page + 5) : rnd(-1, 2), rnd(0, 2) ? rnd(-1, n_q + 2) : n_q);
            CHECK(x.len >= -1 && x.len <= width * page && x.count >= 0 && x.count <= n_q && (x.len >= 0 || x.count == 0));
        }
        int64_t work = 0, longest = 0;
        std::map<std::tuple<int, int, int>, int64_t> begin;
        for (int i = 0; i < n_seq; ++i) {
            const int pairs = pairs_of(s, seq[i]);
            CHECK(pairs <= s.pairs && (pairs > 0) == (seq[i].count > 0));
            int most = 0, rows = 0;
            const int64_t places = places_of(s, seq[i], &most);
            int64_t sum = 0;
            for (int h = 0; h < heads; ++h)
                for (int p = 0; p < pairs; ++p) {
                    begin[{i, h, p}] = work + sum;
                    const int t = tiles_of(s, seq[i], p);
                    // every key that a row of the unit may see lies in its tiles
                    const int last = std::min((2 * p + 2) * s.tokens, seq[i].count);
                    const int keys = s.chain ? std::max(0, seq[i].len - seq[i].count + last) : seq[i].len;
                    CHECK(t >= 1 && t * kRows >= keys && (t == 1 || (t - 1) * kRows < keys));
                    sum += cost_of(s, seq[i], p);
                    CHECK(cost_of(s, seq[i], p) == (row_tiles_of(s, seq[i], p) == 2 ? t * kPairCost + kPairUnitCost : t * kTileCost + kUnitCost));
                    if (h == 0) rows += std::min(row_tiles_of(s, seq[i], p) * s.tokens, seq[i].count - 2 * p * s.tokens);
                }
            CHECK(sum == places && rows == seq[i].count);
            work += places;
            longest = std::max<int64_t>(longest, most);
        }
        if (!work) continue;
        const int n = static_cast<int>(std::min<int64_t>(rnd(1, 160), std::max<int64_t>(1, work / kPairCost)));
        const Ranges r = make_ranges(work, n);
        std::map<std::tuple<int, int, int>, int> at;        // tiles taken of each unit
        std::map<std::tuple<int, int, int>, int> first, parts;
        for (int c = 0; c < n; ++c) {
            const int64_t lo = range_start(r, c), hi = range_start(r, c + 1);
            CHECK(hi > lo && cta_of(r, lo) == c && cta_of(r, hi - 1) == c);
            // the sequence in which the range begins
            int64_t before = 0;
            int i = 0, most = 0;
            for (;; ++i) {
                const int64_t p = places_of(s, seq[i], &most);
                if (lo < before + p) break;
                before += p;
            }
            Walk w = begin_walk(s, i, seq[i], lo - before, hi - lo);
            CHECK((begin[{w.s, w.h, w.p}] + w.j) == lo);
            Piece x;
            int pieces = 0, cut_first = 0, cut_later = 0;
            while (next_piece(s, w, x, [&](int y) { return seq[y]; })) {
                const std::tuple<int, int, int> u{x.s, x.h, x.p};
                CHECK(x.tiles == tiles_of(s, seq[x.s], x.p) && x.rt == row_tiles_of(s, seq[x.s], x.p));
                CHECK(x.j0 == at[u] && x.j1 > x.j0 && x.j1 <= x.tiles);
                at[u] = x.j1;
                CHECK((x.part == -1) == (x.j0 == 0 && x.j1 == x.tiles) && (x.part == 1) == (x.j0 == 0 && x.j1 < x.tiles));
                cut_first += x.part == 1;
                cut_later += x.part == 0;
                CHECK(x.part != 0 || pieces == 0);  // one that continues a unit comes first
                CHECK(cut_first == (x.part == 1));  // one that begins a cut unit comes last
                if (x.part == 1) {
                    first[u] = c;
                    CHECK(x.to_last >= 0);
                    parts[u] = cta_of(r, hi + x.to_last) - c + 1;
                    CHECK(parts[u] >= 2 && c + parts[u] <= n);
                } else if (x.part == 0) {
                    CHECK(c - first[u] < parts[u] && (x.j1 < x.tiles || c == first[u] + parts[u] - 1));
                }
                ++pieces;
            }
            CHECK(cut_first <= 1 && cut_later <= 1);
        }
        for (const auto &[u, b] : begin) CHECK(at[u] == tiles_of(s, seq[std::get<0>(u)], std::get<2>(u)));
        // the bits
        for (int y = 0; y < 20; ++y) {
            const Seq q = seq[rnd(0, n_seq - 1)];
            if (!q.count) continue;
            const int i = rnd(0, q.count - 1), key = rnd(0, q.len / 32 + 2) * 32;
            std::vector<uint32_t> mask((n_q + 31) / 32);
            for (auto &m : mask) m = rnd(0, 3) ? g() : ~0u;
            const uint32_t a = chain_bits(q, i, key), b = mask_bits(q, key, [&](int w) {
                if (w < 0 || w >= static_cast<int>(mask.size())) std::abort();
                return mask[w];
            });
            for (int k = 0; k < 32; ++k) {
                const int j = key + k, t = j - (q.len - q.count);
                const bool in = j < q.len;
                CHECK((a >> k & 1u) == (in && t <= i));
                CHECK((b >> k & 1u) == (in && (t < 0 || (mask[t / 32] >> (t % 32) & 1u))));
            }
        }
    }
    std::puts("ok");
}
"""

LAYOUT = r"""
#include <cstdio>
#include "tree_split.h"
using namespace rps::tree;
int main() {
    for (uintptr_t base = 1 << 20; base < (1 << 20) + 512; base += kBaseAlign) {
        const Workspace w = workspace_at(base, 32, 128), zero = workspace_at(0, 32, 128);
        const size_t slots = 2 * kMaxCtas * 2 * kRows;
        const bool good = (base + w.o) % kPartAlign == 0 && (base + w.ml) % 8 == 0 && (base + w.cut) % 16 == 0 &&
                          w.cut + 32 * kMaxCtas <= w.ml && w.ml + 8 * slots <= w.o && w.o + 4 * slots * 128 <= w.bytes &&
                          w.bytes == zero.bytes;
        if (!good) return 1;
    }
    std::puts("ok");
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_the_parts_of_a_workspace_lie_on_their_bounds(tmp_path):
    """Partial results are moved 32 bytes at a time, wherever a workspace begins (16-byte bounds), and lie inside it."""
    src, exe = tmp_path / "layout.cc", tmp_path / "layout"
    src.write_text(LAYOUT)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True).stdout.strip() == "ok"


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_tile_is_taken_once(tmp_path):
    src, exe = tmp_path / "split.cc", tmp_path / "split"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover", f"-I{CSRC}", str(src),
                    "-o", str(exe)], check=True)
    for seed in range(25):
        r = subprocess.run([str(exe), str(seed)], capture_output=True, text=True)
        assert r.returncode == 0 and r.stdout.strip() == "ok", (seed, r.stdout, r.stderr)
