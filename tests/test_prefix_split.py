"""The cut of the attention over the paged cache (csrc/prefix_split.h), on the host:
every key that a row sees is taken exactly once, by the columns its row is given and
by the product's steps; steps that overwrite come first; every address stays inside."""
import shutil
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2608_11742_gb300" / "csrc"

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <algorithm>
#include <array>
#include <map>
#include <random>
#include <vector>
#include "prefix_split.h"
using namespace rps::prefix;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (trial %d)\n", __LINE__, #x, trial); return 1; } } while (0)

int main(int argc, char **argv) {
    const int trial = -1;
    for (int d = 1; d < 5000; d += 1 + d / 9) {
        const Div v = make_div(d);
        for (int64_t n = 0; n < (int64_t{1} << 31); n += 1 + n / 40 + d / 3)
            for (int64_t m = n - 1; m <= n + 1; ++m)
                if (m >= 0 && m < (int64_t{1} << 31)) CHECK(quotient(static_cast<int>(m), v) == m / d);
        for (int64_t n = d; n < (int64_t{1} << 31); n += d * (1 + n / d / 9)) CHECK(quotient(static_cast<int>(n - 1), v) == (n - 1) / d && quotient(static_cast<int>(n), v) == n / d);
    }
    std::mt19937 g(std::atoi(argv[1]));
    const auto rnd = [&](int lo, int hi) { return lo + static_cast<int>(g() % static_cast<unsigned>(hi - lo + 1)); };
    for (int trial = 0; trial < 12; ++trial) {
        const int pages[] = {16, 32, 64, 128, 256};
        const int groups[] = {1, 2, 3, 7, 8, 33, 128};
        const int n_req = rnd(1, 4), nb = rnd(0, 3) ? rnd(1, 9) : rnd(1, 150), n_q = rnd(0, 2) ? rnd(1, 5) : rnd(1, 150);
        const int page = pages[rnd(0, 4)], group = groups[rnd(0, 6)], heads = rnd(1, 3);
        const int most = rnd(1, 3) * 256 / (nb > 20 || n_q > 20 ? 4 : 1), width = ceil_div(most, page);
        const Shape s = make_shape(n_req, nb, n_q, heads, group, page, 1000, width, rnd(0, 1));
        CHECK(s.tokens * s.group <= kRows && s.tokens >= 1);
        std::vector<int> len(n_req * nb), shared_len(n_req);
        for (auto &x : len) x = rnd(0, 5) ? rnd(-1, width * page + 3) : rnd(-1, 1);
        for (auto &x : shared_len) x = rnd(-2, width * page);
        if (rnd(0, 2) == 0) for (auto &x : len) x = x % 40;
        for (auto &x : len) x = used_len(s, x);
        // the whole work, as the CTAs walk it
        struct Tile { int q, rt; int64_t start; Tiles t; int tiles; };
        std::vector<Tile> all;
        int64_t work = 0;
        for (int q = 0; q < n_req; ++q)
            for (int h = 0; h < heads; ++h)
                for (int rt = 0; rt < s.row_tiles; ++rt) {
                    const RowTile r = row_tile(s, rt);
                    KeySum k{0, 0, 1 << 30};
                    for (int i = 0; i < r.nb; ++i) add_sequence(s, k, len[q * nb + r.b0 + i]);
                    const Tiles t = key_tiles(s, k, shared_slots(s, k, shared_len[q]));
                    all.push_back({q, rt, work, t, t.shared + t.own});
                    work += cost_of(t);
                }
        const int n = static_cast<int>(std::min<int64_t>(rnd(1, 160), std::max<int64_t>(1, work / kWidest)));
        if (!work) continue;
        const Ranges ranges = make_ranges(work, n);
        CHECK(ranges.base == work / n && ranges.extra == work % n);
        CHECK(make_ranges(work * 1000003 * 4099, n).base == work * 1000003 * 4099 / n);
        const auto range_start = [&](int c, int64_t, int) { return rps::prefix::range_start(ranges, c); };
        int64_t sum = 0;
        for (int c = 0; c < n; ++c) sum += range_start(c + 1, work, n) - range_start(c, work, n);
        CHECK(sum == work);
        for (int c = 0; c < n && work; ++c) CHECK(range_start(c + 1, work, n) > range_start(c, work, n));
        std::vector<int> covered(n_req * s.row_tiles, 0), taken(n, 0);
        int64_t before = -1;  // place of the tile before
        for (const Tile &x : all) {
            CHECK(cost_of(x.t) == (x.tiles ? kRowCost + kSharedCost * x.t.shared + kOwnCost * x.t.own : 0));
            if (!x.tiles) continue;
            for (int k = 0; k < x.tiles; ++k) {
                const int64_t at = x.start + place(x.t, k);
                CHECK(at > before && at - before <= kWidest && place(x.t, k) < cost_of(x.t));
                CHECK(reach(x.t, place(x.t, k)) == k + 1 && reach(x.t, place(x.t, k) - 1) == k);
                before = at;
            }
            CHECK(reach(x.t, -1000) == 0 && reach(x.t, 0) == 0 && reach(x.t, cost_of(x.t)) == x.tiles);
            CHECK(reach(x.t, int64_t{1} << 60) == x.tiles);
            // pieces of this row tile: cut at the CTAs' range ends
            std::vector<std::pair<int, int>> pieces;
            int first = -1, last = -1;
            for (int c = 0; c < n; ++c) {
                const int lo = reach(x.t, range_start(c, work, n) - x.start), hi = reach(x.t, range_start(c + 1, work, n) - x.start);
                CHECK(lo <= hi);
                if (lo >= hi) continue;
                CHECK(pieces.empty() ? lo == 0 : lo == pieces.back().second);
                CHECK(first < 0 || c == last + 1);  // the parts of a cut row tile are neighbours
                if (first < 0) first = c;
                last = c;
                taken[c] += hi - lo;
                pieces.push_back({lo, hi});
            }
            CHECK(pieces.back().second == x.tiles);
            CHECK(cta_of(ranges, x.start + place(x.t, x.tiles - 1) - 1) == last && cta_of(ranges, x.start + place(x.t, 0) - 1) == first);
            if (covered[x.q * s.row_tiles + x.rt]++) continue;  // (another head: the same but for its pieces' ends)
            const RowTile r = row_tile(s, x.rt);
            CHECK(r.nb >= 1 && r.nb <= kRows && r.b0 + r.nb <= nb);
            KeySum k{0, 0, 1 << 30};
            std::vector<int> off(r.nb + 1, 0), ln(r.nb);
            for (int i = 0; i < r.nb; ++i) add_sequence(s, k, ln[i] = len[x.q * nb + r.b0 + i]);
            const int shared = shared_slots(s, k, shared_len[x.q]), st = ceil_div(shared, s.spt);
            for (int i = 0; i < r.nb; ++i) off[i + 1] = off[i] + (ln[i] < 0 ? 0 : ceil_div(ln[i], s.slot) - shared);
            for (int i = 0; i < r.nb; ++i) CHECK(off[i + 1] >= off[i]);
            CHECK(x.tiles == imax(1, st + ceil_div(off[r.nb], s.spt)));
            // what each row takes: columns and steps
            std::vector<std::map<int, int>> by_columns(kRows), by_steps(kRows);
            for (const auto &p : pieces) {
                std::vector<std::array<int, 2>> touched(kRows, {0, 0});
                for (int j = p.first; j < p.second; ++j) {
                    const int half = (j - p.first) & 1;
                    for (int u = 0; u < s.spt && j >= st; ++u) {
                        const int idx = (j - st) * s.spt + u;
                        if (idx >= off[r.nb]) continue;
                        const int i = slot_owner(off.data(), r.nb, idx);
                        CHECK(off[i] <= idx && idx < off[i + 1]);
                        CHECK((idx - off[i] + shared) / s.sub < width);
                    }
                    for (int row = 0; row < r.n_tok * s.group; ++row) {
                        const int tok = r.tok0 + row / s.group, i = tok / s.n_q - r.b0, qi = tok % s.n_q;
                        if (ln[i] < 0) continue;
                        const int limit = row_limit(s, ln[i], qi);
                        const Columns c = row_columns(s, j, st, shared, off[i], limit);
                        const int base = j < st ? j * kRows : shared * s.slot + ((j - st) * s.spt - off[i]) * s.slot;
                        for (int col = c.lo; col < c.hi; ++col) by_columns[row][base + col]++;
                        if (j < st) {
                            for (int kk = 0; kk < 8; ++kk)
                                for (int e = 0; e < 16; ++e) {
                                    const int key = j * kRows + kk * 16 + e;
                                    if (key < limit && key < shared * s.slot) by_steps[row][key]++;
                                }
                            touched[row][half] = 1;
                        }
                    }
                    if (j < st) continue;
                    for (int kk = 0; kk < 8; ++kk) {
                        const Step w = own_step(s, r, off.data(), ln.data(), st, shared, p.first, j, kk);
                        if (!w.keys) continue;
                        CHECK(w.r0 >= 0 && w.r0 < w.r1 && w.r1 <= r.n_tok * s.group);
                        const int key0 = ((j - st) * s.spt + kk * 16 / s.slot - off[w.who] + shared) * s.slot + kk * 16 % s.slot;
                        for (int row = w.r0; row < w.r1; ++row) {
                            const int tok = r.tok0 + row / s.group;
                            CHECK(tok / s.n_q - r.b0 == w.who);
                            CHECK(w.fresh == !touched[row][half]);
                            touched[row][half] = 1;
                            for (int e = 0; e < w.keys; ++e)
                                if (key0 + e < row_limit(s, ln[w.who], tok % s.n_q)) by_steps[row][key0 + e]++;
                        }
                    }
                }
            }
            for (int row = 0; row < r.n_tok * s.group; ++row) {
                const int tok = r.tok0 + row / s.group, i = tok / s.n_q - r.b0;
                const int limit = ln[i] < 0 ? 0 : row_limit(s, ln[i], tok % s.n_q);
                for (const auto *m : {&by_columns[row], &by_steps[row]}) {
                    CHECK(static_cast<int>(m->size()) == limit);
                    for (const auto &e : *m) CHECK(e.first >= 0 && e.first < limit && e.second == 1);
                }
            }
        }
        if (n > 1) for (int c = 0; c < n; ++c) CHECK(taken[c] > 0);  // each CTA has a tile
    }
    std::printf("ok\n");
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("prefix")
    src, exe = d / "split.cpp", d / "split"
    src.write_text(PROGRAM)
    subprocess.run([gxx, "-std=c++17", "-O2", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    return exe


@pytest.mark.parametrize("seed", range(4))
def test_every_visible_key_is_taken_once(program, seed):
    out = subprocess.run([str(program), str(seed)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr
