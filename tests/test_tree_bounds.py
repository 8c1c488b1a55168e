"""Lengths and positions out of range in the index arithmetic of the tree operators (csrc/cache_layout.h, plain C++), played through on the host."""
import subprocess

from test_tree_layout import CSRC

_HEAD = r"""
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "cache_layout.h"
#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); exit(1); } } while (0)
int main() {
"""


def play(tmp_path, body):
    (tmp_path / "main.cpp").write_text(_HEAD + body + '    puts("ok");\n}\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-I", CSRC, str(tmp_path / "main.cpp"), "-o",
                    str(tmp_path / "main")], check=True)
    r = subprocess.run([str(tmp_path / "main")], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_first_positions_outside(tmp_path):
    """The tiles of such a sequence hold all of its rows, and no page: its row of the largest table is not even looked at (it is a null pointer here)."""
    play(tmp_path, r"""
    for (int first : {INT_MIN, -1000, -3, -1, 1 << 30, (1 << 30) + 1, (1 << 30) + 40, INT_MAX})
        for (int n : {0, 1, 31, 32, 33, 100, 1 << 29})
            for (int page_tokens : {32, 96, 1 << 20}) {
                const int f = cache_first(first), tiles = cache_tiles(f, n), per_seq = (1 << 30) / page_tokens;
                CHECK(tiles <= cache_max_tiles(n, 1));
                CHECK(n == 0 ? tiles == 0 : ((f >> 5) << 5) <= f && (((f >> 5) + tiles) << 5) >= f + n);
                for (int t = 0; t < tiles; t += 1 + tiles / 50) CHECK(cache_page(nullptr, per_seq, page_tokens, INT_MAX, ((f >> 5) + t) << 5) == -1);
            }
    for (int first : {0, 1, 31, 1000, (1 << 30) - 1}) CHECK(cache_first(first) == first);
""")


def test_walks_stay_within_their_trees(tmp_path):
    """Whatever stands at a tree's rows: here what a larger tree, whose rows they are as well, has left there.  Every node of a walk is read at its index."""
    play(tmp_path, r"""
    std::vector<int> choice(1000);
    for (int i = 0; i < 1000; ++i) choice[i] = i + 50;
    std::vector<int> mine(choice.begin(), choice.begin() + 100);     // rows 900 .. 999 of these, as the nodes 0 .. 99 of a tree of their own: 850 further on
    for (int &c : mine) c += 900;
    CHECK(mine[0] == 950 && tree_step(mine[0], 0, 100) == -1);
    srand(1);
    const int odd[] = {INT_MIN, -1, 0, 1, 5, 99, 100, 101, 1023, 1024, INT_MAX};
    for (int it = 0; it < 2000; ++it) {
        const int n = 1 + rand() % 100;
        std::vector<int> c(n);
        for (int &x : c) x = rand() % 4 ? rand() % (n + 3) : odd[rand() % 11];
        int at = 0, steps = 0;
        for (;;) {
            const int next = tree_step(c.at(at), at, n);
            CHECK(next == (c[at] > at && c[at] < n ? c[at] : -1));
            if (next < 0) break;
            at = next;
            CHECK(++steps < n);
        }
    }
""")
