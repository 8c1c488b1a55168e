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
