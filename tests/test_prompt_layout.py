"""The division of packed prompts' attention (csrc/prompt_layout.h, plain C++), compiled for the host: tiles, what they see, splits, places in LDS."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_07503_amd", "csrc")
_MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "prompt_layout.h"
#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); exit(1); } } while (0)

int main() {
    srand(1);
    // tiles: an upper bound over any cut of the rows; the keys that a tile's rows see
    for (int it = 0; it < 20000; ++it) {
        const int seqs = 1 + rand() % 9, G = 1 + rand() % 8, tile = 32 << rand() % 4;
        long rows = rand() % 3 ? 0 : rand() % 200, tiles = 0, place = 0;
        for (int b = 0; b < seqs; ++b) {
            const int n = rand() % 3 ? rand() % 300 : 0, keys = rand() % 400;
            const int t = prompt_tiles(n, G, tile), at = prompt_first_tile((int)rows, b, G, tile);
            CHECK(at >= place);
            place = at + (t ? t : 1);
            rows += n;
            CHECK((long)t * tile >= (long)n * G && (n == 0 ? t == 0 : (long)(t - 1) * tile < (long)n * G));
            tiles += t;
            for (int i = 0; i < t; ++i) {
                int seen = 0;
                for (int r = i * tile; r < (i + 1) * tile && r < n * G; ++r)
                    for (int key = seen; key < keys; ++key)
                        if (key <= r / G + prompt_offset(n, keys)) seen = key + 1;
                CHECK(prompt_keys(i, n, keys, G, tile) == seen);
            }
        }
        CHECK(tiles <= prompt_max_tiles(rows, seqs, G, tile) && place <= rows * G / tile + seqs);
    }
    CHECK(prompt_max_tiles(0, 5, 3, 128) == 0 && prompt_max_tiles(1280, 65, 3, 128) == 95);
    // splits go through every block once, whatever was expected of the number of keys
    for (int it = 0; it < 200000; ++it) {
        const int keys = rand() % 3000, block = 32 << rand() % 3, n_splits = 1 + rand() % 9, per = 1 + rand() % 20, blocks = (keys + block - 1) / block;
        int at = 0, some = 0;
        for (int s = 0; s < n_splits; ++s) {
            const PromptBlocks r = prompt_blocks(keys, block, s, n_splits, per);
            if (!r.any) continue;
            CHECK(some == s && r.first == at && r.last >= r.first);
            at = r.last;
            ++some;
        }
        CHECK(at == blocks && some >= 1);
        for (int s = 0; s < n_splits; ++s) CHECK(prompt_blocks(keys, block, s, n_splits, per).several == (some > 1));
    }
    // pieces of a row in LDS: each has a place in its row, and 8 tokens' pieces, and 64 bytes of 4 tokens, lie in different banks
    for (int row : {64, 128, 192, 256, 384, 512, 768, 1024}) {
        const int n = row / 16;
        for (int t = 0; t < 64; ++t) {
            std::vector<char> seen(n, 0);
            for (int c = 0; c < n; ++c) {
                const int p = prompt_swizzle(t, c, row);
                CHECK(p >= 0 && p < n && !seen[p]);
                seen[p] = 1;
            }
        }
        const int again = row % 128 == 64 ? 4 : row % 256 == 128 ? 8 : 16;      // pieces after which places repeat
        for (int t = 0; t < 64; ++t)
            for (int c = 0; c + again < n; ++c) CHECK(prompt_swizzle(t, c + again, row) == prompt_swizzle(t, c, row) + again && prompt_swizzle(t + 16, c, row) == prompt_swizzle(t, c, row));
        auto bank = [&](int t, int c) { return (t * row / 16 + prompt_swizzle(t, c, row)) % 16; };      // of 16 bytes
        for (int c = 0; c < n; ++c)
            for (int t0 = 0; t0 < 64; t0 += 8) {
                int used = 0;
                for (int t = t0; t < t0 + 8; ++t) used |= 1 << bank(t, c);
                CHECK(__builtin_popcount(used) == 8);
            }
        for (int c = 0; c < n; c += 4)
            for (int t0 = 0; t0 < 64; t0 += 4) {
                int used = 0;
                for (int t = t0; t < t0 + 4; ++t)
                    for (int i = 0; i < 4; ++i) used |= 1 << bank(t, c + i);
                CHECK(used == 0xFFFF);
            }
    }
    puts("ok");
}
"""


def test_tiles_splits_and_places(tmp_path):
    (tmp_path / "main.cpp").write_text(_MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-I", CSRC, str(tmp_path / "main.cpp"), "-o",
                    str(tmp_path / "main")], check=True)
    r = subprocess.run([str(tmp_path / "main")], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


_PLACES = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "prompt_layout.h"
#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); exit(1); } } while (0)

int main() {
    srand(2);
    for (int it = 0; it < 3000; ++it) {
        const int seqs = 1 + rand() % (it % 2 ? 9 : 400), G = 1 + rand() % 8, tile = 32 << rand() % 4, live = 1 + rand() % 100;
        std::vector<int> start(seqs + 1), owner, of;
        start[0] = rand() % 3 ? 0 : rand() % 300;
        for (int b = 0; b < seqs; ++b) start[b + 1] = start[b] + (rand() % 100 < live ? rand() % (rand() % 4 ? 3 : 300) : 0);
        const int rows = start[seqs] + (rand() % 2 ? rand() % 50 : 0);
        const long places = prompt_max_tiles(rows, seqs, G, tile);
        CHECK(places <= (long)rows * G / tile + seqs && places <= (long)rows * G / tile + rows);
        // every tile has a place below the bound, and no two have the same
        std::vector<int> b_of(places, -1), t_of(places, -1);
        for (int b = 0, before = 0; b < seqs; ++b) {
            const int at = prompt_place(start[b], b, G, tile);
            CHECK(at >= before);
            before = at;
            for (int t = 0; t < prompt_tiles(start[b + 1] - start[b], G, tile); ++t) {
                CHECK(at + t < places && b_of[at + t] < 0);
                b_of[at + t] = b;
                t_of[at + t] = t;
            }
        }
        // and is found as the last sequence that begins at or before it
        for (long i = 0; i < places; ++i) {
            int b = -1;
            for (int c = 0; c < seqs; ++c)
                if (prompt_place(start[c], c, G, tile) <= i) b = c;
            const int t = b < 0 ? -1 : (int)i - prompt_place(start[b], b, G, tile);
            const bool there = b >= 0 && t < prompt_tiles(start[b + 1] - start[b], G, tile);
            CHECK(there == (b_of[i] >= 0) && (!there || (b == b_of[i] && t == t_of[i])));
        }
    }
    CHECK(prompt_max_tiles(8, 100000, 4, 128) == 8 && prompt_max_tiles(0, 100000, 4, 128) == 0);
    puts("ok");
}
"""


def test_places_of_sequences_with_rows(tmp_path):
    """Sequences without rows take no places: the bound is that of the rows, and the search still finds every tile."""
    (tmp_path / "main.cpp").write_text(_PLACES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-I", CSRC, str(tmp_path / "main.cpp"), "-o",
                    str(tmp_path / "main")], check=True)
    r = subprocess.run([str(tmp_path / "main")], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
