"""The index arithmetic of the paged cache and of tree attention (csrc/cache_layout.h, plain C++), compiled for the host: where elements
lie, what entries of a page table and lengths outside their range lead to, what a row sees, how work is divided."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_07503_amd", "csrc")
_MAIN = r"""
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "cache_layout.h"
#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); exit(1); } } while (0)

template <int KIND> void layout(int hd, int pt) {
    const size_t n = (size_t)pt * hd;
    CHECK(cache_block_bytes(KIND, pt, hd) == 2 * n * cache_elem_bytes(KIND) + (KIND == 2 ? 2 * pt : 0));
    CHECK(cache_block_bytes(KIND, pt, hd) % 16 == 0);
    for (int v = 0; v < 2; ++v) {
        std::vector<char> seen(n, 0);
        for (int t = 0; t < pt; ++t)
            for (int j = 0; j < hd; ++j) {
                const size_t i = cache_index<KIND>(v, t, j, hd);
                CHECK(i < n && !seen[i]);
                seen[i] = 1;
            }
        // what is loaded or stored in one piece is contiguous and aligned to its size
        for (int t = 0; t < pt; ++t)
            for (int j = 0; j < hd; j += 8)
                for (int e = 0; e < 8 && !v; ++e) {
                    const int piece = KIND == 0 ? 4 : 8;
                    CHECK(cache_k_index<KIND>(t, j + e, hd) == cache_k_index<KIND>(t, j + e / piece * piece, hd) + e % piece);
                    CHECK(cache_k_index<KIND>(t, j + e / piece * piece, hd) % piece == 0);
                }
        for (int t = 0; t < pt; t += 4)
            for (int j = 0; j < hd && v; ++j) {
                CHECK(cache_v_index<KIND>(t, j, hd) % 4 == 0);
                for (int e = 0; e < 4; ++e) CHECK(cache_v_index<KIND>(t + e, j, hd) == cache_v_index<KIND>(t, j, hd) + e);
            }
    }
}

int main() {
    for (int hd : {32, 64, 96, 128, 192, 256})
        for (int pt : {32, 96}) { layout<0>(hd, pt); layout<1>(hd, pt); layout<2>(hd, pt); }

    // page table entries and positions out of range are no page
    const int32_t table[6] = {0, -1, 6, 7, INT_MAX, INT_MIN};
    for (long pos : {0L, 31L, 32L, 64L, 96L, 128L, 160L, 191L, 192L, 1000000L, (long)INT_MAX, -1L, (long)INT_MIN}) {
        const int page = cache_page(table, 6, 32, 7, (int)pos);
        CHECK(page == (pos >= 0 && pos < 32 ? 0 : pos >= 64 && pos < 96 ? 6 : -1));
    }
    // rows: whatever row_start holds, they lie in [0, n_rows)
    const int odd[] = {INT_MIN, -1, 0, 1, 5, 9, 10, 11, INT_MAX};
    for (int a : odd)
        for (int b : odd)
            for (int n_rows : {0, 1, 10}) {
                const int32_t rs[2] = {a, b};
                const int r0 = rows_first(rs, 0, n_rows), n = rows_count(rs, 0, n_rows);
                CHECK(r0 >= 0 && n >= 0 && r0 + n <= n_rows);
                if (a >= 0 && b >= a && b <= n_rows) CHECK(r0 == a && n == b - a);
            }
    // tiles, and their bound
    for (int first : {0, 1, 31, 32, 63, 1 << 30})
        for (int n = 0; n < 200; ++n) {
            int touched = 0, last = -1;
            for (int i = 0; i < n; ++i) if ((first + i) / 32 != last) { last = (first + i) / 32; ++touched; }
            CHECK(cache_tiles(first, n) == touched);
        }
    CHECK(cache_tiles(-1, 5) == 0 && cache_tiles(INT_MIN, 5) == 0 && cache_tiles(INT_MAX, 5) == 0 && cache_tiles((1 << 30) + 1, 1) == 0);
    srand(1);
    for (int it = 0; it < 20000; ++it) {
        const int seqs = 1 + rand() % 9;
        int rows = 0;
        long tiles = 0;
        for (int b = 0; b < seqs; ++b) {
            const int n = rand() % 4 ? rand() % (1 + rand() % 130) : 0;
            rows += n;
            tiles += cache_tiles(rand() % 100, n);
        }
        CHECK(tiles <= cache_max_tiles(rows, seqs));
    }
    // visibility, against the definition
    for (int it = 0; it < 200000; ++it) {
        const int ctx = rand() % 80, n = rand() % 70, n_tot = ctx + n - (rand() % 8 == 0 ? rand() % (n + 1) : 0), words = 1 + rand() % 3;
        const int node = n ? rand() % n : 0, t0 = 32 * (rand() % 6);
        uint32_t m[4];
        for (int w = 0; w < 4; ++w) m[w] = (uint32_t)rand() * 2654435761u;
        const bool window = rand() % 3 == 0;
        uint32_t want = 0;
        for (int k = 0; k < 32; ++k) {
            const int t = t0 + k, j = t - ctx;
            const bool sees = t < n_tot && (t < ctx || (window ? j <= node : j < 32 * words && (m[j / 32] >> (j % 32) & 1)));
            if (sees) want |= 1u << k;
        }
        CHECK(tree_visible(window ? nullptr : m, words, ctx, n_tot, node, t0) == want);
    }
    // the splits of a context go through every block once, and none behind the last visible token
    for (int it = 0; it < 20000; ++it) {
        const int ctx = rand() % 3000, n = 1 + rand() % 70, n_tot = ctx + n, last_node = rand() % n, splits = 1 + rand() % 20;
        const bool mask = rand() % 2;
        const int blocks = ((mask ? n_tot : ctx + last_node + 1) + 31) / 32;
        int at = 0;
        for (int s = 0; s < splits; ++s) {
            const TreeBlocks r = tree_blocks(mask, ctx, n_tot, last_node, s, splits);
            CHECK(r.first == at && r.last >= r.first);
            at = r.last;
        }
        CHECK(at == blocks);
    }
    puts("ok");
}
"""


def test_layout_pages_visibility_and_splits(tmp_path):
    (tmp_path / "main.cpp").write_text(_MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined,address", "-fno-sanitize-recover=all", "-I", CSRC, str(tmp_path / "main.cpp"), "-o",
                    str(tmp_path / "main")], check=True)
    r = subprocess.run([str(tmp_path / "main")], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
