// The paged cache of the tree operators: where an element of it lies, which page holds a position, what a row of a tree sees, how the
// work on it is divided.  Plain C++ (constexpr: host and device), so that a test can play it through without a GPU.
//
// A page holds one block per key/value head: keys, values and (fp8) a scale byte per token for either.  Keys and values are stored in
// blocks of 32 tokens in the order in which the 64 lanes of a wavefront feed the matrix instructions of the attention
// (kernels_tree.hip.h): a lane's share is 16 contiguous bytes and a wavefront's load 1 KiB, so that attention streams a page through
// registers without a transposition.  The price is paid once per token, by the write.
//   keys    rows of the operand = tokens, lane 32 g + t % 32:
//     fp32  16 bytes = dimensions 8 c + 4 g + (0 .. 3)                        [t / 32][c]
//     bf16  16 bytes = dimensions 16 c + 8 g + (0 .. 7)                       [t / 32][c]
//     fp8   16 bytes = the two bf16 pieces of c = 2 d and 2 d + 1             [t / 32][d]
//   values  rows of the operand = dimensions, lane 32 g + j % 32; a score tile leaves the matrix core with tokens
//           8 m + 4 g + (0 .. 3), m < 4, in a lane, so that is what a lane's share of the other operand holds:
//     fp32  16 bytes = those of one m                                         [t / 32][j / 32][m]
//     bf16  16 bytes = those of m = 2 i and 2 i + 1                           [t / 32][i][j / 32]
//     fp8   16 bytes = those of m = 0 .. 3                                    [t / 32][j / 32]
// Kinds are the values of sjd_dtype: 0 fp32, 1 bf16, 2 fp8.
#pragma once
#include <stddef.h>
#include <stdint.h>

constexpr int kCacheMinExp = -100, kCacheMaxExp = 119;   // of the scales; a scale byte is the exponent + 127

constexpr size_t cache_elem_bytes(int kind) { return kind == 0 ? 4 : kind == 1 ? 2 : 1; }
constexpr size_t cache_block_bytes(int kind, int page_tokens, int hd) {
    return 2 * (size_t)page_tokens * hd * cache_elem_bytes(kind) + (kind == 2 ? 2 * (size_t)page_tokens : 0);
}

// element of token t, dimension j within the keys (or values) of a block
template <int KIND> constexpr size_t cache_k_index(int t, int j, int hd) {
    const size_t base = (size_t)(t >> 5) * 32 * hd;
    if (KIND == 0) return base + (j >> 3) * 256 + (((j >> 2) & 1) * 32 + (t & 31)) * 4 + (j & 3);
    if (KIND == 1) return base + (j >> 4) * 512 + (((j >> 3) & 1) * 32 + (t & 31)) * 8 + (j & 7);
    return base + (j >> 5) * 1024 + (((j >> 3) & 1) * 32 + (t & 31)) * 16 + ((j >> 4) & 1) * 8 + (j & 7);
}
template <int KIND> constexpr size_t cache_v_index(int t, int j, int hd) {
    const size_t base = (size_t)(t >> 5) * 32 * hd;
    const int g = (t >> 2) & 1, m = (t >> 3) & 3, e = t & 3, lane = g * 32 + (j & 31);
    if (KIND == 0) return base + ((j >> 5) * 4 + m) * 256 + lane * 4 + e;
    if (KIND == 1) return base + ((m >> 1) * (hd >> 5) + (j >> 5)) * 512 + lane * 8 + (m & 1) * 4 + e;
    return base + (j >> 5) * 1024 + lane * 16 + m * 4 + e;
}
template <int KIND> constexpr size_t cache_index(bool v, int t, int j, int hd) { return v ? cache_v_index<KIND>(t, j, hd) : cache_k_index<KIND>(t, j, hd); }

// page that holds position pos of the sequence whose row of the page table is `table`, -1 if there is none
constexpr int cache_page(const int32_t *table, int pages_per_seq, int page_tokens, int n_pages, int pos) {
    if (pos < 0 || pos / page_tokens >= pages_per_seq) return -1;
    const int page = table[pos / page_tokens];
    return page >= 0 && page < n_pages ? page : -1;
}

// rows of sequence b, cut to [0, n_rows): first one and number
constexpr int rows_cut(int r, int n_rows) { return r < 0 ? 0 : r > n_rows ? n_rows : r; }
constexpr int rows_first(const int32_t *row_start, int b, int n_rows) { return rows_cut(row_start[b], n_rows); }
constexpr int rows_count(const int32_t *row_start, int b, int n_rows) {
    const int n = rows_cut(row_start[b + 1], n_rows) - rows_cut(row_start[b], n_rows);
    return n > 0 ? n : 0;
}

// First position of a sequence's rows as a write or a read takes it.  One that is negative or beyond 2^30 is outside, and with it the whole
// sequence: its rows stand where no table reaches (a sequence has at most 2^30 positions), so that writes drop them and reads give zeros.
constexpr int kCacheOutside = 1 << 30;
constexpr int cache_first(int first) { return first < 0 || first > kCacheOutside ? kCacheOutside : first; }

// tiles of 32 positions that n rows from position `first` on touch
constexpr int cache_tiles(int first, int n) { return n > 0 && first >= 0 && first <= kCacheOutside ? ((first + n - 1) >> 5) - (first >> 5) + 1 : 0; }
// and an upper bound over n_rows rows of n_seqs sequences: n >= 1 rows touch at most 1 + (n + 30) / 32 of them, and no more than n
constexpr long cache_max_tiles(int n_rows, int n_seqs) {
    const long s = n_seqs < n_rows ? n_seqs : n_rows, t = (n_rows + 30 * s) / 32 + s;
    return t < n_rows ? t : n_rows;
}

// Bit k: node `node` of a tree, whose row of the mask is `mask` (NULL: a window), sees the token at position t0 + k.  ctx positions are
// cached, n_tot there at all.
constexpr uint32_t tree_visible(const uint32_t *mask, int mask_words, int ctx, int n_tot, int node, int t0) {
    const int off = t0 - ctx;          // node that stands at t0
    uint32_t nodes = 0;                // bits off .. off + 31 of the mask
    if (off > -32) {
        if (mask) {
            const int w = off >> 5, sh = off & 31;                     // w >= -1
            const uint32_t lo = w >= 0 && w < mask_words ? mask[w] : 0u, hi = w + 1 < mask_words ? mask[w + 1] : 0u;
            nodes = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
        } else {
            const int k = node - off;  // last bit that is set
            nodes = k >= 31 ? 0xFFFFFFFFu : k >= 0 ? (2u << k) - 1u : 0u;
        }
    }
    const uint32_t cached = off >= 0 ? 0u : off <= -32 ? 0xFFFFFFFFu : (1u << -off) - 1u;
    const int left = n_tot - t0;
    const uint32_t there = left >= 32 ? 0xFFFFFFFFu : left > 0 ? (1u << left) - 1u : 0u;
    return ((nodes & ~cached) | cached) & there;
}

// The node that a walk through a tree of n nodes goes on to from node `at`, whose accepted child is said to be `choice`; -1: it ends there.  (Where row_start does not
// ascend, sequences share rows, and what one of them says of its nodes may have been written for the larger tree of another.)
constexpr int tree_step(int choice, int at, int n) { return choice > at && choice < n ? choice : -1; }

// Blocks of 32 tokens [first, last) that split `split` of n_splits goes through, of rows the last of which is node last_node
struct TreeBlocks { int first, last; };
constexpr TreeBlocks tree_blocks(bool mask, int ctx, int n_tot, int last_node, int split, int n_splits) {
    // a window's rows see no node behind the last one
    const int n_vis = mask || ctx + last_node + 1 > n_tot ? n_tot : ctx + last_node + 1;
    const int blocks = (n_vis + 31) >> 5, chunk = (blocks + n_splits - 1) / n_splits;
    TreeBlocks r{split * chunk, split * chunk + chunk};
    if (r.first > blocks) r.first = blocks;
    if (r.last > blocks) r.last = blocks;
    return r;
}
