// How attention of packed prompts is divided (kernels_prompt.hip.h).  Plain C++ (constexpr: host and device), so that a test can play
// it through without a GPU.
//
// The query rows (i, h) of one kv head of a sequence, ordered by i, then by the query head h of the group of G, are cut into tiles of `tile` rows.  The keys that a
// tile sees are cut into blocks, and those of long ones into splits.
#pragma once
#include "cache_layout.h"

// keys that come before a sequence's first query's own: query i sees keys 0 .. i + prompt_offset (negative: its first queries see nothing)
constexpr int prompt_offset(int n, int n_keys) { return n_keys - n; }

// tiles of n rows
constexpr int prompt_tiles(int n, int G, int tile) { return (int)(((long)n * G + tile - 1) / tile); }
// Where the tiles of sequence b begin whose rows begin at `first`, if every sequence has its place whatever those before it have: places ascend, and those behind a sequence's tiles are empty.
constexpr int prompt_first_tile(int first, int b, int G, int tile) { return (int)((long)first * G / tile) + b; }
// Where they begin if only sequences with rows have places (those without lie where the next one begins, or behind the last): of the sequences before b at most `first` have rows.
constexpr int prompt_place(int first, int b, int G, int tile) { return prompt_first_tile(first, b < first ? b : first, G, tile); }
// An upper bound of the tiles, and of these places, over n_rows rows of n_seqs sequences, however many of them have rows
constexpr long prompt_max_tiles(long n_rows, long n_seqs, int G, int tile) { return n_rows * G / tile + (n_seqs < n_rows ? n_seqs : n_rows); }
// keys that some row of tile t of a sequence sees: 0 .. prompt_keys - 1
constexpr int prompt_keys(int t, int n, int n_keys, int G, int tile) {
    const long last = ((long)(t + 1) * tile - 1) / G;
    const int i = last < n ? (int)last : n - 1;
    const int seen = i + 1 + prompt_offset(n, n_keys);
    return seen < 0 ? 0 : seen;
}
// Workgroups that a CU holds at a time, by the registers and the LDS of the kernel for aligned rows (size: bytes of an element)
constexpr int prompt_resident(int size, int hd) { return size == 2 ? hd <= 64 ? 4 : hd <= 128 ? 3 : 2 : hd <= 32 ? 5 : hd <= 64 ? 4 : hd <= 96 ? 3 : hd <= 128 ? 2 : 1; }
// How many splits there are of a tile whose rows see n_keys_seen keys, of at most n_splits, of `per` blocks each (the last of all takes what is left)
constexpr int prompt_splits(int n_keys_seen, int block, int n_splits, int per) {
    const int blocks = (n_keys_seen + block - 1) / block, want = (blocks + per - 1) / per;
    return want < 1 ? 1 : want < n_splits ? want : n_splits;
}
// Blocks [first, last) of split `split`, whether there is such a split, and whether there is more than one
struct PromptBlocks { int first, last; bool any, several; };
constexpr PromptBlocks prompt_blocks(int n_keys_seen, int block, int split, int n_splits, int per) {
    const int blocks = (n_keys_seen + block - 1) / block, splits = prompt_splits(n_keys_seen, block, n_splits, per);
    PromptBlocks r{split * per < blocks ? split * per : blocks, blocks, split < splits, splits > 1};
    if (split + 1 < splits) r.last = r.first + per;
    return r;
}

// Where the 16-byte piece c of token t's row of row_bytes lies within a block in LDS: at piece prompt_swizzle(...) of the row.  Reads of a piece of
// 8 tokens in a row, and of 64 bytes of 4 tokens, then go to different banks; rows of an odd multiple of 64 bytes do so half by themselves.
constexpr int prompt_swizzle(int t, int c, int row_bytes) {
    const int s = row_bytes % 128 == 64 ? 0 : row_bytes % 256 == 128 ? (t >> 1) & 1 : t & 3;
    return c ^ (s << 2 | ((t >> 2) & 3));
}
