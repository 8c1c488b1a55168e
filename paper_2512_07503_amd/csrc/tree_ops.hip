// Entry points of the tree operators but for the verification (tree_verify.hip): rotary positions, the paged cache, tree attention.
#include <math.h>

#include "common.hip.h"
#include "kernels_cache.hip.h"
#include "kernels_rotary.hip.h"
#include "kernels_tree.hip.h"
#include "tree_ops.h"

namespace {

#define TREE_FAIL(code, ...)                            \
    do {                                                \
        sjd_set_error(sjd_call_error(), __VA_ARGS__);   \
        return code;                                    \
    } while (0)
#define TREE_TRY(expr) SJD_HIP_TRY(sjd_call_error(), expr)

// A launch has at most 2^32 - 1 work-items a dimension: so many workgroups of 256
constexpr size_t kMaxWorkgroups = (1u << 24) - 1;

bool wide(const void *p, int64_t stride, int size, int bytes) { return (uintptr_t)p % bytes == 0 && stride * size % bytes == 0; }

int check_shape(const sjd_kv_cache *c) {
    if (!c) TREE_FAIL(SJD_EINVAL, "null cache");
    if (c->dtype != SJD_F32 && c->dtype != SJD_BF16 && c->dtype != SJD_FP8) TREE_FAIL(SJD_EINVAL, "unknown cache dtype %d", c->dtype);
    if (c->page_tokens < 32 || c->page_tokens % 32 || c->page_tokens > 1 << 20) TREE_FAIL(SJD_EINVAL, "page_tokens must be a multiple of 32");
    if (c->n_kv_heads < 1 || c->n_kv_heads > 65535) TREE_FAIL(SJD_EINVAL, "n_kv_heads must be 1 .. 65535");
    switch (c->head_dim) {
    case 32: case 64: case 96: case 128: case 192: case 256: return SJD_OK;
    }
    TREE_FAIL(SJD_EINVAL, "head_dim must be 32, 64, 96, 128, 192 or 256");
}

int check_cache(const sjd_kv_cache *c) {
    const int rc = check_shape(c);
    if (rc) return rc;
    if (!c->pages || (uintptr_t)c->pages % 16 || !c->page_table) TREE_FAIL(SJD_EINVAL, "pages (16-byte aligned) or page_table missing");
    if (c->n_pages < 1 || c->n_seqs < 1 || c->pages_per_seq < 1) TREE_FAIL(SJD_EINVAL, "n_pages, n_seqs and pages_per_seq must be positive");
    if ((int64_t)c->pages_per_seq * c->page_tokens > 1 << 30) TREE_FAIL(SJD_EINVAL, "a sequence has at most 2^30 positions");
    return SJD_OK;
}

CacheView view(const sjd_kv_cache *c) {
    return CacheView{(unsigned char *)c->pages, c->page_table, c->n_pages, c->page_tokens, c->n_kv_heads, c->head_dim, c->n_seqs, c->pages_per_seq,
                     cache_block_bytes(c->dtype, c->page_tokens, c->head_dim)};
}

// kernel of the (cache kind, row type) instance
template <template <int, typename> class K, typename Args> hipError_t launch_rows(hipStream_t st, dim3 grid, int kind, int dtype, const Args &a) {
    const bool f32 = dtype == SJD_F32;
    switch (kind) {
    case SJD_F32: f32 ? K<SJD_F32, float>::run(st, grid, a) : K<SJD_F32, bf16_t>::run(st, grid, a); break;
    case SJD_BF16: f32 ? K<SJD_BF16, float>::run(st, grid, a) : K<SJD_BF16, bf16_t>::run(st, grid, a); break;
    default: f32 ? K<SJD_FP8, float>::run(st, grid, a) : K<SJD_FP8, bf16_t>::run(st, grid, a); break;
    }
    return hipGetLastError();
}
template <int KIND, typename T> struct WriteRows {
    static void run(hipStream_t st, dim3 grid, const CacheRowsArgs &a) { cache_write_kernel<KIND, T><<<grid, 256, 0, st>>>(a); }
};
template <int KIND, typename T> struct ReadRows {
    static void run(hipStream_t st, dim3 grid, const CacheRowsArgs &a) { cache_read_kernel<KIND, T><<<grid, 256, 0, st>>>(a); }
};

// kv heads that a workgroup of a write or a read takes: several once there are 16 workgroups a compute unit without (7808 of them: write 28.4 us
// for 33.1, read 18.6 for 22.5), one below, where what counts is how long a workgroup takes (1200: read 10.0 us for 13.5; 128: write 5.7 for 6.8)
int head_group(const sjd_kv_cache *c, int n_rows) {
    return 2 * cache_max_tiles(n_rows, c->n_seqs) * c->n_kv_heads >= 4096 ? cache_heads(c->head_dim) : 1;
}
unsigned head_groups(const sjd_kv_cache *c, int group) { return (unsigned)(c->n_kv_heads + group - 1) / group; }

// Do n_rows rows of x and of y, x_row and y_row elements long, have no element in common?  (Rows with the same stride may interleave: parts of a
// fused projection.)
bool rows_apart(const void *x, long x_stride, long x_row, const void *y, long y_stride, long y_row, int n_rows, int size) {
    const uintptr_t x0 = (uintptr_t)x, x1 = x0 + ((uintptr_t)(n_rows - 1) * x_stride + x_row) * size;
    const uintptr_t y0 = (uintptr_t)y, y1 = y0 + ((uintptr_t)(n_rows - 1) * y_stride + y_row) * size;
    if (x1 <= y0 || y1 <= x0) return true;
    if (n_rows == 1 || x_stride != y_stride || x_stride <= 0) return false;
    const long d = ((long)(y0 - x0) / size % x_stride + x_stride) % x_stride;   // where y's row starts within x's
    return d >= x_row && d + y_row <= x_stride;
}

int check_rows(const sjd_kv_cache *cache, int32_t dtype, const void *k, const void *v, const int32_t *row_start, const int32_t *first_pos, int32_t n_rows) {
    const int rc = check_cache(cache);
    if (rc) return rc;
    if (dtype != SJD_F32 && dtype != SJD_BF16) TREE_FAIL(SJD_EINVAL, "rows are SJD_F32 or SJD_BF16");
    if (n_rows < 0 || n_rows > 1 << 29) TREE_FAIL(SJD_EINVAL, "n_rows must be 0 .. 2^29");
    if (!row_start || !first_pos || (n_rows && (!k || !v))) TREE_FAIL(SJD_EINVAL, "null argument");
    if ((size_t)cache_max_tiles(n_rows, cache->n_seqs) > kMaxWorkgroups) TREE_FAIL(SJD_EINVAL, "too many rows or sequences for one launch");
    const unsigned size = dtype == SJD_F32 ? 4 : 2;
    if ((uintptr_t)k % size || (uintptr_t)v % size) TREE_FAIL(SJD_EINVAL, "rows are not aligned to their elements");
    return SJD_OK;
}

// ------------------------------------------------------------------------------------------------------------- attention
struct TreePlan { int tiles, groups, n_splits; bool by_rows; size_t part_o, part_ml; };

// Which kernel, and how many ways a context is split.  By rows, where a bf16 cache has more than two tiles of 32 rows a kv head: four tiles a
// workgroup share what is fetched (by rows against by tokens, calls in turn: 16 sequences of 7 000 tokens, 8 kv heads of 128, 244 rows: 187 us against 225, 80
// rows: 103 against 126; 5 200 - 11 200 tokens and 176 - 312 rows: 179 against 207; one of 2 300 with 32 heads of 96 rows: 26.9 against 28.2).  A variant by rows for fp8,
// whose conversions it does not save a wavefront but moves, was slower and is not here any more (185 us against 178 then for the sixteen sequences, with
// heads of 64 151 against 110).
TreePlan tree_plan(const sjd_kv_cache *c, int n_heads, int max_rows, int max_ctx) {
    TreePlan p;
    const int G = n_heads / c->n_kv_heads;
    p.tiles = (int)ceil_div_sz((size_t)max_rows * G, 32);
    p.by_rows = c->dtype == SJD_BF16 && p.tiles > 2 && c->head_dim <= 192;     // (heads of 256 would spill registers)
    const int per_group = p.by_rows ? kTreeRowWaves : 1;
    p.groups = ceil_div(p.tiles, per_group);
    p.tiles = p.groups * per_group;
    const size_t work = (size_t)c->n_seqs * c->n_kv_heads * p.groups, blocks = ceil_div_sz((size_t)max_ctx + max_rows, 32);
    // two workgroups for each of the 256 CUs, but no split with less than two blocks of 32 tokens for each of a workgroup's wavefronts, on which its
    // merge would weigh more than its share of the stream
    const size_t want = ceil_div_sz(512, work), most = blocks / (2 * kTreeWaves) ? blocks / (2 * kTreeWaves) : 1;
    p.n_splits = (int)(want < most ? want : most);
    const size_t slots = p.n_splits > 1 ? (size_t)c->n_seqs * c->n_kv_heads * p.n_splits * p.tiles : 0;
    p.part_o = slots * 32 * c->head_dim * sizeof(float);
    p.part_ml = slots * 64 * sizeof(float);
    return p;
}

int check_attention(const sjd_kv_cache *c, int32_t n_heads, int32_t max_rows, int32_t max_ctx) {
    if (n_heads < 1 || n_heads % c->n_kv_heads || n_heads > 1 << 20) TREE_FAIL(SJD_EINVAL, "n_heads must be a multiple of n_kv_heads");
    if (max_rows < 1 || max_rows > 1 << 16 || max_ctx < 0 || max_ctx > 1 << 30) TREE_FAIL(SJD_EINVAL, "max_rows must be 1 .. 65536, max_ctx 0 .. 2^30");
    const size_t pairs = (size_t)c->n_seqs * c->n_kv_heads;
    // (so many at least, of four tiles of 32 rows; what follows stays within its integers)
    if (pairs > kMaxWorkgroups || (size_t)max_rows * (n_heads / c->n_kv_heads) > kMaxWorkgroups * 128) TREE_FAIL(SJD_EINVAL, "too many rows for one launch");
    const TreePlan p = tree_plan(c, n_heads, max_rows, max_ctx);
    // (of the kernel: its workgroups come in eights, for the XCDs; of the joining of splits: 256 threads own four dimensions each)
    if (pairs * p.tiles > 1u << 24 || ceil_div_sz(pairs * p.n_splits, 8) * 8 * p.groups > kMaxWorkgroups ||
        (p.n_splits > 1 && pairs * p.tiles * ceil_div(8 * c->head_dim, 256) > kMaxWorkgroups)) TREE_FAIL(SJD_EINVAL, "too many rows for one launch");
    return SJD_OK;
}

template <int KIND, int HD> void run_tree(hipStream_t st, const TreeArgs &a, bool by_rows) {
    if constexpr (KIND == SJD_BF16 && HD <= 192)
        if (by_rows) {
            tree_attention_rows_kernel<HD><<<tree_grid(a), kTreeRowThreads, 0, st>>>(a);
            return;
        }
    tree_attention_kernel<KIND, HD><<<tree_grid(a), kTreeWaves * 64, 0, st>>>(a);
}
template <int KIND> void run_tree_kind(hipStream_t st, const TreeArgs &a, bool by_rows) {
    switch (a.c.hd) {
    case 32: run_tree<KIND, 32>(st, a, by_rows); break;
    case 64: run_tree<KIND, 64>(st, a, by_rows); break;
    case 96: run_tree<KIND, 96>(st, a, by_rows); break;
    case 128: run_tree<KIND, 128>(st, a, by_rows); break;
    case 192: run_tree<KIND, 192>(st, a, by_rows); break;
    default: run_tree<KIND, 256>(st, a, by_rows); break;
    }
}

}  // namespace

extern "C" {

int sjd_cache_page_bytes(const sjd_kv_cache *cache, uint64_t *bytes) {
    const int rc = check_shape(cache);
    if (rc) return rc;
    if (!bytes) TREE_FAIL(SJD_EINVAL, "null argument");
    *bytes = cache_block_bytes(cache->dtype, cache->page_tokens, cache->head_dim) * cache->n_kv_heads;
    return SJD_OK;
}

int sjd_op_cache_write(void *hip_stream, const sjd_kv_cache *cache, int32_t src_dtype, const void *k, int64_t k_stride, const void *v,
                       int64_t v_stride, const int32_t *row_start, const int32_t *first_pos, int32_t n_rows) {
    const int rc = check_rows(cache, src_dtype, k, v, row_start, first_pos, n_rows);
    if (rc) return rc;
    if (!n_rows) return SJD_OK;
    const int size = src_dtype == SJD_F32 ? 4 : 2;
    const CacheRowsArgs a = {view(cache), row_start, first_pos, const_cast<void *>(k), const_cast<void *>(v), (long)k_stride, (long)v_stride, n_rows, head_group(cache, n_rows),
                             wide(k, k_stride, size, 16), wide(v, v_stride, size, 16)};
    TREE_TRY(launch_rows<WriteRows>((hipStream_t)hip_stream, dim3((unsigned)cache_max_tiles(n_rows, cache->n_seqs), head_groups(cache, a.group), 2), cache->dtype,
                                    src_dtype, a));
    return SJD_OK;
}

int sjd_op_cache_read(void *hip_stream, const sjd_kv_cache *cache, int32_t dst_dtype, void *k, void *v, const int32_t *row_start,
                      const int32_t *first_pos, int32_t n_rows) {
    const int rc = check_rows(cache, dst_dtype, k, v, row_start, first_pos, n_rows);
    if (rc) return rc;
    if (!n_rows) return SJD_OK;
    const int size = dst_dtype == SJD_F32 ? 4 : 2;
    const long stride = (long)cache->n_kv_heads * cache->head_dim;
    if (!rows_apart(k, stride, stride, v, stride, stride, n_rows, size)) TREE_FAIL(SJD_EINVAL, "k and v overlap");
    const CacheRowsArgs a = {view(cache), row_start, first_pos, k, v, stride, stride, n_rows, head_group(cache, n_rows), wide(k, stride, size, 16), wide(v, stride, size, 16)};
    TREE_TRY(launch_rows<ReadRows>((hipStream_t)hip_stream, dim3((unsigned)cache_max_tiles(n_rows, cache->n_seqs), head_groups(cache, a.group), 2), cache->dtype,
                                   dst_dtype, a));
    return SJD_OK;
}

int sjd_op_cache_compact(void *hip_stream, const sjd_kv_cache *cache, const int32_t *first_pos, const int32_t *path, const int32_t *path_len,
                         int32_t max_path) {
    const int rc = check_cache(cache);
    if (rc) return rc;
    if (!first_pos || !path || !path_len || max_path < 1) TREE_FAIL(SJD_EINVAL, "null argument or max_path < 1");
    if ((size_t)cache->n_seqs > kMaxWorkgroups) TREE_FAIL(SJD_EINVAL, "too many sequences for one launch");
    const dim3 grid(cache->n_seqs, cache->n_kv_heads, 2);
    hipStream_t st = (hipStream_t)hip_stream;
    const CacheView c = view(cache);
    if (cache->dtype == SJD_F32) cache_compact_kernel<SJD_F32><<<grid, 256, 0, st>>>(c, first_pos, path, path_len, max_path);
    else if (cache->dtype == SJD_BF16) cache_compact_kernel<SJD_BF16><<<grid, 256, 0, st>>>(c, first_pos, path, path_len, max_path);
    else cache_compact_kernel<SJD_FP8><<<grid, 256, 0, st>>>(c, first_pos, path, path_len, max_path);
    TREE_TRY(hipGetLastError());
    return SJD_OK;
}

int sjd_rope_table(int32_t rotary_dim, double theta, int32_t scaling, double factor, double trained_ctx, double low_turns, double high_turns,
                   uint64_t *table) {
    if (!table || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 2 * kRotaryMaxHalf) TREE_FAIL(SJD_EINVAL, "rotary_dim must be even, 2 .. 512");
    if (!(theta > 1.0) || !(theta < INFINITY)) TREE_FAIL(SJD_EINVAL, "theta must be above 1");
    if (scaling < SJD_ROPE_PLAIN || scaling > SJD_ROPE_PARTS) TREE_FAIL(SJD_EINVAL, "unknown scaling %d", scaling);
    if (scaling != SJD_ROPE_PLAIN && (!(factor >= 1.0) || !(factor < INFINITY))) TREE_FAIL(SJD_EINVAL, "factor must be at least 1");
    if (scaling == SJD_ROPE_BASE && rotary_dim == 2) TREE_FAIL(SJD_EINVAL, "another base has no effect on a single pair");
    if (scaling == SJD_ROPE_PARTS && (!(trained_ctx > 0.0) || !(trained_ctx < INFINITY) || !(low_turns >= 0.0) || !(high_turns > low_turns)))
        TREE_FAIL(SJD_EINVAL, "trained_ctx > 0 and 0 <= low_turns < high_turns are needed");
    const long double two_pi = 6.283185307179586476925286766559005768L;
    const long double base = scaling == SJD_ROPE_BASE ? (long double)theta * powl(factor, (long double)rotary_dim / (rotary_dim - 2)) : (long double)theta;
    for (int i = 0; i < rotary_dim / 2; ++i) {
        long double f = powl(base, -2.0L * i / rotary_dim);
        if (scaling == SJD_ROPE_LINEAR) f /= factor;
        if (scaling == SJD_ROPE_PARTS) {
            const long double turns = trained_ctx * f / two_pi;
            long double keep = (turns - low_turns) / ((long double)high_turns - low_turns);
            keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
            f *= keep + (1.0L - keep) / factor;
        }
        table[i] = (uint64_t)(f / two_pi * 18446744073709551616.0L + 0.5L);   // f <= 1: below 2^62
    }
    return SJD_OK;
}

int sjd_op_rotary(void *hip_stream, int32_t dtype, int32_t interleaved, const uint64_t *table, int32_t rotary_dim, float magnitude,
                  const int32_t *positions, int32_t n_rows, int32_t head_dim, const void *q, int64_t q_stride, void *q_out,
                  int64_t q_out_stride, int32_t n_heads, const void *k, int64_t k_stride, void *k_out, int64_t k_out_stride,
                  int32_t n_kv_heads) {
    if (dtype != SJD_F32 && dtype != SJD_BF16) TREE_FAIL(SJD_EINVAL, "rows are SJD_F32 or SJD_BF16");
    if (head_dim < 2 || head_dim > 2 * kRotaryMaxHalf || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > head_dim)
        TREE_FAIL(SJD_EINVAL, "rotary_dim must be even and 2 .. head_dim, head_dim at most 512");
    if (n_heads < 1 || n_kv_heads < 0 || n_heads > 1 << 16 || n_kv_heads > 1 << 16 || n_rows < 0 || n_rows > 1 << 29)
        TREE_FAIL(SJD_EINVAL, "n_heads must be 1 .. 65536, n_kv_heads 0 .. 65536, n_rows 0 .. 2^29");
    if (!table || (n_rows && (!positions || !q || !q_out || (n_kv_heads && (!k || !k_out))))) TREE_FAIL(SJD_EINVAL, "null argument");
    const int size = dtype == SJD_F32 ? 4 : 2;
    RotaryArgs a = {table, positions, {q, k}, {q_out, k_out}, {(long)q_stride, (long)k_stride}, {(long)q_out_stride, (long)k_out_stride},
                    {n_heads, n_kv_heads}, n_rows, head_dim, rotary_dim / 2, interleaved ? 1 : 0, 1, magnitude};
    bool w = interleaved ? head_dim % 8 == 0 : a.half % 8 == 0 && (head_dim - rotary_dim) % 8 == 0;
    for (int s = 0; s < 2; ++s) {
        const long row = (long)a.heads[s] * head_dim;
        if (!row || !n_rows) continue;
        if ((uintptr_t)a.x[s] % size || (uintptr_t)a.y[s] % size) TREE_FAIL(SJD_EINVAL, "rows are not aligned to their elements");
        if (n_rows > 1 && a.y_stride[s] < row) TREE_FAIL(SJD_EINVAL, "output rows overlap");
        if (n_rows > 1 && a.x_stride[s] < 0) TREE_FAIL(SJD_EINVAL, "negative stride");
        w = w && wide(a.x[s], a.x_stride[s], size, 16) && wide(a.y[s], a.y_stride[s], size, 16);
        for (int o = 0; o < 2; ++o) {
            const long out_row = (long)a.heads[o] * head_dim;
            const bool same = o == s && a.x[s] == a.y[s] && (a.x_stride[s] == a.y_stride[s] || n_rows == 1);
            if (out_row && !same && !rows_apart(a.x[s], a.x_stride[s], row, a.y[o], a.y_stride[o], out_row, n_rows, size))
                TREE_FAIL(SJD_EINVAL, "an output overlaps an input");
        }
    }
    if (!n_rows) return SJD_OK;
    if (n_kv_heads && !rows_apart(q_out, q_out_stride, (long)n_heads * head_dim, k_out, k_out_stride, (long)n_kv_heads * head_dim, n_rows, size))
        TREE_FAIL(SJD_EINVAL, "q_out and k_out overlap");
    // Rows a workgroup: their sines and cosines are shared by the heads of a row only, so more rows mean nothing but fewer workgroups;
    // two for each of the 256 CUs, and few rows are split over their heads' units instead.
    while (a.rows_per_wg < 8 && a.rows_per_wg * a.half * 2 <= 8 * kRotaryMaxHalf && n_rows / (2 * a.rows_per_wg) >= 512) a.rows_per_wg *= 2;
    const unsigned gx = (unsigned)ceil_div(n_rows, a.rows_per_wg);
    if (gx > kMaxWorkgroups) TREE_FAIL(SJD_EINVAL, "too many rows for one launch");
    const long units = (long)a.rows_per_wg * (n_heads + n_kv_heads) * (w ? head_dim / 8 : head_dim);
    long gy = gx >= 512 ? 1 : 512 / gx;
    if (gy > (units + 255) / 256) gy = (units + 255) / 256;
    const dim3 grid(gx, (unsigned)gy);
    hipStream_t st = (hipStream_t)hip_stream;
    if (dtype == SJD_F32) w ? rotary_kernel<float, true><<<grid, 256, 0, st>>>(a) : rotary_kernel<float, false><<<grid, 256, 0, st>>>(a);
    else w ? rotary_kernel<bf16_t, true><<<grid, 256, 0, st>>>(a) : rotary_kernel<bf16_t, false><<<grid, 256, 0, st>>>(a);
    TREE_TRY(hipGetLastError());
    return SJD_OK;
}

int sjd_tree_masks(const int32_t *parents, int32_t n, int32_t mask_words, uint32_t *mask, int32_t *depth) {
    if (n < 0 || (n && (!parents || !mask)) || mask_words < 0 || (int64_t)mask_words * 32 < n) TREE_FAIL(SJD_EINVAL, "null argument, or too few mask words");
    for (int32_t i = 0; i < n; ++i)
        if (parents[i] >= i) TREE_FAIL(SJD_EINVAL, "node %d: its parent %d does not come first", i, parents[i]);
    for (int32_t i = 0; i < n; ++i) {
        const int32_t p = parents[i];
        uint32_t *row = mask + (size_t)i * mask_words;
        for (int32_t w = 0; w < mask_words; ++w) row[w] = p >= 0 ? mask[(size_t)p * mask_words + w] : 0u;
        row[i >> 5] |= 1u << (i & 31);
        if (depth) depth[i] = p >= 0 ? depth[p] + 1 : 0;
    }
    return SJD_OK;
}

int sjd_op_tree_attention_workspace(const sjd_kv_cache *cache, int32_t n_heads, int32_t max_rows, int32_t max_ctx, uint64_t *bytes) {
    int rc = check_shape(cache);
    if (rc) return rc;
    if (!bytes || cache->n_seqs < 1) TREE_FAIL(SJD_EINVAL, "null argument or n_seqs < 1");
    if ((rc = check_attention(cache, n_heads, max_rows, max_ctx))) return rc;
    const TreePlan p = tree_plan(cache, n_heads, max_rows, max_ctx);
    *bytes = p.part_o + p.part_ml;
    return SJD_OK;
}

int sjd_op_tree_attention(void *hip_stream, const sjd_kv_cache *cache, int32_t dtype, const void *q, int64_t q_stride, void *out,
                          int64_t out_stride, const int32_t *row_start, const int32_t *ctx_len, const uint32_t *mask, int32_t mask_words,
                          int32_t n_rows, int32_t n_heads, float scale, int32_t max_rows, int32_t max_ctx, void *workspace,
                          uint64_t workspace_bytes) {
    int rc = check_cache(cache);
    if (rc) return rc;
    if ((rc = check_attention(cache, n_heads, max_rows, max_ctx))) return rc;
    if (dtype != (cache->dtype == SJD_F32 ? SJD_F32 : SJD_BF16)) TREE_FAIL(SJD_EINVAL, "rows are SJD_F32 for an SJD_F32 cache, SJD_BF16 for the others");
    if (n_rows < 0 || n_rows > 1 << 29 || (n_rows && (!q || !out)) || !row_start || !ctx_len) TREE_FAIL(SJD_EINVAL, "null argument, or n_rows out of 0 .. 2^29");
    if (!(scale >= 0.0f) || !(scale < INFINITY)) TREE_FAIL(SJD_EINVAL, "scale must be positive, or 0 for 1 / sqrt(head_dim)");
    if (mask && (mask_words < 1 || (uintptr_t)mask % 4)) TREE_FAIL(SJD_EINVAL, "a mask needs mask_words >= 1 and 4-byte alignment");
    const int size = dtype == SJD_F32 ? 4 : 2;
    if ((uintptr_t)q % size || (uintptr_t)out % size) TREE_FAIL(SJD_EINVAL, "rows are not aligned to their elements");
    if (n_rows > 1 && out_stride < (int64_t)n_heads * cache->head_dim) TREE_FAIL(SJD_EINVAL, "output rows overlap");
    if (n_rows > 1 && q_stride < 0) TREE_FAIL(SJD_EINVAL, "negative stride");
    if (!n_rows) return SJD_OK;
    // in place: a workgroup has read its queries when it writes their results
    const long row = (long)n_heads * cache->head_dim;
    if (!(q == out && (q_stride == out_stride || n_rows == 1)) && !rows_apart(q, q_stride, row, out, out_stride, row, n_rows, size))
        TREE_FAIL(SJD_EINVAL, "the output overlaps the queries");
    const TreePlan p = tree_plan(cache, n_heads, max_rows, max_ctx);
    if (p.part_o + p.part_ml > workspace_bytes)
        TREE_FAIL(SJD_ECAPACITY, "the workspace holds %llu bytes, %zu are needed", (unsigned long long)workspace_bytes, p.part_o + p.part_ml);
    if (p.part_o && (!workspace || (uintptr_t)workspace % 16)) TREE_FAIL(SJD_EINVAL, "the workspace must be 16-byte aligned");
    TreeArgs a;
    a.c = view(cache);
    a.q = q; a.out = out; a.q_stride = q_stride; a.out_stride = out_stride;
    a.row_start = row_start; a.ctx_len = ctx_len; a.mask = mask;
    a.mask_words = mask_words; a.n_rows = n_rows; a.max_rows = max_rows; a.H = n_heads; a.G = n_heads / cache->n_kv_heads;
    a.tiles = p.tiles; a.groups = p.groups; a.n_splits = p.n_splits;
    a.scale_log2e = (float)(1.4426950408889634 * (scale > 0.0f ? (double)scale : 1.0 / sqrt((double)cache->head_dim)));
    a.part_o = (float *)workspace;
    a.part_ml = (float *)((char *)workspace + p.part_o);
    a.q_wide = wide(q, q_stride, size, 16);
    a.out_wide = wide(out, out_stride, size, 4 * size);
    hipStream_t st = (hipStream_t)hip_stream;
    if (cache->dtype == SJD_F32) run_tree_kind<SJD_F32>(st, a, p.by_rows);
    else if (cache->dtype == SJD_BF16) run_tree_kind<SJD_BF16>(st, a, p.by_rows);
    else run_tree_kind<SJD_FP8>(st, a, p.by_rows);
    TREE_TRY(hipGetLastError());
    if (a.n_splits > 1) {
        if (dtype == SJD_F32) launch_tree_combine<SJD_F32>(st, a);
        else launch_tree_combine<SJD_BF16>(st, a);
        TREE_TRY(hipGetLastError());
    }
    return SJD_OK;
}

}  // extern "C"
