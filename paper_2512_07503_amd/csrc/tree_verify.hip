// Verification of a tree of drafted tokens against the target's probabilities, from given random words.
//
// Every result is specified bit for bit, in double precision and integers, so that it does not depend on how the work is divided:
//   rho_0(v) = p(v) (0 where p is negative or NaN),  S_0 = 1
//   child k of a node, token x:  accepted where (r * q(x)) * S_k < rho_k(x),  r = (u32 + 1/2) 2^-32
//   else  rho_{k+1}(v) = max(0, rho_k(v) - S_k * q(v)),  S_{k+1} = 2^-44 * sum_v w(rho_{k+1}(v)),  w(y) = trunc(min(y, 1) * 2^44)
//   without q the proposal is certain: q(x) = 1, and rho_{k+1} = rho_k but for rho_{k+1}(x) = 0
//   the next token: first v with prefix_w(v) > floor(u64 * Z / 2^64), w of the last rho of the last accepted node, Z = sum_v w; of p if Z = 0
// With rho normalised by S_k this is the acceptance of Eq. 2 of the paper, min(1, rho / q), and the residual of Eq. 3, once per sibling:
// what a rejected proposal could have been is taken off, and the next sibling is tested against the rest.
//
// What a node decides follows from its own rows alone, so all nodes are decided at once, and the path is walked afterwards. A first child
// takes two values; a sum over the vocabulary is needed only for a second child whose first sibling was rejected, at a node that is
// not ruled out by the first children above it.  Bound by latency: two rows a sequence are all that has to be read, but
// what a node needs next is known only when its last sum is: 16 trees of 61 nodes over 65 536 ids, 36.4 + 7.2 + 7.4 us for the three launches; one window of
// 16 over 16 384 ids, 3.4 + 5.0 + 5.6 us.
//
// This translation unit must be compiled with -ffp-contract=off.
#include "cache_layout.h"
#include "common.hip.h"
#include "tree_ops.h"

#pragma clang fp contract(off)

namespace {

constexpr int kMaxNodes = 1024, kMaxVocab = 1 << 19;
constexpr int kSlice = 2048;          // ids of a row that a workgroup sums for the last draw
constexpr int kNodeThreads = 1024;    // of a node's workgroup; <= 512 ids a thread, whose sums are exact in a double

struct VerifyArgs {
    const int32_t *tokens, *parents, *row_start;
    const float *p, *q;
    long p_stride, q_stride;
    const uint32_t *accept_words;
    const uint64_t *draw_words;
    int32_t *path, *path_len, *next_token;
    int n_rows, n_seqs, max_rows, max_path, V, n_slices;
    bool wide;                 // rows 16-byte aligned
    // workspace
    int32_t *choice;           // [n_rows]  accepted child of a node, -1: none
    double *mass;              // [n_rows]  S after the rejection of that node
    uint64_t *part;            // [n_seqs][n_slices][2]  sums of a slice: of the last rho, of p
    int32_t *stop;             // [n_seqs][2]  row of the last accepted node (-1: empty tree), number of its rejected children
    double *stop_mass;         // [n_rows]  S_0, S_1, ... of these, at the sequence's rows
    int32_t *stop_token;       // [n_rows]  their tokens
};

SJD_D void tree_rows(const VerifyArgs &a, int b, int &r0, int &n) {
    r0 = rows_first(a.row_start, b, a.n_rows);
    n = min(rows_count(a.row_start, b, a.n_rows), a.max_rows);
}
// p of an id as rho_0: NaN and negatives are 0
SJD_D float target(float p) { return fmaxf(p, 0.0f); }
SJD_D double positive(double x) { return fmax(x, 0.0); }                       // (NaN -> 0)
SJD_D double weight(double y) { return __builtin_trunc(fmin(y, 1.0) * 0x1p44); }
// rho after `m` >= 1 rejections (S_0 = 1)
SJD_D double residual(float p, float q, const double *mass, int m) {
    double r = positive((double)target(p) - (double)q);
    for (int k = 1; k < m; ++k) r = positive(r - mass[k] * (double)q);
    return r;
}
SJD_D bool accepts(uint32_t word, double q, double mass, double rho) {
    const double r = ((double)word + 0.5) * 0x1p-32;
    return (r * q) * mass < rho;
}

SJD_D uint64_t shfl_xor_u64(uint64_t v, int d) {
    const uint32_t lo = __shfl_xor((uint32_t)v, d, 64), hi = __shfl_xor((uint32_t)(v >> 32), d, 64);
    return (uint64_t)hi << 32 | lo;
}
template <int NW> SJD_D uint64_t block_sum(uint64_t v, uint64_t *scratch /* NW */) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += shfl_xor_u64(v, d);
    __syncthreads();
    if (lane == 0) scratch[wave] = v;
    __syncthreads();
    uint64_t t = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) t += scratch[i];
    return t;
}

SJD_D bool known(const VerifyArgs &a, int x) { return (unsigned)x < (unsigned)a.V; }

// Is the first child of the node in row `row` accepted
SJD_D bool first_accepted(const VerifyArgs &a, int r0, int node, int child) {
    const int x = a.tokens[r0 + child];
    if (!known(a, x)) return false;
    const size_t row = (size_t)(r0 + node);
    const double q = a.q ? (double)a.q[row * a.q_stride + x] : 1.0;
    return accepts(a.accept_words[r0 + child], q, 1.0, (double)target(a.p[row * a.p_stride + x]));
}

// f(id, p, q) for every id of a row, 4 ids at a time, U times 4 of them on their way (one round trip to memory for all)
template <int THREADS, int U, typename F> SJD_D void for_row(const VerifyArgs &a, const float *p, const float *q, int lo, int hi, F f) {
    if (a.wide) {
        for (int v0 = lo + 4 * threadIdx.x; v0 < hi; v0 += 4 * THREADS * U) {
            float4 pv[U], qv[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = v0 + 4 * THREADS * u;
                if (v + 4 <= hi) {
                    pv[u] = *reinterpret_cast<const float4 *>(p + v);
                    qv[u] = q ? *reinterpret_cast<const float4 *>(q + v) : float4{0.0f, 0.0f, 0.0f, 0.0f};
                } else {
                    float x[4], y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = v + e < hi ? p[v + e] : 0.0f;
                        y[e] = v + e < hi && q ? q[v + e] : 0.0f;
                    }
                    pv[u] = float4{x[0], x[1], x[2], x[3]};
                    qv[u] = float4{y[0], y[1], y[2], y[3]};
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = v0 + 4 * THREADS * u;
                if (v >= hi) continue;
                f(v, pv[u].x, qv[u].x); f(v + 1, pv[u].y, qv[u].y); f(v + 2, pv[u].z, qv[u].z); f(v + 3, pv[u].w, qv[u].w);
            }
        }
    } else {
        for (int v = lo + threadIdx.x; v < hi; v += THREADS) f(v, p[v], q ? q[v] : 0.0f);
    }
}

// A thread's share of sum_v w(rho_m(v)): of integers, at most 512 of up to 2^44, exact in a double.  The first few rejections, which is what nodes
// have, without a loop per id (16 trees of 61 nodes over 65 536 ids: 36.7 us in place of 45.9 with one).
template <int M> SJD_D double row_mass_of(const VerifyArgs &a, const float *p, const float *q, const double *mass) {
    double s[M > 1 ? M : 1], sum = 0.0;
#pragma unroll
    for (int k = 1; k < M; ++k) s[k] = mass[k];
    for_row<kNodeThreads, 8>(a, p, q, 0, a.V, [&](int, float pv, float qv) {
        double r = (double)target(pv);
        if (M > 0) r = positive(r - (double)qv);
#pragma unroll
        for (int k = 1; k < M; ++k) r = positive(r - s[k] * (double)qv);
        sum += weight(r);
    });
    return sum;
}
SJD_D double row_mass(const VerifyArgs &a, const float *p, const float *q, const double *mass, int m) {
    switch (m) {
    case 0: return row_mass_of<0>(a, p, q, mass);
    case 1: return row_mass_of<1>(a, p, q, mass);
    case 2: return row_mass_of<2>(a, p, q, mass);
    case 3: return row_mass_of<3>(a, p, q, mass);
    case 4: return row_mass_of<4>(a, p, q, mass);
    }
    double sum = 0.0;
    for_row<kNodeThreads, 8>(a, p, q, 0, a.V, [&](int, float pv, float qv) { sum += weight(residual(pv, qv, mass, m)); });
    return sum;
}

// Workgroup = node of a tree: which of its children is accepted
__global__ __launch_bounds__(kNodeThreads) void verify_nodes_kernel(VerifyArgs a) {
    const int b = blockIdx.y, node = blockIdx.x, tid = threadIdx.x;
    int r0, n;
    tree_rows(a, b, r0, n);
    if (node >= n) return;
    __shared__ int parent[kMaxNodes], first[kMaxNodes], child[kMaxNodes], wave_count[kNodeThreads / 64], flag;
    __shared__ int token[kMaxNodes];            // of the children: tokens (-1: outside the vocabulary), test words, p and q of the tokens
    __shared__ uint32_t word[kMaxNodes];
    __shared__ float token_p[kMaxNodes], token_q[kMaxNodes];
    __shared__ bool repeat[kMaxNodes];
    __shared__ double mass[kMaxNodes];
    __shared__ uint64_t scratch[kNodeThreads / 64];
    const int mine = tid < n ? a.parents[r0 + tid] : -1;
    const bool is_child = tid > node && tid < n && mine == node;
    // children in ascending order
    const unsigned long long here = __ballot(is_child);
    const int lane = tid & 63, wave = tid >> 6;
    if (lane == 0) wave_count[wave] = __popcll(here);
    __syncthreads();
    int before = 0, m = 0;
    for (int w = 0; w < kNodeThreads / 64; ++w) {
        if (w < wave) before += wave_count[w];
        m += wave_count[w];
    }
    if (is_child) child[before + __popcll(here & ((1ull << lane) - 1ull))] = tid;
    __syncthreads();
    int32_t *out = a.choice + r0 + node;
    if (m == 0) {
        if (tid == 0) *out = -1;
        return;
    }
    const float *p = a.p + (size_t)(r0 + node) * a.p_stride, *q = a.q ? a.q + (size_t)(r0 + node) * a.q_stride : nullptr;
    // everything that the tests take, of all children at once: two round trips to memory here in place of two a test
    if (tid < m) {
        const int x = a.tokens[r0 + child[tid]];
        word[tid] = a.accept_words[r0 + child[tid]];
        token[tid] = known(a, x) ? x : -1;
        token_p[tid] = known(a, x) ? target(p[x]) : 0.0f;
        token_q[tid] = known(a, x) && q ? q[x] : 1.0f;
    }
    parent[tid] = tid < n && mine >= 0 && mine < tid ? mine : -1;
    first[tid] = kMaxNodes;
    __syncthreads();
    const bool first_fits = token[0] >= 0 && accepts(word[0], (double)token_q[0], 1.0, (double)token_p[0]);
    if (first_fits || m == 1) {
        if (tid == 0) *out = first_fits ? child[0] : -1;
        return;
    }
    // Is the node ruled out: on the way up, a first child that is rejected, or another one whose first sibling is accepted
    if (tid < n && parent[tid] >= 0) atomicMin(&first[parent[tid]], tid);
    __syncthreads();
    if (tid == 0) flag = 0;
    int at = node, up = 0;               // every thread climbs; thread t tests step t of the way
    while (parent[at] >= 0 && up < tid) { at = parent[at]; ++up; }
    __syncthreads();
    if (up == tid && parent[at] >= 0) {
        const int above = parent[at];
        if (first_accepted(a, r0, above, first[above]) != (first[above] == at)) flag = 1;
    } 
    __syncthreads();
    if (flag) {
        if (tid == 0) *out = -1;
        return;
    }
    if (tid == 0) mass[0] = 1.0;
    if (!q && tid < m) {                 // has a sibling before this one the same token
        bool again = false;
        for (int j = 0; j < tid && !again; ++j) again = token[j] == token[tid];
        repeat[tid] = again;
    }
    int accepted = -1;
    uint64_t total = 0;                  // sum of the weights of rho_k
    for (int k = 1; k < m; ++k) {
        if (q || k == 1) {
            __syncthreads();
            total = block_sum<kNodeThreads / 64>((uint64_t)row_mass(a, p, q, mass, q ? k : 0), scratch);
        }
        // Without q it is the sum for p less the rejected tokens, each of which is taken off once, when it is rejected.  (All of them anew for every child is a
        // number of steps that grows with the cube of the children: 1023 of them took 9.2 s.)
        if (!q && token[k - 1] >= 0 && !repeat[k - 1]) total -= (uint64_t)weight((double)token_p[k - 1]);
        const double s = (double)total * 0x1p-44;
        if (q) {
            if (tid == 0) {
                mass[k] = s;
                a.mass[r0 + child[k - 1]] = s;
            }
            __syncthreads();
        }
        if (token[k] < 0) continue;
        const double rho = q ? residual(token_p[k], token_q[k], mass, k) : repeat[k] ? 0.0 : (double)token_p[k];
        if (accepts(word[k], (double)token_q[k], s, rho)) { accepted = child[k]; break; }
    }
    if (tid == 0) *out = accepted;
}

// rho of an id after m rejections: of drawn children by their masses, of chosen ones by their tokens
SJD_D double last_rho(int v, float p, float q, bool drawn, const double *mass, const int *token, int m) {
    if (drawn && m) return residual(p, q, mass, m);
    double r = (double)target(p);
    for (int k = 0; k < m && !drawn; ++k) if (token[k] == v) r = 0.0;
    return r;
}

// Workgroup = slice of the last accepted node's rows: walks the path (slice 0 writes it) and sums the slice's weights.  (The draw is a launch of its
// own: done by the last of a sequence's slices behind a device-wide fence it took 23.8 us in place of 17.9 for 16 sequences.)
__global__ __launch_bounds__(256) void verify_walk_kernel(VerifyArgs a) {
    const int b = blockIdx.y, slice = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int r0, n;
    tree_rows(a, b, r0, n);
    __shared__ int choice[kMaxNodes], parent[kMaxNodes], child[kMaxNodes], way, way_len, wave_count[4];
    __shared__ double mass[kMaxNodes];
    __shared__ uint64_t scratch[4];
    for (int i = tid; i < n; i += 256) {
        choice[i] = a.choice[r0 + i];
        parent[i] = a.parents[r0 + i];
    }
    if (slice == 0) for (int i = tid; i < a.max_path; i += 256) a.path[(size_t)b * a.max_path + i] = -1;
    __syncthreads();
    if (tid == 0) {
        int at = n > 0 ? 0 : -1, len = n > 0 ? 1 : 0;
        if (slice == 0 && len) a.path[(size_t)b * a.max_path] = 0;
        while (at >= 0 && len < a.max_path) {
            const int next = tree_step(choice[at], at, n);
            if (next < 0) break;
            at = next;
            if (slice == 0) a.path[(size_t)b * a.max_path + len] = at;
            ++len;
        }
        way = at;
        way_len = len;
        if (slice == 0) a.path_len[b] = len;
    }
    __syncthreads();
    const int at = way;
    // its rejected children: all of them, but none of the last node that the path has room for, whose children do not count: a draw that took its
    // residual where they are rejected, and its p where one is accepted, would not be the target's
    int m = 0;
    if (at >= 0 && way_len < a.max_path)
        for (int j0 = at + 1; j0 < n; j0 += 256) {
            const int j = j0 + tid;
            const bool is_child = j < n && parent[j] == at;
            const unsigned long long here = __ballot(is_child);
            if (lane == 0) wave_count[wave] = __popcll(here);
            __syncthreads();
            int before = m;
            for (int w = 0; w < 4; ++w) {
                if (w < wave) before += wave_count[w];
                m += wave_count[w];
            }
            if (is_child) child[before + __popcll(here & ((1ull << lane) - 1ull))] = j;
            __syncthreads();
        }
    for (int k = tid; k < m; k += 256) mass[k] = k && a.q ? a.mass[r0 + child[k - 1]] : 1.0;
    __syncthreads();
    for (int k = tid; k < m; k += 256) {
        child[k] = a.tokens[r0 + child[k]];     // from here on: their tokens
        if (slice == 0) {
            a.stop_mass[r0 + k] = mass[k];
            a.stop_token[r0 + k] = child[k];
        }
    }
    if (slice == 0 && tid == 0) { a.stop[2 * b] = at >= 0 ? r0 + at : -1; a.stop[2 * b + 1] = m; }
    if (at < 0) return;
    __syncthreads();
    const float *p = a.p + (size_t)(r0 + at) * a.p_stride, *q = a.q ? a.q + (size_t)(r0 + at) * a.q_stride : nullptr;
    const int lo = slice * kSlice, hi = min(lo + kSlice, a.V);
    double sum = 0.0, plain = 0.0;              // of integers, 8 of up to 2^44 a thread: exact
    for_row<256, kSlice / 1024>(a, p, q, lo, hi, [&](int v, float pv, float qv) {
        plain += weight((double)target(pv));
        sum += weight(last_rho(v, pv, qv, q != nullptr, mass, child, m));
    });
    const uint64_t total = block_sum<4>((uint64_t)sum, scratch), total_plain = block_sum<4>((uint64_t)plain, scratch);
    if (tid == 0) {
        uint64_t *part = a.part + ((size_t)b * a.n_slices + slice) * 2;
        part[0] = total;
        part[1] = total_plain;
    }
}

// Workgroup = sequence: the next token
__global__ __launch_bounds__(256) void verify_draw_kernel(VerifyArgs a) {
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // n_slices <= 256: a thread per slice (asked for along with the row; of a sequence without rows it is not looked at)
    const uint64_t *part = a.part + (size_t)b * a.n_slices * 2;
    uint64_t mine = tid < a.n_slices ? part[2 * tid] : 0;
    const uint64_t mine_plain = tid < a.n_slices ? part[2 * tid + 1] : 0, word = a.draw_words[b];
    const int row = a.stop[2 * b];
    int m = a.stop[2 * b + 1], r0, n;
    tree_rows(a, b, r0, n);
    if (row < 0) {
        if (tid == 0) a.next_token[b] = -1;
        return;
    }
    __shared__ uint64_t scratch[4], start;
    __shared__ int found;
    uint64_t Z = block_sum<4>(mine, scratch);
    if (Z == 0) {                                   // nothing is left: from p
        m = 0;
        mine = mine_plain;
        Z = block_sum<4>(mine, scratch);
    }
    if (Z == 0) {
        if (tid == 0) a.next_token[b] = -1;
        return;
    }
    const uint64_t t = __umul64hi(word, Z);
    if (tid == 0) a.next_token[b] = -1;             // (stays where sequences that share rows have left each other's rejections here)
    auto upto = [&](uint64_t v) {                   // inclusive prefix sum over the workgroup
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t l = __shfl_up((uint32_t)v, d, 64), h = __shfl_up((uint32_t)(v >> 32), d, 64);
            if (lane >= d) v += (uint64_t)h << 32 | l;
        }
        __syncthreads();
        if (lane == 63) scratch[wave] = v;
        __syncthreads();
        for (int w = 0; w < wave; ++w) v += scratch[w];
        return v;
    };
    const uint64_t s = upto(mine);
    if (s > t && s - mine <= t) { found = tid; start = s - mine; }
    __syncthreads();
    // within the slice: a thread owns 8 consecutive ids
    constexpr int PER = kSlice / 256;
    const int v0 = found * kSlice + tid * PER;
    const float *p = a.p + (size_t)row * a.p_stride, *q = a.q ? a.q + (size_t)row * a.q_stride : nullptr;
    float pv[PER], qv[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        pv[e] = v0 + e < a.V ? p[v0 + e] : 0.0f;
        qv[e] = v0 + e < a.V && q ? q[v0 + e] : 0.0f;
    }
    uint64_t w[PER], own = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        w[e] = v0 + e < a.V ? (uint64_t)weight(last_rho(v0 + e, pv[e], qv[e], q != nullptr, a.stop_mass + r0, a.stop_token + r0, m)) : 0;
        own += w[e];
    }
    uint64_t c = start + upto(own) - own;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        if (c <= t && c + w[e] > t) a.next_token[b] = v0 + e;
        c += w[e];
    }
}

#define VERIFY_FAIL(code, ...)                          \
    do {                                                \
        sjd_set_error(sjd_call_error(), __VA_ARGS__);   \
        return code;                                    \
    } while (0)
#define VERIFY_TRY(expr) SJD_HIP_TRY(sjd_call_error(), expr)

int check_sizes(int32_t n_rows, int32_t n_seqs, int32_t vocab) {
    if (n_rows < 0 || n_rows > 1 << 29 || n_seqs < 1 || n_seqs > 65535) VERIFY_FAIL(SJD_EINVAL, "n_rows must be 0 .. 2^29, n_seqs 1 .. 65535");
    if (vocab < 1 || vocab > kMaxVocab) VERIFY_FAIL(SJD_EINVAL, "vocab must be 1 .. %d", kMaxVocab);
    return SJD_OK;
}
size_t up16(size_t b) { return (b + 15) / 16 * 16; }
// parts of the workspace
size_t workspace(VerifyArgs &a, char *base) {
    size_t at = 0;
    auto take = [&](size_t bytes) { char *p = base ? base + at : nullptr; at += up16(bytes); return (void *)p; };
    a.mass = (double *)take((size_t)a.n_rows * 8);
    a.stop_mass = (double *)take((size_t)a.n_rows * 8);
    a.part = (uint64_t *)take((size_t)a.n_seqs * a.n_slices * 16);
    a.choice = (int32_t *)take((size_t)a.n_rows * 4);
    a.stop_token = (int32_t *)take((size_t)a.n_rows * 4);
    a.stop = (int32_t *)take((size_t)a.n_seqs * 8);
    return at;
}

}  // namespace

extern "C" {

int sjd_op_tree_verify_workspace(int32_t n_rows, int32_t n_seqs, int32_t vocab, uint64_t *bytes) {
    const int rc = check_sizes(n_rows, n_seqs, vocab);
    if (rc) return rc;
    if (!bytes) VERIFY_FAIL(SJD_EINVAL, "null argument");
    VerifyArgs a = {};
    a.n_rows = n_rows;
    a.n_seqs = n_seqs;
    a.n_slices = ceil_div(vocab, kSlice);
    *bytes = workspace(a, nullptr);
    return SJD_OK;
}

int sjd_op_tree_verify(void *hip_stream, const int32_t *tokens, const int32_t *parents, const int32_t *row_start, const float *p, int64_t p_stride,
                       const float *q, int64_t q_stride, const uint32_t *accept_words, const uint64_t *draw_words, int32_t *path,
                       int32_t *path_len, int32_t *next_token, int32_t n_rows, int32_t n_seqs, int32_t vocab, int32_t max_rows,
                       int32_t max_path, void *ws, uint64_t workspace_bytes) {
    const int rc = check_sizes(n_rows, n_seqs, vocab);
    if (rc) return rc;
    if (max_rows < 1 || max_rows > kMaxNodes) VERIFY_FAIL(SJD_EINVAL, "max_rows must be 1 .. %d", kMaxNodes);
    if (max_path < 1) VERIFY_FAIL(SJD_EINVAL, "max_path must be positive");
    if (!row_start || !draw_words || !path || !path_len || !next_token || (n_rows && (!tokens || !parents || !p || !accept_words)))
        VERIFY_FAIL(SJD_EINVAL, "null argument");
    if (((uintptr_t)tokens | (uintptr_t)parents | (uintptr_t)row_start | (uintptr_t)p | (uintptr_t)q | (uintptr_t)accept_words | (uintptr_t)path |
         (uintptr_t)path_len | (uintptr_t)next_token) % 4 || (uintptr_t)draw_words % 8) VERIFY_FAIL(SJD_EINVAL, "an array is not aligned to its elements");
    VerifyArgs a = {};
    a.tokens = tokens; a.parents = parents; a.row_start = row_start;
    a.p = p; a.q = q; a.p_stride = (long)p_stride; a.q_stride = (long)q_stride;
    a.accept_words = accept_words; a.draw_words = draw_words;
    a.path = path; a.path_len = path_len; a.next_token = next_token;
    a.n_rows = n_rows; a.n_seqs = n_seqs; a.max_rows = max_rows; a.max_path = max_path; a.V = vocab;
    a.n_slices = ceil_div(vocab, kSlice);
    a.wide = (uintptr_t)p % 16 == 0 && p_stride % 4 == 0 && (uintptr_t)q % 16 == 0 && q_stride % 4 == 0;
    const size_t need = workspace(a, (char *)ws);
    if (need > workspace_bytes) VERIFY_FAIL(SJD_ECAPACITY, "the workspace holds %llu bytes, %zu are needed", (unsigned long long)workspace_bytes, need);
    if (!ws || (uintptr_t)ws % 16) VERIFY_FAIL(SJD_EINVAL, "the workspace must be 16-byte aligned");
    hipStream_t st = (hipStream_t)hip_stream;
    if (n_rows) verify_nodes_kernel<<<dim3(max_rows < n_rows ? max_rows : n_rows, n_seqs), kNodeThreads, 0, st>>>(a);
    VERIFY_TRY(hipGetLastError());
    verify_walk_kernel<<<dim3(a.n_slices, n_seqs), 256, 0, st>>>(a);
    VERIFY_TRY(hipGetLastError());
    verify_draw_kernel<<<n_seqs, 256, 0, st>>>(a);
    VERIFY_TRY(hipGetLastError());
    return SJD_OK;
}

}  // extern "C"
