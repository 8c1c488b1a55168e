// Log probabilities of given tokens, with the token's rank, the row's entropy and its likeliest ids, in one pass over the logits.
//
// Of a row z with a reference m near its maximum:  s = sum 2^(L (z - m)), t = sum 2^(L (z - m)) L (z - m), L = log2 e:
//   log p = z_token - m - ln s,   entropy = ln s - ln 2 t / s.
// Lanes have a reference of their own, and join at the end.  Until then exponents are L z - c, one instruction, with c = L m rounded once: the same factor 2^(L m - c) in
// every term of a lane, which its end takes off again.  From magnitudes of 2^22 on, where that factor is anything, they are L (z - m).
//
// The n likeliest ids: a wavefront goes through its part of the row in the order of the ids, 64 lanes x 16 elements at a time, and collects, in LDS, what may still be
// among them: what is not below a threshold.  The n-th largest of the 64 lanes' maxima of a step is one, since n elements reach it; from the next step on only what is larger counts,
// as equal ones have larger ids.  At most one step's elements come at a time, so that a buffer of them and 64 more always holds them, after a selection of the n best.
//
// What bounds it: without ids memory, and the vector units behind it, an exponential and four to five other instructions an element (bf16, 4 099 rows of 65 536: 99 us, 5.4 TB/s; vector units busy for
// 75 % of the cycles).  With ids, what is collected: short rows are few steps, the first of which collects the most (fp32, 256 rows of 65 536, 20 ids: 25.8 + 4.2 us for the joining
// launch, 2.3 TB/s; vector units 43 %, the rest waits; of a row four workgroups have a part each).  Few rows: latency (8 of 16 384, 5 ids: 13.8 us; bf16, 33 rows of 184 621 of which 32 770 ids may be
// taken, 20 ids: 15.8 + 4.8 us).
// Tried, and not here: four steps' loads at a time (registers: 37 against 30 us for the 256 rows), thresholds from every lane's largest element so far in every step (the same there, 33 masked rows 23
// against 20 us), a second round of workgroups that only ranks.
#pragma once
#include "common.hip.h"
#include "kernels_cache.hip.h"
#include "lanes.hip.h"

constexpr int kTopMax = 64;                        // likeliest ids at most: a lane's each
constexpr int kLogprobStep = 1024;                 // elements a wavefront takes at a time
constexpr int kLogprobBuffer = kLogprobStep + kTopMax;
constexpr int kLogprobWaves = 4;
constexpr int kLogprobSift = 256;                  // so many are collected before they are sifted, which makes what follows rarer

struct LogprobArgs {
    const void *z;             // [n_rows][vocab], rows a stride apart
    long stride;
    const int32_t *tokens;
    int n_rows, vocab, n_top, n_splits;
    float *logprob, *entropy, *top_logprob;        // [n_rows], [n_rows], [n_rows][n_top]
    int32_t *rank, *top_id;                        // [n_rows], [n_rows][n_top]
    unsigned char *parts;                          // [n_rows][n_splits] of logprob_part_bytes
};

// What a part of a row comes to
struct LogprobSum { float m, s, t; int rank; };
constexpr size_t logprob_part_bytes(int n_top) { return 16 + 8 * (size_t)n_top; }    // LogprobSum, keys (0: none)

// Order of (z, id): larger z first, then the lower id.  0 is below all.
SJD_D uint32_t logprob_order(float z) {
    const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.0f);          // (-0 is 0)
    return u >> 31 ? ~u : u | 0x80000000u;
}
SJD_D float logprob_unorder(uint32_t o) { return __builtin_bit_cast(float, o >> 31 ? o & 0x7FFFFFFFu : ~o); }
SJD_D uint64_t logprob_key(float z, int id) { return (uint64_t)logprob_order(z) << 32 | (uint32_t)~id; }
SJD_D int logprob_key_id(uint64_t key) { return (int)~(uint32_t)key; }
SJD_D float logprob_key_z(uint64_t key) { return logprob_unorder((uint32_t)(key >> 32)); }
// the least float above x (x < inf)
SJD_D float logprob_above(float x) { return logprob_unorder(logprob_order(x) + 1u); }

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kLogprobFar = 0x1p22f, kLogprobSlack = 8.0f;

// The same about another reference, that is not below
SJD_D void logprob_move(LogprobSum &a, float m) {
    const float d = (a.m - m) * kLog2e, f = __builtin_amdgcn_exp2f(d);
    // (an empty part has s = 0 and a reference of -inf; NaN stays)
    a.t = a.s == 0.0f || f == 0.0f ? 0.0f : fmaf(a.s, d, a.t) * f;
    a.s = a.s == 0.0f ? 0.0f : a.s * f;
    a.m = m;
}
SJD_D LogprobSum logprob_join(LogprobSum a, LogprobSum b) {
    const float m = fmaxf(a.m, b.m);
    logprob_move(a, m);
    logprob_move(b, m);
    return LogprobSum{m, a.s + b.s, a.t + b.t, a.rank + b.rank};
}
// of all lanes; the ranks are left as they are
SJD_D LogprobSum logprob_join_lanes(LogprobSum a) {
    logprob_move(a, lanes_max<64>(a.m));
    a.s = lanes_sum<64>(a.s);
    a.t = lanes_sum<64>(a.t);
    return a;
}

// n-th largest of the lanes' x: the largest float that n lanes reach; kLowest if fewer than n are above -inf
SJD_D float logprob_lane_threshold(float x, int n) {
    const uint32_t o = logprob_order(x);
    uint32_t t = 0u;
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t u = t | 1u << bit;
        const int count = __popcll(__ballot(o >= u));
        if (count >= n) t = u;
        if (count == n) break;
    }
    return fmaxf(logprob_unorder(t), kLowest);
}

// Keeps the n largest of `count` keys, in the order in which they are, and says the least of them.  A wavefront's own buffer; the keys are distinct.  get(i): key i, 0 behind the last;
// GROUPS of 64 of them are looked at (0: as many as there are).
template <int GROUPS, typename Get> SJD_D int logprob_sift(uint64_t *keys, int count, int n, int lane, Get get, uint64_t &least) {
    const int groups = GROUPS ? GROUPS : (count + 63) >> 6;
    auto reach = [&](auto good) {       // how many keys are good
        int c = 0;
        if constexpr (GROUPS > 0) {
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) c += __popcll(__ballot(good(get(i))));
        } else {
#pragma unroll 1
            for (int i = 0; i < groups; ++i) c += __popcll(__ballot(good(get(i))));
        }
        return c;
    };
    uint32_t hi = 0u, lo = 0u;
    bool exact = false;
#pragma unroll 1
    for (int bit = 31; bit >= 0 && !exact; --bit) {
        const uint32_t u = hi | 1u << bit;
        const int c = reach([&](uint64_t k) { return (uint32_t)(k >> 32) >= u; });
        if (c >= n) hi = u;
        exact = c == n;
    }
    if (!exact) {                       // equal logits at the border: the lower ids, whose low halves are larger
        const int need = n - reach([&](uint64_t k) { return (uint32_t)(k >> 32) > hi; });
#pragma unroll 1
        for (int bit = 31; bit >= 0 && !exact; --bit) {
            const uint32_t u = lo | 1u << bit;
            const int c = reach([&](uint64_t k) { return (uint32_t)(k >> 32) == hi && (uint32_t)k >= u; });
            if (c >= need) lo = u;
            exact = c == need;
        }
    }
    least = (uint64_t)hi << 32 | lo;
    int kept = 0;
    auto keep = [&](uint64_t k) {
        const bool takes = k >= least;
        const uint64_t all = __ballot(takes);
        if (takes) keys[kept + __popcll(all & ((1ull << lane) - 1))] = k;     // (at or before its place)
        kept += __popcll(all);
    };
    if constexpr (GROUPS > 0) {
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) keep(get(i));
    } else {
#pragma unroll 1
        for (int i = 0; i < groups; ++i) keep(get(i));
    }
    return kept;
}
SJD_D int logprob_select(uint64_t *keys, int count, int n, int lane, uint64_t &least) {
    constexpr int G = kLogprobSift / 64;
    if (count <= kLogprobSift) {        // in registers
        uint64_t k[G];
#pragma unroll
        for (int i = 0; i < G; ++i) k[i] = 64 * i + lane < count ? keys[64 * i + lane] : 0;
        return logprob_sift<G>(keys, count, n, lane, [&](int i) { return k[i]; }, least);
    }
    return logprob_sift<0>(keys, count, n, lane, [&](int i) { return 64 * i + lane < count ? keys[64 * i + lane] : 0; }, least);
}

// A row's results from its sum and its `n` best keys; key(i): the i-th, 0 where there are fewer
template <typename Key> SJD_D void logprob_finish(const LogprobArgs &a, size_t row, const LogprobSum &r, float z_token, Key key, int first, int step) {
    // NaN and +inf among the logits make s NaN
    const bool bad = r.s != r.s;
    const float log2_s = __builtin_amdgcn_logf(r.s), ln_s = kLn2 * log2_s;
    // (s may have been rounded below the term of the row's only likely id: no logarithm of a probability is above 0)
    auto of = [&](float z) { return bad ? __builtin_nanf("") : z == -INFINITY ? -INFINITY : fminf((z - r.m) - ln_s, 0.0f); };
    if (first == 0) {
        a.logprob[row] = of(z_token);
        a.rank[row] = r.rank;
        a.entropy[row] = bad ? r.s : r.s == 0.0f ? 0.0f : fmaxf(kLn2 * (log2_s - r.t / r.s), 0.0f);
    }
    for (int i = first; i < a.n_top; i += step) {
        const uint64_t k = bad ? 0 : key(i);
        a.top_id[row * a.n_top + i] = k ? logprob_key_id(k) : -1;
        a.top_logprob[row * a.n_top + i] = k ? of(logprob_key_z(k)) : bad ? __builtin_nanf("") : -INFINITY;
    }
}

// The larger of two or three; one that is NaN is left out, or (a signaling one) makes it NaN.  (fmaxf would first make sure, element by element, that none is a signaling NaN.)
SJD_D float logprob_max(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
SJD_D float logprob_max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// One step: 16 elements of every lane.  id(e): of a lane's element e; `live`: bit e is set where there is one.  TOP: candidates are collected.
// WHERE: all ids are before the token (-1), behind it (1), or anything (0).
// The state of a lane: exponents are L (z - o) - c; of a wavefront: rank, keys collected, threshold, whether any o is not 0.
struct LogprobState {
    float m, o, c, s, t;
    int rank, count;
    float least;
    bool far;
    SJD_D LogprobSum sum() const {
        const float rho = o == 0.0f && m > -INFINITY ? fmaf(m, kLog2e, -c) : 0.0f, f = __builtin_amdgcn_exp2f(-rho);
        return LogprobSum{m, s * f, (t - rho * s) * f, 0};
    }
};
template <bool TOP, int WHERE, typename Id>
SJD_D void logprob_step(LogprobState &st, const float (&z)[16], Id id, uint32_t live, float z_token, int token, int n_top, uint64_t *keys, int lane) {
    float top = logprob_max(z[0], z[1]);
#pragma unroll
    for (int e = 2; e < 16; e += 2) top = logprob_max3(top, z[e], z[e + 1]);
    // The reference is the largest logit of a lane, but for 8: it moves where it is exceeded by more (exponentials of up to 2^11.6 cost the sums
    // nothing; the logarithm of one id that has nearly all the weight, a difference of two numbers of up to 8 then, is up to 1e-6 off).
    if (__ballot(top > st.m + kLogprobSlack)) {
        const float m = top > st.m + kLogprobSlack ? top : st.m;
        const bool far = fabsf(m) >= kLogprobFar && m > -INFINITY;
        const float o = far ? m : 0.0f, c = far || m == -INFINITY ? 0.0f : m * kLog2e;
        const float d = fmaf(st.o - o, kLog2e, st.c - c), f = __builtin_amdgcn_exp2f(d);
        // (as long as there was nothing f is anything; NaN stays)
        st.t = st.s == 0.0f || f == 0.0f ? 0.0f : fmaf(st.s, d, st.t) * f;
        st.s = st.s == 0.0f ? 0.0f : st.s * f;
        st.m = m; st.o = o; st.c = c;
        st.far = __ballot(far);
    }
    float x[16];
    if (st.far) {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = fmaf(z[e] - st.o, kLog2e, -st.c);
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = fmaf(z[e], kLog2e, -st.c);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(x[e]);
        st.s += p;
        st.t = fmaf(p, logprob_max(x[e], -300.0f), st.t);       // (p of -inf is 0)
        if (WHERE < 0) st.rank += __popcll(__ballot(z[e] >= z_token));
        else if (WHERE > 0) st.rank += __popcll(__ballot(z[e] > z_token));
        else st.rank += __popcll(__ballot((live >> e & 1u) && (z[e] > z_token || (z[e] == z_token && id(e) < token))));
    }
    if constexpr (TOP) {
        if (!__ballot(top >= st.least)) return;
        auto number = [&]() {
            int n = 0;
#pragma unroll
            for (int e = 0; e < 16; ++e) n += __popcll(__ballot(z[e] >= st.least));
            return n;
        };
        int n = number();
        if (n > 2 * n_top) {
            const float t = logprob_lane_threshold(top, n_top);
            if (t > st.least) {
                st.least = t;
                n = number();
            }
        }
        if (st.count + n > kLogprobSift && st.count > n_top) {
            uint64_t worst;
            st.count = logprob_select(keys, st.count, n_top, lane, worst);
            // (n_top keys with lower ids reach it: what comes has to be larger.  This step's own threshold, if that is higher, takes equal ones)
            const float above = logprob_above(logprob_key_z(worst));
            if (above > st.least) {
                st.least = above;
                n = number();
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint64_t takes = __ballot(z[e] >= st.least);
            if (!takes) continue;
            const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(takes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)takes, 0u));
            if (z[e] >= st.least) keys[st.count + before] = logprob_key(z[e], id(e));
            st.count += __popcll(takes);
        }
        if (n >= n_top) st.least = logprob_above(st.least);
    }
}

// Workgroup = a part of a row, a quarter of it a wavefront.  Rows begin with the elements ahead of the first 16-byte boundary and end with those behind the last.
template <typename T, bool TOP>
__global__ __launch_bounds__(kLogprobWaves * 64) void logprob_kernel(LogprobArgs a) {
    constexpr int VE = 16 / sizeof(T), VECS = 16 / VE;                 // elements of a vector, vectors of a lane's step
    __shared__ uint64_t buffer[TOP ? kLogprobWaves : 1][TOP ? kLogprobBuffer : 1];
    __shared__ LogprobSum sums[kLogprobWaves];
    __shared__ int counts[kLogprobWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t row = blockIdx.x / a.n_splits;
    const int split = blockIdx.x % a.n_splits, V = a.vocab;
    const T *z = (const T *)a.z + row * a.stride;
    const int head = min((int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T), V), vecs = (V - head) / VE, tail = head + vecs * VE;
    const int parts = a.n_splits * kLogprobWaves, part = split * kLogprobWaves + wave;
    const int v0 = (int)((long)vecs * part / parts), v1 = (int)((long)vecs * (part + 1) / parts);
    uint64_t *keys = buffer[TOP ? wave : 0];
    const u32x4 *p = reinterpret_cast<const u32x4 *>(z + head);
    u32x4 next[VECS] = {};
    auto fetch = [&](int v) {
#pragma unroll
        for (int i = 0; i < VECS; ++i)
            if (v + 64 * i + lane < v1) next[i] = p[v + 64 * i + lane];
    };
    const int token = a.tokens[row];
    fetch(v0);                          // (on its way beside the token's logit)
    const bool known = token >= 0 && token < V;
    const float z_token = known ? to_float<T>(z[token]) : __builtin_nanf("");
    LogprobState st = {-INFINITY, 0.0f, 0.0f, 0.0f, 0.0f, 0, 0, kLowest, false};
    auto single = [&](int first, int end) {                            // at most 15 elements
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = -INFINITY;
        const bool there = first + lane < end;
        if (there) x[0] = to_float<T>(z[first + lane]);
        logprob_step<TOP, 0>(st, x, [&](int) { return first + lane; }, there ? 1u : 0u, z_token, token, a.n_top, keys, lane);
    };
    if (part == 0 && head) single(0, head);
    for (int v = v0; v < v1; v += 64 * VECS) {
        float x[16];
#pragma unroll
        for (int i = 0; i < VECS; ++i)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const uint32_t w = next[i][e * sizeof(T) / 4];
                x[i * VE + e] = sizeof(T) == 4 ? __builtin_bit_cast(float, w) : __builtin_bit_cast(float, e & 1 ? w & 0xFFFF0000u : w << 16);
            }
        const bool whole = v + 64 * VECS <= v1;
        uint32_t live = 0xFFFFu;
        if (!whole) {
            live = 0u;
#pragma unroll
            for (int i = 0; i < VECS; ++i) {
                const bool there = v + 64 * i + lane < v1;
                live |= there ? ((1u << VE) - 1u) << (VE * i) : 0u;
#pragma unroll
                for (int e = 0; e < VE; ++e) x[i * VE + e] = there ? x[i * VE + e] : -INFINITY;
            }
        }
        fetch(v + 64 * VECS);
        auto id = [&](int e) { return head + (v + 64 * (e / VE) + lane) * VE + e % VE; };
        const int id0 = head + v * VE, id1 = head + (v + 64 * VECS) * VE;
        if (whole && id1 <= token) logprob_step<TOP, -1>(st, x, id, live, z_token, token, a.n_top, keys, lane);
        else if (whole && id0 > token) logprob_step<TOP, 1>(st, x, id, live, z_token, token, a.n_top, keys, lane);
        else logprob_step<TOP, 0>(st, x, id, live, z_token, token, a.n_top, keys, lane);
    }
    if (part == parts - 1 && tail < V) single(tail, V);

    // the wavefront's, then the workgroup's
    LogprobSum r = logprob_join_lanes(st.sum());
    r.rank = st.rank;
    if constexpr (TOP)
        if (st.count > 64) {            // a lane's key each
            uint64_t worst;
            st.count = logprob_select(keys, st.count, a.n_top, lane, worst);
        }
    if (lane == 0) {
        sums[wave] = r;
        counts[wave] = st.count;
    }
    __syncthreads();
    r = sums[0];
#pragma unroll
    for (int w = 1; w < kLogprobWaves; ++w) r = logprob_join(r, sums[w]);
    // a key's place among the four buffers' is the number of larger ones
    uint64_t mine = 0;
    int place = 0;
    if constexpr (TOP) {
        if (lane < st.count) mine = keys[lane];
#pragma unroll
        for (int w = 0; w < kLogprobWaves; ++w)
#pragma unroll 4
            for (int i = 0; i < counts[w]; ++i) place += buffer[w][i] > mine;
        __syncthreads();
        if (threadIdx.x < kTopMax) buffer[0][threadIdx.x] = 0;
        __syncthreads();
        if (mine && place < a.n_top) buffer[0][place] = mine;
        __syncthreads();
    }
    if (!known) r.rank = -1;
    if (a.n_splits == 1) logprob_finish(a, row, r, known ? z_token : -INFINITY, [&](int i) { return buffer[0][TOP ? i : 0]; }, threadIdx.x, kLogprobWaves * 64);
    else {
        unsigned char *out = a.parts + (row * a.n_splits + split) * logprob_part_bytes(a.n_top);
        if (threadIdx.x == 0) *reinterpret_cast<LogprobSum *>(out) = r;
        if (TOP && threadIdx.x < a.n_top) reinterpret_cast<uint64_t *>(out + 16)[threadIdx.x] = buffer[0][threadIdx.x];
    }
}

// Joins the parts of a row.  n_splits * n_top keys are at most kLogprobJoin.
constexpr int kLogprobJoin = 1024;
template <typename T>
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobArgs a) {
    __shared__ uint64_t keys[kLogprobJoin], best[kTopMax];
    __shared__ int some;
    const size_t row = blockIdx.x, bytes = logprob_part_bytes(a.n_top);
    const unsigned char *parts = a.parts + row * a.n_splits * bytes;
    const int tid = threadIdx.x, lane = tid & 63, n = a.n_splits * a.n_top;
    uint64_t mine[kLogprobJoin / 256];
#pragma unroll
    for (int i = 0; i < kLogprobJoin / 256; ++i) {
        const int u = tid + 256 * i;
        mine[i] = u < n ? reinterpret_cast<const uint64_t *>(parts + u / a.n_top * bytes + 16)[u % a.n_top] : 0;
    }
    const int token = a.tokens[row];
    const bool known = token >= 0 && token < a.vocab;
    const float z_token = known ? to_float<T>(((const T *)a.z)[row * a.stride + token]) : -INFINITY;
    // A part's last key is reached by n_top of its own: only what reaches the largest of them can be among the best.
    uint64_t least = 0;
    if (a.n_top)
        for (int i = lane; i < a.n_splits; i += 64) least = max(least, reinterpret_cast<const uint64_t *>(parts + i * bytes + 16)[a.n_top - 1]);
    LogprobSum r = {-INFINITY, 0.0f, 0.0f, 0};
    for (int i = lane; i < a.n_splits; i += 64) r = logprob_join(r, *reinterpret_cast<const LogprobSum *>(parts + i * bytes));
    r = logprob_join_lanes(r);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        r.rank += __shfl_xor(r.rank, d, 64);
        least = max(least, (uint64_t)__shfl_xor((unsigned long long)least, d, 64));
    }
    if (!known) r.rank = -1;
    if (tid < kTopMax) best[tid] = 0;
    if (tid == 0) some = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLogprobJoin / 256; ++i)
        if (mine[i] && mine[i] >= least) keys[atomicAdd(&some, 1)] = mine[i];       // (in any order: a key's place is the number of larger ones)
    __syncthreads();
    for (int i = tid; i < some; i += 256) {
        const uint64_t key = keys[i];
        int place = 0;
#pragma unroll 4
        for (int j = 0; j < some; ++j) place += keys[j] > key;
        if (place < a.n_top) best[place] = key;
    }
    __syncthreads();
    logprob_finish(a, row, r, z_token, [&](int i) { return best[i]; }, tid, 256);
}
