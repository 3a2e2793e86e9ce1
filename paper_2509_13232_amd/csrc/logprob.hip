// Log-probs of given tokens, their entropy and the top alternatives from existing logits, the gradient of all of them, and the
// C entry points of both the logits-in and the head form (whose kernels are the sweeps of pg_fused.hip).
//
//   forward   one pass over the rows keeps (max, sum of exp, sum of x exp) per thread and joins them; for the alternatives
//             every thread also leaves the largest logit it met, and a second kernel finds the K largest of a row from
//             those: the K-th largest of 256 such maxima is a lower bound on the K-th largest logit, and few logits pass it;
//   backward  dz_i = a [i = y] + sum_k b_k [i = id_k] - p_i (a + sum_k b_k + e (log p_i + H)), one read and one write.
#include <algorithm>

#include "logprob.hpp"
#include "row_stream.hpp"
#include "timing.hpp"

namespace spo {

constexpr int kScoreGroup = 4, kScoreRounds = 2, kScoreGradGroup = 2;
constexpr int kScoreNarrow = 5, kScoreGradNarrow = 4;  // see row_grid
constexpr float kLowestFloat = -3.402823466e38f;       // starts a maximum: finite, and no logit but -inf is below it

// What every row carries besides its logits.
struct ScoreRows {
    int64_t T, V, stride;   // stride: elements from row to row
    const int32_t *target;  // NULL: no log-prob
    const uint8_t *mask;    // NULL: every row counts
};
struct ScoreOut {
    float *logp, *lse, *entropy;  // logp, entropy: NULL where not asked for
    int32_t *top_id;
    float *top_logp;
    int K;
};

template <typename T>
__device__ __forceinline__ float target_logit(const T *row, const ScoreRows &r, int64_t t) {
    const int64_t y = r.target[t];  // an id outside [0, V) gives NaN instead of a read out of bounds
    return y >= 0 && y < r.V ? Vec<T>::get(row + y) : __builtin_nanf("");
}

__device__ __forceinline__ void store_scores(const ScoreOut &o, int64_t t, float zt, float m, float s, float u) {
    const float l = logf(s);
    o.lse[t] = m + l;
    if (o.logp) o.logp[t] = (zt - m) - l;  // (beside a logit of 1e8 the sum m + l has lost l)
    if (o.entropy) o.entropy[t] = score_entropy(s, u);
}
// a row that the mask leaves out: nothing of it is read
__device__ __forceinline__ void store_left_out(const ScoreOut &o, int64_t t) {
    o.lse[t] = 0.0f;
    if (o.logp) o.logp[t] = 0.0f;
    if (o.entropy) o.entropy[t] = 0.0f;
}

// The lanes' running values joined, for every lane: one maximum, then one rescaling and the sums.
__device__ __forceinline__ void join_lanes(float &m, float &s, float &u) {
    float top = m;
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
    const float d = fmaxf((m - top) * kLog2e, kLowest2), f = __builtin_amdgcn_exp2f(d);
    u = wave_sum(f * fmaf(d, s, u));
    s = wave_sum(s * f);
    m = top;
}

// (max, sum of 2^x, sum of x 2^x) of one segment of a row by TR threads, a workgroup or one wavefront of it, and with Top each
// thread's own maximum, group_max[row][segment * TR + thread].  Rows of one segment (whole) are finished here unless
// alternatives are asked for.  Bound by HBM in fp32 (535 of 713 rows of 100003, 214 MB in 38.8 us = 5.5 TB/s), in bf16 by
// instructions as well (6554 of 8192 rows of 151936, 1.99 GB in 330 to 393 us = 5.1 to 6.0 TB/s); single rows by latency (4 us).
template <typename T, int TR, int Rounds, bool Stream, bool Top>
__global__ void __launch_bounds__(kRowThreads)
score_rows_kernel(const T *__restrict__ logits, ScoreRows rows, RowGrid grid, float *__restrict__ part, float *__restrict__ group_max,
                  ScoreOut out) {
    constexpr int N = Vec<T>::N, U = kScoreGroup;
    const int64_t unit = group_unit<TR>();
    const int tid = threadIdx.x % TR;
    if (unit >= grid.units()) return;  // TR < kRowThreads only: no barrier below in that case
    const uint32_t nseg = static_cast<uint32_t>(grid.nseg), seg = static_cast<uint32_t>(unit) % nseg;
    const int64_t t = static_cast<uint32_t>(unit) / nseg, e0 = seg * grid.seg_len;
    const bool whole = !Top && nseg == 1;
    if (rows.mask && !rows.mask[t]) {
        if (whole && tid == 0) store_left_out(out, t);
        return;
    }
    const T *row = logits + t * rows.stride, *p = row + e0;
    const Span sp(p, static_cast<int>(rows.V - e0 < grid.seg_len ? rows.V - e0 : grid.seg_len));
    float zt = 0.0f;
    if (whole && tid == 0 && rows.target) zt = target_logit(row, rows, t);
    // the few elements outside the whole vectors, one per thread
    float m = kLowestFloat, s = 0.0f, u2 = 0.0f;
    if (tid < sp.head + sp.tail) {
        const float x = Vec<T>::get(p + (tid < sp.head ? tid : tid + sp.nvec * N));
        m = fmaxf(m, x);
        const float d = fmaxf((x - m) * kLog2e, kLowest2);
        s = __builtin_amdgcn_exp2f((x - m) * kLog2e);
        u2 = s * d;
    }
    const T *body = p + sp.head;
    auto request = [&](uint4 (&v)[U], int i0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * TR < sp.nvec) v[u] = load16<Stream>(body + (i0 + u * TR) * N);
    };
    auto take = [&](const uint4 (&v)[U], int i0) {
        // one new maximum and one rescaling of the running sums for the whole group
        float x[U][N], mx = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * TR >= sp.nvec) break;
            Vec<T>::unpack(v[u], x[u]);
#pragma unroll
            for (int i = 0; i < N; ++i) mx = fmaxf(mx, x[u][i]);
        }
        // What bounds rows of bf16 is this sum: besides the exponential (four operations' time) a logit takes half an operation
        // for the maximum and one each for its value, exponent, sum and weighted sum.  The weighted sum goes without kLowest2:
        // a NaN in it says that there was a logit of -inf (or a NaN), and then it is formed again with it.  (8192 rows of
        // 151936: with kLowest2 for every logit 376 us, without 354.)
        // What rounding -mx log2(e) took off all exponents alike goes back into the sums (rows about 1e4: 3e-4 of them).
        const float nm2 = -mx * kLog2e;
        float a[U] = {}, w[U] = {}, rest = 0.0f;
        auto add = [&](auto exponent, auto bound) {
#pragma unroll
            for (int u = 0; u < U; ++u) a[u] = w[u] = 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u * TR >= sp.nvec) break;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float d = exponent(x[u][i]), e = __builtin_amdgcn_exp2f(d);
                    a[u] += e;
                    w[u] = fmaf(e, bound(d), w[u]);
                }
            }
        };
        const bool far = fabsf(mx) > kFarLogit;
        if (!__any(i0 < sp.nvec && far)) {
            add([&](float v) { return fmaf(v, kLog2e, nm2); }, [](float d) { return d; });
            rest = far ? 0.0f : fmaf(-mx, kLog2e, -nm2);  // (far: a thread without logits)
        }
        const float sum = (w[0] + w[1]) + (w[2] + w[3]);
        if (__any(i0 < sp.nvec && (far || sum != sum))) {
            add([&](float v) { return (v - mx) * kLog2e; }, [](float d) { return fmaxf(d, kLowest2); });
            rest = 0.0f;
        }
        const float d = fmaxf((m - mx) * kLog2e, kLowest2), f = __builtin_amdgcn_exp2f(d), g = __builtin_amdgcn_exp2f(rest);
        const float sa = (a[0] + a[1]) + (a[2] + a[3]), sw = (w[0] + w[1]) + (w[2] + w[3]);
        u2 = f * fmaf(d, s, u2) + g * fmaf(rest, sa, sw);
        s = s * f + g * sa;
        m = mx;
    };
    // a segment is at most Rounds rounds: all of it is requested at once
    static_assert(Rounds <= 2, "two sets of registers");
    uint4 first[U], second[U];
    request(first, tid);
    if constexpr (Rounds > 1) request(second, tid + U * TR);
    take(first, tid);
    if constexpr (Rounds > 1)
        if (U * TR < sp.nvec) take(second, tid + U * TR);
    if constexpr (Top) group_max[(t * nseg + seg) * TR + tid] = m;
    join_lanes(m, s, u2);
    if constexpr (TR > kWave) {
        __shared__ float sm[TR / kWave], ss[TR / kWave], su[TR / kWave];
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) { sm[wave] = m; ss[wave] = s; su[wave] = u2; }
        __syncthreads();
        m = sm[0]; s = ss[0]; u2 = su[0];
        for (int w = 1; w < TR / kWave; ++w) score_join(m, s, u2, sm[w], ss[w], su[w]);
    }
    if (tid != 0) return;
    if (whole) return store_scores(out, t, zt, m, s, u2);
    float *q = part + (t * nseg + seg) * 3;
    q[0] = m;
    q[1] = s;
    q[2] = u2;
}

// The segments of row t joined by one wavefront; every lane receives the result.
__device__ __forceinline__ void join_segments(const float *__restrict__ part, int nseg, int64_t t, float &m, float &s, float &u) {
    const int lane = threadIdx.x & 63;
    m = kLowestFloat;
    s = u = 0.0f;
    for (int i = lane; i < nseg; i += kWave) {
        const float *q = part + (t * nseg + i) * 3;
        score_join(m, s, u, q[0], q[1], q[2]);
    }
    join_lanes(m, s, u);
}

// Rows of several segments finished, a wavefront each (8192 rows: 5.4 us).
template <typename T>
__global__ void __launch_bounds__(256)
score_join_kernel(const T *__restrict__ logits, ScoreRows rows, int nseg, const float *__restrict__ part, ScoreOut out) {
    const int64_t t = flat_block() * 4 + (threadIdx.x >> 6);
    if (t >= rows.T) return;
    const int lane = threadIdx.x & 63;
    if (rows.mask && !rows.mask[t]) {
        if (lane == 0) store_left_out(out, t);
        return;
    }
    float zt = 0.0f, m, s, u;
    if (lane == 0 && rows.target) zt = target_logit(logits + t * rows.stride, rows, t);
    join_segments(part, nseg, t, m, s, u);
    if (lane == 0) store_scores(out, t, zt, m, s, u);
}

// ----------------------------------------------------------------------------
// the K largest logits of a row
// ----------------------------------------------------------------------------
// Order: by value, ties to the lowest id; -0 and +0 tie.  As one whole number, the larger the better: the value's bits made
// monotone, then the id from above.  A NaN has no place in the order (it gets one by its bits).
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t order_of(float x, uint32_t id) { return static_cast<uint64_t>(order_key(x)) << 32 | static_cast<uint32_t>(~id); }

constexpr int kPickThreads = 256;
constexpr int kPickGroups = 512;             // groups of a row that are looked into at a time
constexpr int kPickStep = kPickThreads * 8;  // logits of the step by step way
constexpr int kPickRoom = kPickStep + SPO_MAX_TOP_K;  // a multiple of kRankStep

// Places of cand[0..n) in their order, `put(place, candidate)` for each of the first K.  n <= kPickRoom; keys are distinct.
// Counted kRankStep at a time (a read by itself takes as long as sixteen): the room behind the last candidate is filled up.
constexpr int kRankStep = 8;
template <typename F>
__device__ __forceinline__ void rank_candidates(uint64_t *cand, int n, int K, F put) {
    if (threadIdx.x < kRankStep && n + threadIdx.x < kPickRoom) cand[n + threadIdx.x] = 0;  // behind every logit's number
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPickThreads) {
        const uint64_t mine = cand[i];
        int place = 0;
        for (int j = 0; j < n; j += kRankStep)
#pragma unroll
            for (int k = 0; k < kRankStep; ++k) place += cand[j + k] > mine ? 1 : 0;
        if (place < K) put(place, mine);
    }
}

// A lower bound on the K-th largest of a wavefront's keys that exactly K of them reach, or the K-th largest itself: bit by bit
// from the highest.
__device__ __forceinline__ uint32_t kth_largest(const uint32_t (&key)[kPickThreads / kWave], int K) {
    uint32_t kth = 0;
    int reach = kPickThreads;
    for (uint32_t bit = 0x80000000u; bit && reach != K; bit >>= 1) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < kPickThreads / kWave; ++i) n += __popcll(__ballot(key[i] >= (kth | bit)));
        if (n >= K) {
            kth |= bit;
            reach = n;
        }
    }
    return kth;
}

// One workgroup per row: joins its segments and finds its K largest logits.
//   1. Every thread takes the maximum of its share of group_max; the K-th largest of these 256 maxima of disjoint sets bounds
//      the K-th largest logit from below, and few shares (K, and those that tie) reach it.
//   2. The groups of these shares whose maximum reaches the bound, somewhat more than K, are looked into: a thread per vector.
//   3. What reaches the bound is ranked by counting.
// Bound by latency, of loads and of instructions not yet in a cache (one row of 151936 in bf16 with 20 alternatives: 16.8 us;
// with loads eight at a time, a second look at these shares instead of all groups and one atomic per vector 7.2, with the search
// for the bound ended as soon as K shares reach it 6.3).
// Rows with more ties at the bound than there is room, or with fewer groups than K, are walked step by step from the first
// logit on, with the K best so far kept; later ones have to beat the last of these, so ties cost little after the first step.
template <typename T, int TR>
__global__ void __launch_bounds__(kPickThreads)
score_pick_kernel(const T *__restrict__ logits, ScoreRows rows, RowGrid grid, const float *__restrict__ part,
                  const float *__restrict__ group_max, ScoreOut out) {
    constexpr int N = Vec<T>::N, VPG = kScoreGroup * kScoreRounds;  // vectors of a thread's group, at most
    __shared__ __attribute__((aligned(16))) float best[kPickThreads];
    __shared__ __attribute__((aligned(16))) uint64_t cand[kPickRoom];
    __shared__ uint64_t kept[SPO_MAX_TOP_K];
    __shared__ int groups[kPickGroups], share[kPickThreads];
    __shared__ int n_cand, n_group, n_share;
    __shared__ float bound, row_max, row_log;
    __shared__ uint32_t second;
    const int64_t t = flat_block();
    if (t >= rows.T) return;
    const int tid = threadIdx.x, K = out.K, nseg = grid.nseg;
    if (rows.mask && !rows.mask[t]) {
        if (tid == 0) store_left_out(out, t);
        if (tid < K) {
            out.top_id[t * K + tid] = -1;
            out.top_logp[t * K + tid] = 0.0f;
        }
        return;
    }
    const T *row = logits + t * rows.stride;
    const float *gm = group_max + t * nseg * TR;
    const int G = nseg * TR;
    float mine = -INFINITY;  // share of thread i: groups i, i + 256, ...; eight on their way at a time
    constexpr int U = 8;
    for (int g0 = tid; g0 < G; g0 += U * kPickThreads) {
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = gm[g0 + u * kPickThreads < G ? g0 + u * kPickThreads : g0];
#pragma unroll
        for (int u = 0; u < U; ++u) mine = fmaxf(mine, x[u]);
    }
    best[tid] = mine;
    if (tid == 0) n_cand = n_group = n_share = 0;
    __syncthreads();
    if (tid < kWave) {  // the first wavefront joins the segments meanwhile
        float zt = 0.0f, m, s, u;
        if (tid == 0 && rows.target) zt = target_logit(row, rows, t);
        join_segments(part, nseg, t, m, s, u);
        if (tid == 0) {
            store_scores(out, t, zt, m, s, u);
            row_max = m;
            row_log = logf(s);
        }
    } else if (tid < 2 * kWave) {
        // The K-th largest by the second wavefront (where the bound's bits end in a NaN's, the row is walked step by step).
        // (Every thread counting the larger ones: 1024 wavefront operations per compute unit, 2 us.)
        uint32_t key[kPickThreads / kWave];
#pragma unroll
        for (int i = 0; i < kPickThreads / kWave; ++i) key[i] = order_key(best[i * kWave + tid - kWave]);
        const uint32_t kth = kth_largest(key, K);
        if (tid == kWave) bound = order_value(kth);
    }
    __syncthreads();
    // the start of a maximum says nothing about a group (it may be empty, or all -inf)
    const float tau = bound;
    bool by_step = !(tau > kLowestFloat);
    if (!by_step) {
        if (mine >= tau) share[atomicAdd(&n_share, 1)] = tid;
        __syncthreads();
        const int ns = n_share, items = ns * ((G + kPickThreads - 1) / kPickThreads);
        constexpr int S = 4;  // on their way at a time
        for (int i0 = tid; i0 < items; i0 += S * kPickThreads) {
            float x[S];
            int g[S];
#pragma unroll
            for (int j = 0; j < S; ++j) {
                const int i = i0 + j * kPickThreads;
                g[j] = i < items ? i / ns * kPickThreads + share[i % ns] : G;
                x[j] = gm[g[j] < G ? g[j] : 0];
            }
#pragma unroll
            for (int j = 0; j < S; ++j)
                if (g[j] < G && x[j] >= tau) {
                    const int at = atomicAdd(&n_group, 1);
                    if (at < kPickGroups) groups[at] = g[j];
                }
        }
        __syncthreads();
        const int ng = n_group;
        by_step = ng > kPickGroups;
        if (!by_step) {
            const bool one_round = grid.seg_len <= TR * kScoreGroup * N;  // (groups of half as many vectors)
            for (int i = tid; i < ng * (one_round ? kScoreGroup + 1 : VPG + 1); i += kPickThreads) {
                const int at_g = one_round ? i / (kScoreGroup + 1) : i / (VPG + 1), j = i - at_g * (one_round ? kScoreGroup + 1 : VPG + 1);
                const int g = groups[at_g], v = one_round && j == kScoreGroup ? VPG : j, th = g % TR;
                const int64_t e0 = (g / TR) * grid.seg_len;
                const Span sp(row + e0, static_cast<int>(rows.V - e0 < grid.seg_len ? rows.V - e0 : grid.seg_len));
                float x[N];
                int first, count = 0;  // elements of the segment that x holds
                if (v == VPG) {        // the thread's element outside the whole vectors
                    first = th < sp.head ? th : th + sp.nvec * N;
                    if (th < sp.head + sp.tail) {
                        x[0] = Vec<T>::get(row + e0 + first);
                        count = 1;
                    }
                } else {
                    first = sp.head + (th + v * TR) * N;
                    if (th + v * TR < sp.nvec) {
                        Vec<T>::unpack(load16<false>(row + e0 + first), x);
                        count = N;
                    }
                }
                uint32_t reach = 0;
#pragma unroll
                for (int j = 0; j < N; ++j) reach |= j < count && x[j] >= tau ? 1u << j : 0u;
                if (!reach) continue;
                const int at = atomicAdd(&n_cand, __popc(reach));
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int place = at + __popc(reach & ((1u << j) - 1));
                    if ((reach >> j & 1) && place < kPickRoom) cand[place] = order_of(x[j], static_cast<uint32_t>(e0 + first + j));
                }
            }
            __syncthreads();
            by_step = n_cand > kPickRoom || n_cand < K;  // (fewer than K: NaNs, which reach no bound)
            if (!by_step && n_cand > kPickThreads) {
                // few groups for so many alternatives: ranking all would take longer than a second bound, from the candidates
                constexpr int U = (kPickRoom + kPickThreads - 1) / kPickThreads;
                uint64_t c[U], top = 0;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    c[u] = tid + u * kPickThreads < n_cand ? cand[tid + u * kPickThreads] : 0;
                    top = c[u] > top ? c[u] : top;
                }
                uint32_t *keys = reinterpret_cast<uint32_t *>(best);
                keys[tid] = static_cast<uint32_t>(top >> 32);
                __syncthreads();
                if (tid == 0) n_cand = 0;
                if (tid < kWave) {
                    uint32_t key[kPickThreads / kWave];
#pragma unroll
                    for (int i = 0; i < kPickThreads / kWave; ++i) key[i] = keys[i * kWave + tid];
                    const uint32_t kth = kth_largest(key, K);
                    if (tid == 0) second = kth;
                }
                __syncthreads();
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (c[u] && c[u] >> 32 >= second) cand[atomicAdd(&n_cand, 1)] = c[u];
                __syncthreads();
            }
        }
    }
    auto put = [&](int place, uint64_t c) {
        out.top_id[t * K + place] = static_cast<int32_t>(~static_cast<uint32_t>(c));
        out.top_logp[t * K + place] = (order_value(static_cast<uint32_t>(c >> 32)) - row_max) - row_log;
    };
    if (!by_step) return rank_candidates(cand, n_cand, K, put);
    uint64_t least = 0;  // of the K kept so far; no logit's number is 0
    int n_kept = 0;
    for (int64_t e0 = 0; e0 < rows.V; e0 += kPickStep) {
        __syncthreads();  // kept and cand are no longer read
        if (tid == 0) n_cand = n_kept;
        if (tid < n_kept) cand[tid] = kept[tid];
        __syncthreads();
        for (int j = 0; j < kPickStep / kPickThreads; ++j) {
            const int64_t e = e0 + j * kPickThreads + tid;
            if (e >= rows.V) break;
            const uint64_t c = order_of(Vec<T>::get(row + e), static_cast<uint32_t>(e));
            if (c > least) cand[atomicAdd(&n_cand, 1)] = c;
        }
        __syncthreads();
        const int n = n_cand;
        if (n == n_kept) continue;
        rank_candidates(cand, n, K, [&](int place, uint64_t c) { kept[place] = c; });
        __syncthreads();
        n_kept = n < K ? n : K;
        if (n_kept == K) least = kept[K - 1];
    }
    __syncthreads();
    if (tid < n_kept) put(tid, kept[tid]);
}

// ----------------------------------------------------------------------------
// backward
// ----------------------------------------------------------------------------
struct ScoreGrads {
    const float *lse, *entropy, *d_logp, *d_entropy;  // d_logp, d_entropy: NULL: zeros
    const int32_t *top_id;
    const float *d_top;                               // NULL: zeros
    int K;
};

// The gradient takes log p = z - lse, and what rounding lse to fp32 took off is an error that all of a row's probabilities share: half
// of its last place, 2^-18 up to 128 and 2^-14 up to 2048.  Beyond that it is no longer small (in fp32 beside the other roundings, in
// bf16 beside the output's 2^-8), and the row's own maximum and sum are formed again.
template <typename T> constexpr float kFarLse = sizeof(T) == 4 ? 128.0f : 2048.0f;
template <typename T> constexpr int kFarLoads = 16 / Vec<T>::N;  // on their way per thread
constexpr uint32_t kFarUnits = 512;  // see score_grad_kernel

// (max, log of the sum of exp(x - max)) of a whole row by a group of TR threads, in one pass.
template <typename T, int TR>
__device__ __forceinline__ void row_max_log(const T *row, int64_t V, float &m, float &l) {
    constexpr int N = Vec<T>::N, U = kFarLoads<T>;
    const int tid = threadIdx.x % TR, nvec = static_cast<int>(V / N);
    float s = 0.0f;
    m = kLowestFloat;
    for (int i0 = tid; i0 < nvec; i0 += U * TR) {
        uint4 v[U];
        float x[N], mx = m;
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load16<false>(row + static_cast<int64_t>(i0 + u * TR < nvec ? i0 + u * TR : i0) * N);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Vec<T>::unpack(v[u], x);
#pragma unroll
            for (int i = 0; i < N; ++i) mx = fmaxf(mx, x[i]);
        }
        s *= __builtin_amdgcn_exp2f((m - mx) * kLog2e);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * TR >= nvec) break;
            Vec<T>::unpack(v[u], x);
#pragma unroll
            for (int i = 0; i < N; ++i) s += __builtin_amdgcn_exp2f((x[i] - mx) * kLog2e);
        }
        m = mx;
    }
    if (tid < static_cast<int>(V - static_cast<int64_t>(nvec) * N)) {
        const float x = Vec<T>::get(row + static_cast<int64_t>(nvec) * N + tid), mx = fmaxf(m, x);
        s = s * __builtin_amdgcn_exp2f((m - mx) * kLog2e) + __builtin_amdgcn_exp2f((x - mx) * kLog2e);
        m = mx;
    }
    float top = m;
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
    s = wave_sum(s * __builtin_amdgcn_exp2f((m - top) * kLog2e));
    m = top;
    if constexpr (TR > kWave) {
        __shared__ float wm[TR / kWave], ws[TR / kWave];
        if ((threadIdx.x & 63) == 0) { wm[threadIdx.x >> 6] = m; ws[threadIdx.x >> 6] = s; }
        __syncthreads();
        m = wm[0];
        for (int w = 1; w < TR / kWave; ++w) m = fmaxf(m, wm[w]);
        s = 0.0f;
        for (int w = 0; w < TR / kWave; ++w) s += ws[w] * __builtin_amdgcn_exp2f((wm[w] - m) * kLog2e);
    }
    l = logf(s);
}

// One segment of a row of d_logits (at most kScoreGradGroup vectors per thread).  Rows that the mask leaves out are not read;
// they and rows whose factors are all zero are written as zeros.  Vectors are aligned on the output side.  Bound by HBM: 8192 rows
// of 151936 in bf16, a fifth left out, 4.48 GB in 770 us = 5.8 TB/s; 512 rows of 1000 in fp32 4.6 us.
// Rows far from zero (kFarLse) are read once more for their own maximum and sum, by each of the groups that then write the row, some
// kFarUnits for all rows together (rows of 151936 in fp32: one 18 us, 27 36, 512 239; by one group per row 63, 74, 252, by one per
// segment 18, 64, 1026; other rows 5, 6, 95).
template <typename T, int TR, bool Stream>
__global__ void __launch_bounds__(kRowThreads, 8)
score_grad_kernel(const T *__restrict__ logits, ScoreRows rows, RowGrid grid, ScoreGrads gr, T *__restrict__ d_logits) {
    constexpr int N = Vec<T>::N, U = kScoreGradGroup;
    const int64_t unit = group_unit<TR>();
    const int tid = threadIdx.x % TR, lane = threadIdx.x & 63;
    if (unit >= grid.units()) return;
    const uint32_t nseg = static_cast<uint32_t>(grid.nseg);
    const int64_t t = static_cast<uint32_t>(unit) / nseg;
    uint32_t seg = static_cast<uint32_t>(unit) % nseg;
    const T *row = logits + t * rows.stride;
    T *out_row = d_logits + t * rows.V;
    // a segment: its start and length, its vectors and this thread's element outside of them
    int64_t e0;
    int len;
    Span sp(out_row, 0);
    auto start = [&] {
        e0 = seg * grid.seg_len;
        len = static_cast<int>(rows.V - e0 < grid.seg_len ? rows.V - e0 : grid.seg_len);
        sp = Span(out_row + e0, len);
    };
    auto edge = [&] { return tid < sp.head + sp.tail; };
    auto at_edge = [&] { return tid < sp.head ? tid : tid + sp.nvec * N; };
    auto vectors = [&] { return reinterpret_cast<uint4 *>(out_row + e0 + sp.head); };
    start();
    auto zeros = [&] {
        if (edge()) Vec<T>::put(out_row + e0 + at_edge(), 0.0f);
        for (int i = tid; i < sp.nvec; i += TR) store16<Stream>(vectors() + i, make_uint4(0u, 0u, 0u, 0u));
    };
    if (rows.mask && !rows.mask[t]) return zeros();
    // everything is requested before any of it is looked at
    uint4 v[U];
    T x_edge;
    auto request = [&] {
        const T *body = row + e0 + sp.head;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (tid + u * TR < sp.nvec) v[u] = load16<Stream>(body + (tid + u * TR) * N);
        x_edge = edge() ? row[e0 + at_edge()] : T(0);  // (as it is: a conversion would wait for it here)
    };
    request();
    const float lse = gr.lse[t], a = gr.d_logp ? gr.d_logp[t] : 0.0f, e = gr.d_entropy ? gr.d_entropy[t] : 0.0f;
    const float h = gr.d_entropy ? gr.entropy[t] : 0.0f;
    const int64_t target = gr.d_logp ? static_cast<int64_t>(rows.target[t]) : -1;
    float total = a;
    int64_t top_id = -1;  // lane k: the k-th alternative, and its factor
    float b = 0.0f;
    bool some = false;
    if (gr.d_top) {
        if (lane < gr.K) {
            b = gr.d_top[t * gr.K + lane];
            top_id = gr.top_id[t * gr.K + lane];
        }
        some = __any(b != 0.0f);  // (factors of both signs may add up to zero)
        total += wave_sum(b);
    }
    if (a == 0.0f && e == 0.0f && !some) return zeros();
    float c = -(e != 0.0f ? fmaf(e, h, total) : total), c2 = -e * kLn2;  // dz = p (c + c2 log2 p) + ...
    auto finish = [&](auto exponent) {
        // places in the segment
        const int64_t yl = target - e0, il = top_id - e0;
        const int y = target >= 0 && yl >= 0 && yl < len ? static_cast<int>(yl) : -1;
        const int id = top_id >= 0 && il >= 0 && il < len ? static_cast<int>(il) : -1;
        const uint64_t hot = some ? __ballot(id >= 0 && b != 0.0f) : 0;
        auto grad = [&](float z) {
            const float d = exponent(z);
            return __builtin_amdgcn_exp2f(d) * fmaf(fmaxf(d, kLowest2), c2, c);
        };
        auto of_hot = [&](auto add) {  // add(place, what is added there)
            add(y, a);
            for (uint64_t k = hot; k; k &= k - 1) {
                const int l = __builtin_ctzll(k);
                add(__builtin_amdgcn_readlane(id, l), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(b), l)));
            }
        };
        if (edge()) {
            float g = grad(Vec<T>::get(&x_edge));
            of_hot([&](int place, float w) { g += place == at_edge() ? w : 0.0f; });
            Vec<T>::put(out_row + e0 + at_edge(), g);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int iv = tid + u * TR, first = sp.head + iv * N;
            if (iv >= sp.nvec) break;
            float x[N];
            Vec<T>::unpack(v[u], x);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = grad(x[i]);
            of_hot([&](int place, float w) {
                const int at = place - first;
                if (static_cast<unsigned>(at) < static_cast<unsigned>(N))  // (no branches inside: they would put x into memory)
#pragma unroll
                    for (int i = 0; i < N; ++i) x[i] += at == i ? w : 0.0f;
            });
            store16<Stream>(vectors() + iv, Vec<T>::pack(x));
        }
    };
    if (fabsf(lse) <= kFarLse<T> || lse != lse) {
        // (what rounding -lse log2(e) takes off all exponents alike goes into the factors)
        const float nl = -lse * kLog2e, rest = fmaf(-lse, kLog2e, -nl), g = __builtin_amdgcn_exp2f(rest);
        c = g * fmaf(c2, rest, c);
        c2 *= g;
        return finish([&](float z) { return fmaf(z, kLog2e, nl); });
    }
    const uint32_t share = kFarUnits / static_cast<uint32_t>(rows.T), groups = share < 1 ? 1 : share;  // of a row
    if (seg >= groups) return;
    float top, log_sum;
    row_max_log<T, TR>(row, rows.V, top, log_sum);
    for (;;) {
        finish([&](float z) { return ((z - top) - log_sum) * kLog2e; });
        seg += groups;
        if (seg >= nseg) return;
        start();
        request();
    }
}

// ----------------------------------------------------------------------------
// a few tokens from hidden states and the head
// ----------------------------------------------------------------------------
// Up to kFewTokens tokens (a server's step): bound by one read of the head, 1.24 GB at 4096 x 151936 in bf16.  The sweep's
// tiles of 128 tokens take 231 us for that, 239 with their preparation and joining.
//   One token, or two of more than 2048 hidden units: a wavefront forms one vocabulary entry's logits after the other as dot
//   products, its row read by whole kilobytes, the hidden states in registers; rows go round the wavefronts of the chip, which
//   so walks the head in order (181 us = 6.9 TB/s; two tokens 184).  The sums over lanes are what does not scale: four tokens
//   take 228 us, of 1024 hidden units 106 (and 57 the other way).
//   More: a wavefront forms the logits of 16 vocabulary entries by 16 tokens, the entries' rows straight from memory into the
//   operands of the matrix instruction, kFewLoads loads of 16 bytes per lane at a time and as many on their way behind them;
//   the hidden states wait in LDS; blocks of 16 entries go round the wavefronts or the workgroups (223 to 247 us; 16 rows of 64
//   bytes per load do not reach the rate of whole rows).
constexpr int kFewTokens = 16, kFewWaves = 8, kFewLoads = 8, kFewGroups = 512;
constexpr int kFewPad = 16;                // bytes behind a token's row in LDS: rows on different banks
constexpr int64_t kFewLds = 140 * 1024;
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// a wavefront's values of tokens 0 .. T-1 joined over the workgroup, into part[token][workgroup]
template <int Waves>
__device__ __forceinline__ void store_few(float (*joined)[kFewTokens][3], int T, float *part) {
    __syncthreads();
    if (threadIdx.x >= T) return;
    const int t = threadIdx.x;
    float m = joined[0][t][0], s = joined[0][t][1], u = joined[0][t][2];
    for (int w = 1; w < Waves; ++w) score_join(m, s, u, joined[w][t][0], joined[w][t][1], joined[w][t][2]);
    float *o = part + (static_cast<int64_t>(t) * gridDim.x + blockIdx.x) * 3;
    o[0] = m;
    o[1] = s;
    o[2] = u;
}

typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
constexpr int kDotSpan = 8 * kWave;  // elements of a row per load of a wavefront
// Up to NT tokens of up to 512 * NC hidden units, R rows of the head at a time (short rows: as many loads on their way as
// long ones have).
template <int NT, int NC, int R>
__global__ void __launch_bounds__(kFewWaves * kWave, 2)
few_dots_kernel(const bf16_t *__restrict__ X, const bf16_t *__restrict__ W, int T, int H, int64_t V, const int32_t *__restrict__ target,
                float *__restrict__ part, float *__restrict__ z_target) {
    static_assert(kWave % R == 0, "a lane keeps whole rounds of rows");
    __shared__ float joined[kFewWaves][kFewTokens][3];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kFewWaves * R, r0 = (static_cast<int64_t>(blockIdx.x) * kFewWaves + wave) * R;
    const int chunks = (H + kDotSpan - 1) / kDotSpan;
    // (past the end of a row its start is read, and counts as zeros; past the last row the last)
    auto request = [&](uint4 (&v)[R][NC], int64_t r) {
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const bf16_t *row = W + (r + q < V ? r + q : V - 1) * H;
#pragma unroll
            for (int j = 0; j < NC; ++j)
                if (j < chunks) {
                    const int k = j * kDotSpan + lane * 8;
                    const u32x4_t w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(row + (k < H ? k : 0)));
                    v[q][j] = make_uint4(w.x, w.y, w.z, w.w);
                }
        }
    };
    uint4 now[R][NC], next[R][NC], x[NT][NC];
    if (r0 < V) request(now, r0);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int k = j * kDotSpan + lane * 8;
            x[t][j] = t < T && k < H ? *reinterpret_cast<const uint4 *>(X + static_cast<int64_t>(t) * H + k) : make_uint4(0u, 0u, 0u, 0u);
        }
    int64_t y[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) y[t] = target && t < T ? target[t] : -1;
    float m[NT], s[NT], u[NT], z[NT];  // lane l: of the logits of the l-th, (l + 64)-th, ... row of this wavefront's
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m[t] = kLowestFloat;
        s[t] = u[t] = 0.0f;
        z[t] = -INFINITY;
    }
    auto take = [&] {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float mx = fmaxf(m[t], z[t]), d = fmaxf((m[t] - mx) * kLog2e, kLowest2), q = (z[t] - mx) * kLog2e;
            const float f = __builtin_amdgcn_exp2f(d), e = __builtin_amdgcn_exp2f(q);  // (a NaN stays one)
            u[t] = f * fmaf(d, s[t], u[t]) + e * fmaxf(q, kLowest2);
            s[t] = f * s[t] + e;
            m[t] = mx;
            z[t] = -INFINITY;
        }
    };
    int n = 0;  // place of the next row among the lanes
    for (int64_t r = r0; r < V; r += stride) {
        if (r + stride < V) request(next, r + stride);
        float a[R][NT][2];
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int t = 0; t < NT; ++t) a[q][t][0] = a[q][t][1] = 0.0f;
#pragma unroll
        for (int j = 0; j < NC; ++j)
            if (j < chunks)
#pragma unroll
                for (int q = 0; q < R; ++q) {
                    uint32_t w[4] = {now[q][j].x, now[q][j].y, now[q][j].z, now[q][j].w};
                    if ((j + 1) * kDotSpan > H)  // an infinite weight times a zero that is not there
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = j * kDotSpan + lane * 8 < H ? w[i] : 0u;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const uint32_t h[4] = {x[t][j].x, x[t][j].y, x[t][j].z, x[t][j].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            a[q][t][i & 1] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2v_t, w[i]),
                                                                             __builtin_bit_cast(bf16x2v_t, h[i]), a[q][t][i & 1], false);
                    }
                }
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float sum = wave_sum(a[q][t][0] + a[q][t][1]);
                if (r + q < V) {
                    z[t] = lane == n + q ? sum : z[t];
                    if (r + q == y[t] && lane == 0) z_target[t] = sum;
                }
            }
        n = (n + R) % kWave;
        if (n == 0) take();
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int j = 0; j < NC; ++j) now[q][j] = next[q][j];
    }
    take();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        join_lanes(m[t], s[t], u[t]);
        if (lane == 0) {
            joined[wave][t][0] = m[t];
            joined[wave][t][1] = s[t];
            joined[wave][t][2] = u[t];
        }
    }
    store_few<kFewWaves>(joined, T, part);
}

static bool few_tokens(const spo_logprob_desc *d) {
    return d->dtype == SPO_BF16 && d->w_layout == SPO_W_VH && d->T <= kFewTokens && d->T * (d->H * 2 + kFewPad) <= kFewLds;
}
constexpr int kFewParts = 2 * kFewWaves * kWave * 16;  // bytes
// Whether the wavefronts of a workgroup share a block of entries.  Blocks of their own leave wavefronts without one where blocks
// are few (three tokens, 2496 x 6024: 22.9 us, shared 11.1; 4096 x 3000 32.0 and 9.7; 256 x 2000 5.6 and 4.3) or the last round of
// them is (960 x 73158 37.2 and 29.0), and rows of 8 KB come faster shared (4096 x 151936 235 and 223).  Otherwise the barrier and
// the joining of every block cost more (512 x 151936 30.3 and 38.8, 2048 x 151936 119 and 126, 512 x 32000 8.2 and 9.7).
static bool shared_few(const spo_logprob_desc *d) {
    const int64_t blocks = ceil_div(d->V, 16), places = kFewGroups / 2 * kFewWaves, taken = ceil_div(blocks, places) * places;
    return d->H >= 4096 || blocks <= places / 2 || (d->H >= 768 && 4 * taken >= 5 * blocks);
}

// part[token][workgroup] = (max, sum of 2^x, sum of x 2^x); z_target[token] where the target is in the vocabulary
// Shared: the wavefronts of a workgroup share the hidden units of a block of entries, and one of them in turn adds their parts
// up in order; otherwise each has blocks of its own.
template <bool Shared>
__global__ void __launch_bounds__(kFewWaves * kWave, 2)
few_tokens_kernel(const bf16_t *__restrict__ X, const bf16_t *__restrict__ W, int T, int H, int64_t V, const int32_t *__restrict__ target,
                  float *__restrict__ part, float *__restrict__ z_target) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float joined[kFewWaves][kFewTokens][3];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const int col = lane & 15, grp = lane >> 4, pitch = H * 2 + kFewPad;
    const int64_t blocks = ceil_div(V, 16), stride = Shared ? gridDim.x : static_cast<int64_t>(gridDim.x) * kFewWaves;
    const int share = Shared ? (H / 32 + kFewWaves - 1) / kFewWaves : H / 32;  // of 32 hidden units: this wavefront's first and number
    const int first = Shared ? wave * share : 0, slices = H / 32 - first < share ? H / 32 - first : share;
    const int chunks = (share + kFewLoads - 1) / kFewLoads;
    // chunk c of block b: this lane's row of W (the last one past the vocabulary) from slice kFewLoads * c of its share on
    uint4 set[2][kFewLoads];
    auto request = [&](uint4 (&v)[kFewLoads], int64_t b, int c) {
        const int64_t r = b * 16 + col;
        const bf16_t *row = W + (r < V ? r : V - 1) * H + first * 32 + 8 * grp;
#pragma unroll
        for (int i = 0; i < kFewLoads; ++i) {
            const int sl = c * kFewLoads + i;
            if (Shared && sl >= slices) break;
            const u32x4_t w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(row + (Shared || sl < slices ? sl : slices - 1) * 32));
            v[i] = make_uint4(w.x, w.y, w.z, w.w);
        }
    };
    int64_t b = Shared ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * kFewWaves + wave;
    if (b < blocks) request(set[0], b, 0);
    for (int i = threadIdx.x; i < T * (H / 8); i += blockDim.x) {
        const int t = i / (H / 8), k = i % (H / 8);
        *reinterpret_cast<uint4 *>(lds + t * pitch + k * 16) = *reinterpret_cast<const uint4 *>(X + static_cast<int64_t>(t) * H + k * 8);
    }
    const int64_t y = target && col < T ? target[col] : -1;
    __syncthreads();
    const char *x = lds + (col < T ? col : 0) * pitch + grp * 16 + first * 64;  // (columns past the tokens: the first, not used)
    f32x4_t *parts = reinterpret_cast<f32x4_t *>(lds + T * pitch);             // Shared: [parity of the block][wavefront][lane]
    int turn = 0;                                                              // blocks so far
    float m = kLowestFloat, s = 0.0f, u = 0.0f;
    f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
    int c = 0;
    auto work = [&](uint4 (&now)[kFewLoads], uint4 (&next)[kFewLoads]) {
        const bool last = c + 1 == chunks;
        const int64_t nb = last ? b + stride : b;
        if (nb < blocks) request(next, nb, last ? 0 : c + 1);
#pragma unroll
        for (int i = 0; i < kFewLoads; ++i) {
            const int sl = c * kFewLoads + i;
            if (sl < slices)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, now[i]),
                                                              *reinterpret_cast<const bf16x8_t *>(x + sl * 64), acc, 0, 0, 0);
        }
        bool mine = last;
        if (Shared && last) {
            // (one barrier: a block's parts are read before the reader comes to the next barrier, and written over after that)
            parts[(turn % 2 * kFewWaves + wave) * kWave + lane] = acc;
            acc = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            __syncthreads();
            mine = turn % kFewWaves == wave;
            if (mine)
                for (int w = 0; w < kFewWaves; ++w) acc += parts[(turn % 2 * kFewWaves + w) * kWave + lane];
            ++turn;
        }
        if (mine) {  // a lane holds entries 4 grp .. 4 grp + 3 of the block for token col
            const int64_t v0 = b * 16 + 4 * grp;
            float mx = m;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (v0 + r >= V) acc[r] = -INFINITY;
                if (v0 + r == y) z_target[col] = acc[r];
                mx = fmaxf(mx, acc[r]);
            }
            const float d = fmaxf((m - mx) * kLog2e, kLowest2), f = __builtin_amdgcn_exp2f(d);
            u = f * fmaf(d, s, u);
            s *= f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float q = (acc[r] - mx) * kLog2e, e = __builtin_amdgcn_exp2f(q);  // (a NaN stays one)
                s += e;
                u = fmaf(e, fmaxf(q, kLowest2), u);
            }
            m = mx;
            acc = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
        c = last ? 0 : c + 1;
        b = nb;
    };
    while (b < blocks) {
        work(set[0], set[1]);
        if (b >= blocks) break;
        work(set[1], set[0]);
    }
#pragma unroll
    for (int o = 16; o < kWave; o <<= 1) {
        // (the lower lane's values first, so that both lanes of a pair form the same sums)
        const float om = __shfl_xor(m, o, kWave), os = __shfl_xor(s, o, kWave), ou = __shfl_xor(u, o, kWave);
        float a = lane & o ? om : m, p = lane & o ? os : s, q = lane & o ? ou : u;
        score_join(a, p, q, lane & o ? m : om, lane & o ? s : os, lane & o ? u : ou);
        m = a; s = p; u = q;
    }
    if (grp == 0) {
        joined[wave][col][0] = m;
        joined[wave][col][1] = s;
        joined[wave][col][2] = u;
    }
    store_few<kFewWaves>(joined, T, part);
}

// Scores of token blockIdx.x from the workgroups' shares: a chain of loads and shuffles, 4.7 us.
__global__ void __launch_bounds__(kWave)
few_scores_kernel(const float *__restrict__ part, int groups, const float *__restrict__ z_target, ScoreRows rows, ScoreOut out) {
    const int64_t t = blockIdx.x;
    if (rows.mask && !rows.mask[t]) {
        if (threadIdx.x == 0) store_left_out(out, t);
        return;
    }
    float zt = 0.0f, m, s, u;
    if (rows.target) {
        const int64_t y = rows.target[t];
        zt = y >= 0 && y < rows.V ? z_target[t] : __builtin_nanf("");
    }
    join_segments(part, groups, t, m, s, u);
    if (threadIdx.x == 0) store_scores(out, t, zt, m, s, u);
}

// ----------------------------------------------------------------------------
// host side
// ----------------------------------------------------------------------------
static ScoreRows score_rows(const spo_logprob_desc *d) {
    return ScoreRows{d->T, d->V, d->logits_stride ? d->logits_stride : d->V, d->target, d->mask};
}

static bool streams(const spo_logprob_desc *d) { return d->T * d->V * (d->dtype == SPO_FP32 ? 4 : 2) > kStreamBytes; }

// one round per segment where two would leave compute units without their eight workgroups
static RowGrid score_grid(const spo_logprob_desc *d) {
    const RowGrid g = row_grid(d->T, d->V, d->dtype, kScoreGroup, kScoreRounds, kScoreNarrow);
    return g.units() >= 2048 ? g : row_grid(d->T, d->V, d->dtype, kScoreGroup, 1, kScoreNarrow);
}

struct ScorePlan {
    RowGrid grid;
    float *part, *group_max;
    size_t bytes;
};
static ScorePlan plan_scores(const spo_logprob_desc *d, void *ws) {
    ScorePlan p;
    const int64_t T = std::max<int64_t>(d->T, 1);
    p.grid = score_grid(d);
    Arena a(ws);
    // room for the shortest segments and groups of either type: those in use get longer with T and V, and room sized for the
    // largest batch is to serve every smaller one
    p.part = a.take<float>(static_cast<size_t>(T * ceil_div(d->V, kWave * kScoreGroup * Vec<float>::N)) * 3);
    p.group_max = d->top_k ? a.take<float>(static_cast<size_t>(T * (ceil_div(d->V, kScoreGroup * Vec<float>::N) + kRowThreads))) : nullptr;
    p.bytes = a.used;
    return p;
}

template <typename T, int TR, bool Stream, bool Top>
static void launch_score_rows(const spo_logprob_desc *d, const ScorePlan &p, const ScoreOut &o, hipStream_t s) {
    auto *kernel = p.grid.seg_len <= TR * kScoreGroup * Vec<T>::N ? score_rows_kernel<T, TR, 1, Stream, Top>
                                                                 : score_rows_kernel<T, TR, kScoreRounds, Stream, Top>;
    kernel<<<p.grid.blocks(), kRowThreads, 0, s>>>(static_cast<const T *>(d->logits), score_rows(d), p.grid, p.part, p.group_max, o);
}
template <typename T, bool Top>
static void launch_scores(const spo_logprob_desc *d, const ScorePlan &p, const ScoreOut &o, hipStream_t s) {
    const bool narrow = p.grid.per_wg > 1;
    if (narrow) streams(d) ? launch_score_rows<T, kWave, true, Top>(d, p, o, s) : launch_score_rows<T, kWave, false, Top>(d, p, o, s);
    else if (streams(d)) launch_score_rows<T, kRowThreads, true, Top>(d, p, o, s);
    else launch_score_rows<T, kRowThreads, false, Top>(d, p, o, s);
    const T *z = static_cast<const T *>(d->logits);
    if constexpr (Top) {
        auto *pick = narrow ? score_pick_kernel<T, kWave> : score_pick_kernel<T, kRowThreads>;
        pick<<<fold_grid(d->T), kPickThreads, 0, s>>>(z, score_rows(d), p.grid, p.part, p.group_max, o);
    } else if (p.grid.nseg > 1) {
        score_join_kernel<T><<<fold_grid(ceil_div(d->T, 4)), 256, 0, s>>>(z, score_rows(d), p.grid.nseg, p.part, o);
    }
}

static int logits_logprob_fwd(const spo_logprob_desc *d, const ScoreOut &o, void *ws, size_t ws_bytes, hipStream_t s) {
    const ScorePlan p = plan_scores(d, ws);
    if (ws_bytes < p.bytes) return SPO_EWORKSPACE;
    if (d->T == 0) return SPO_OK;
    ScopedKernelTimer timer(kTimeLogitsFwd, s);
    if (d->dtype == SPO_BF16) o.K ? launch_scores<bf16_t, true>(d, p, o, s) : launch_scores<bf16_t, false>(d, p, o, s);
    else o.K ? launch_scores<float, true>(d, p, o, s) : launch_scores<float, false>(d, p, o, s);
    return launch_status();
}

struct FewPlan {
    float *part, *z_target;
    size_t bytes;
};
static FewPlan plan_few(void *ws) {
    FewPlan p;
    Arena a(ws);
    p.part = a.take<float>(kFewTokens * kFewGroups * 3);
    p.z_target = a.take<float>(kFewTokens);
    p.bytes = a.used;
    return p;
}

static int few_logprob_fwd(const spo_logprob_desc *d, const ScoreOut &o, void *ws, size_t ws_bytes, hipStream_t s) {
    const FewPlan p = plan_few(ws);
    if (ws_bytes < p.bytes) return SPO_EWORKSPACE;
    if (d->T == 0) return SPO_OK;
    const int64_t chunks = ceil_div(d->H, kDotSpan);
    const bool dots = (d->T == 1 && chunks <= 16) || (d->T == 2 && chunks > 4 && chunks <= 8);
    const int64_t rows = !dots ? 16 : chunks <= 2 ? 4 : chunks <= 4 ? 2 : 1;  // that a wavefront takes at a time
    const bool shared = !dots && shared_few(d);
    const int groups = static_cast<int>(std::min<int64_t>(dots || shared ? kFewGroups : kFewGroups / 2, ceil_div(d->V, shared ? rows : rows * kFewWaves)));
    const int lds = dots ? 0 : static_cast<int>(d->T * (d->H * 2 + kFewPad)) + (shared ? kFewParts : 0);
    auto *kernel = shared       ? few_tokens_kernel<true>
                   : !dots      ? few_tokens_kernel<false>
                   : d->T == 2  ? few_dots_kernel<2, 8, 1>
                   : chunks > 8 ? few_dots_kernel<1, 16, 1>
                   : rows == 4  ? few_dots_kernel<1, 2, 4>
                   : rows == 2  ? few_dots_kernel<1, 4, 2>
                                : few_dots_kernel<1, 8, 1>;
    // (the limit is the kernel's, not this call's: every call sets the same, so that no other thread's can lower it before the launch)
    if (!dots && hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                     static_cast<int>(kFewLds) + (shared ? kFewParts : 0)) != hipSuccess)
        return SPO_EHIP;
    {
        ScopedKernelTimer timer(kTimeFwdSweep, s);
        kernel<<<groups, kFewWaves * kWave, lds, s>>>(static_cast<const bf16_t *>(d->hidden), static_cast<const bf16_t *>(d->W),
                                                      static_cast<int>(d->T), static_cast<int>(d->H), d->V, d->target, p.part, p.z_target);
    }
    few_scores_kernel<<<static_cast<unsigned>(d->T), kWave, 0, s>>>(p.part, groups, p.z_target, score_rows(d), o);
    return launch_status();
}

template <typename T>
static void launch_score_grad(const spo_logprob_desc *d, const ScoreGrads &g, void *d_logits, hipStream_t s) {
    const RowGrid grid = row_grid(d->T, d->V, d->dtype, kScoreGradGroup, 1, kScoreGradNarrow);
    auto *kernel = grid.per_wg > 1 ? score_grad_kernel<T, kWave, false>
                 : streams(d)      ? score_grad_kernel<T, kRowThreads, true>
                                   : score_grad_kernel<T, kRowThreads, false>;
    kernel<<<grid.blocks(), kRowThreads, 0, s>>>(static_cast<const T *>(d->logits), score_rows(d), grid, g, static_cast<T *>(d_logits));
}

}  // namespace spo

using namespace spo;

static int validate(const spo_logprob_desc *d) {
    if (!d) return SPO_ENULL;
    if (d->struct_size != sizeof(spo_logprob_desc)) return SPO_EINVAL;
    if (d->dtype != SPO_BF16 && d->dtype != SPO_FP32) return SPO_EINVAL;
    if (d->T < 0 || d->V < 1) return SPO_EINVAL;
    if (d->T >= (int64_t(1) << 31) || d->V >= (int64_t(1) << 31)) return SPO_ERANGE;
    if (d->top_k < 0 || d->top_k > d->V) return SPO_EINVAL;
    if (d->top_k > SPO_MAX_TOP_K) return SPO_ERANGE;
    const uintptr_t elt = d->dtype == SPO_FP32 ? 4 : 2;
    if (d->logits) {
        if (d->logits_stride != 0 && d->logits_stride < d->V) return SPO_EINVAL;
        if (reinterpret_cast<uintptr_t>(d->logits) % elt) return SPO_EINVAL;
        return SPO_OK;
    }
    if (d->w_layout != SPO_W_VH && d->w_layout != SPO_W_HV) return SPO_EINVAL;
    if (!d->W || (d->T > 0 && !d->hidden)) return SPO_ENULL;
    if (d->H < 1) return SPO_EINVAL;
    if (d->H % 64 != 0 || d->top_k != 0) return SPO_EUNSUPPORTED;
    if (d->H > 65536) return SPO_ERANGE;
    if (reinterpret_cast<uintptr_t>(d->hidden) % 16 || reinterpret_cast<uintptr_t>(d->W) % 16) return SPO_EINVAL;
    return SPO_OK;
}

extern "C" size_t spo_logprob_fwd_workspace_bytes(const spo_logprob_desc *d) {
    if (validate(d) != SPO_OK) return 0;
    size_t b = 0;
    if (d->logits) return plan_scores(d, nullptr).bytes;
    head_logprob_fwd_workspace(d, &b);
    return std::max(b, plan_few(nullptr).bytes);  // (of any number of tokens: it serves smaller batches)
}

extern "C" int spo_logprob_fwd(const spo_logprob_desc *d, float *logp, float *lse, float *entropy, int32_t *top_id, float *top_logp,
                               void *ws, size_t ws_bytes, spo_stream_t stream) {
    const int rc = validate(d);
    if (rc) return rc;
    if (d->T > 0 && (!lse || (d->target && !logp) || (d->top_k && (!top_id || !top_logp)))) return SPO_ENULL;
    if (!ws) return SPO_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0) return SPO_EINVAL;
    if (!d->target) logp = nullptr;
    if (!d->logits && few_tokens(d)) return few_logprob_fwd(d, ScoreOut{logp, lse, entropy, nullptr, nullptr, 0}, ws, ws_bytes, as_stream(stream));
    if (!d->logits) return head_logprob_fwd(d, logp, lse, entropy, ws, ws_bytes, as_stream(stream));
    return logits_logprob_fwd(d, ScoreOut{logp, lse, entropy, top_id, top_logp, d->top_k}, ws, ws_bytes, as_stream(stream));
}

extern "C" size_t spo_logprob_bwd_workspace_bytes(const spo_logprob_desc *d, int64_t chunk_tokens) {
    if (validate(d) != SPO_OK || chunk_tokens < 0) return 0;
    size_t b = 256;  // the logits-in form needs none; a size that serves as one
    if (!d->logits) head_logprob_bwd_workspace(d, chunk_tokens, &b);
    return b;
}

extern "C" int spo_logprob_bwd(const spo_logprob_desc *d, const float *lse, const float *entropy, const float *d_logp,
                               const float *d_entropy, const int32_t *top_id, const float *d_top_logp, void *d_hidden,
                               int d_hidden_dtype, void *d_W, int d_W_dtype, int accumulate_dW, void *d_logits, int64_t chunk_tokens,
                               void *ws, size_t ws_bytes, spo_stream_t stream) {
    const int rc = validate(d);
    if (rc) return rc;
    if (chunk_tokens < 0) return SPO_EINVAL;
    if (d->T > 0 && (!lse || (d_entropy && !entropy) || (d_logp && !d->target) || (d_top_logp && !top_id))) return SPO_ENULL;
    if (d_top_logp && !d->top_k) return SPO_EINVAL;
    if (d->logits) {
        if (d->T == 0) return SPO_OK;
        if (!d_logits) return SPO_ENULL;
        const uintptr_t elt = d->dtype == SPO_FP32 ? 4 : 2;
        if (reinterpret_cast<uintptr_t>(d_logits) % elt) return SPO_EINVAL;
        const ScoreGrads g{lse, entropy, d_logp, d_entropy, top_id, d_top_logp, d->top_k};
        ScopedKernelTimer timer(kTimeLogitsBwd, as_stream(stream));
        if (d->dtype == SPO_BF16) launch_score_grad<bf16_t>(d, g, d_logits, as_stream(stream));
        else launch_score_grad<float>(d, g, d_logits, as_stream(stream));
        return launch_status();
    }
    if (!ws) return SPO_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(ws) % 256 != 0) return SPO_EINVAL;
    auto type_ok = [](int t) { return t == SPO_FP32 || t == SPO_BF16; };
    if ((d_hidden && !type_ok(d_hidden_dtype)) || (d_W && !type_ok(d_W_dtype))) return SPO_EINVAL;
    if (reinterpret_cast<uintptr_t>(d_hidden) % 16 || reinterpret_cast<uintptr_t>(d_W) % 16) return SPO_EINVAL;
    return head_logprob_bwd(d, lse, entropy, d_logp, d_entropy, d_hidden, d_hidden_dtype, d_W, d_W_dtype, accumulate_dW, chunk_tokens, ws,
                            ws_bytes, as_stream(stream));
}
