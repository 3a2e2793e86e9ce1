// Logits-in form of the clipped policy-gradient loss: the [T x V] logits already
// exist and are streamed once (forward) or read once and written once
// (backward).  Pure HBM streaming, 16 bytes per lane and access.
#include <algorithm>

#include "row_stream.hpp"
#include "timing.hpp"

namespace spo {

// What bounds both kernels is memory, and how many separate streams of addresses are open at once:
// a workgroup per row of 304 KB keeps 2048 rows open (8192 x 151936 bf16: forward 451 us, backward
// 968 us = 5.5 and 5.1 TB/s).  So a row is cut into short segments, neighbouring workgroups work on
// neighbouring segments, and the chip sweeps the array nearly in order (350 us = 7.1 TB/s and
// 772 us = 6.4 TB/s).  The forward takes two rounds of kLseGroup 16-byte loads per thread (a third of
// the partial results of one round; with four 368 us), the second on its way while the first is worked
// on; the backward has nothing to carry along and takes one round of kGradGroup (four per thread:
// 806 us, two rounds of four 842 us).
// Arrays that no cache can hold are read and written with the non-temporal hint: the forward of the
// next pass then finds no modified lines of the gradients to drain first (forward 437 -> 350 us).
// Rows of a few thousand entries are bound by instructions as well: a thread works on two or three vectors per
// row.  There vectors that a segment does not have are not worked on, a segment of one round has no second one to
// request, and a wavefront's pairs are merged with one exponential (60000 rows of 4104 in bf16: 138 -> 81 us;
// a workgroup per row without segments took 96).
constexpr int kLseGroup = 4, kLseRounds = 2, kGradGroup = 2;

// running (max, sum of exp(x - max)) merged with another pair
__device__ __forceinline__ void lse_merge(float &m, float &s, float om, float os) {
    const float nm = fmaxf(m, om);
    s = s * __builtin_amdgcn_exp2f((m - nm) * kLog2e) + os * __builtin_amdgcn_exp2f((om - nm) * kLog2e);
    m = nm;
}

// (max, sum-exp) of one segment of a row, by TR threads (a workgroup or one wavefront of it), and the
// target's logit.  part_max / part_sum [segment][row].  Also clears *done.
template <typename T, int TR, int Rounds, bool Stream>
__global__ void __launch_bounds__(kRowThreads)
logits_row_lse_kernel(const T *__restrict__ logits, int64_t V, RowGrid grid, const int32_t *__restrict__ target,
                      float *__restrict__ part_max, float *__restrict__ part_sum, float *__restrict__ z_target,
                      uint32_t *__restrict__ done) {
    constexpr int N = Vec<T>::N, U = kLseGroup;
    const int64_t unit = group_unit<TR>();
    const int tid = threadIdx.x % TR;
    if (unit == 0 && threadIdx.x == 0) *done = 0u;  // for the kernel that follows
    if (unit >= grid.units()) return;  // TR < kRowThreads only: no barrier below in that case
    const uint32_t seg = static_cast<uint32_t>(unit) % static_cast<uint32_t>(grid.nseg);
    const int64_t t = static_cast<uint32_t>(unit) / static_cast<uint32_t>(grid.nseg), e0 = seg * grid.seg_len;
    const T *p = logits + t * V + e0;
    const Span sp(p, static_cast<int>(V - e0 < grid.seg_len ? V - e0 : grid.seg_len));
    float zt = 0.0f;
    if (seg == 0 && tid == 0) {
        const int64_t y = target[t];  // an id outside [0, V) gives NaN instead of a read out of bounds
        zt = (y >= 0 && y < V) ? Vec<T>::get(logits + t * V + y) : __builtin_nanf("");
    }
    // the few elements outside the whole vectors, one per thread
    float m = kNegBig, s = 0.0f;
    if (tid < sp.head + sp.tail) {
        const float x = Vec<T>::get(p + (tid < sp.head ? tid : tid + sp.nvec * N));
        m = fmaxf(m, x);
        s = __builtin_amdgcn_exp2f((x - m) * kLog2e);
    }
    const T *body = p + sp.head;
    auto request = [&](uint4 (&v)[U], int i0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * TR < sp.nvec) v[u] = load16<Stream>(body + (i0 + u * TR) * N);
    };
    auto take = [&](const uint4 (&v)[U], int i0) {
        // one new maximum and one rescaling of the running sum for the whole group; vectors past the end are left out
        // (rows of 4104: one in two of the group's)
        float x[U][N], mx = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * TR >= sp.nvec) break;
            Vec<T>::unpack(v[u], x[u]);
#pragma unroll
            for (int i = 0; i < N; ++i) mx = fmaxf(mx, x[u][i]);
        }
        const float nm2 = -mx * kLog2e;
        float a[U] = {};
        auto add = [&](auto exponent) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u * TR >= sp.nvec) break;
#pragma unroll
                for (int i = 0; i < N; ++i) a[u] += __builtin_amdgcn_exp2f(exponent(x[u][i]));
            }
        };
        if (__any(i0 < sp.nvec && fabsf(mx) > kFarLogit)) add([&](float v) { return (v - mx) * kLog2e; });
        else add([&](float v) { return fmaf(v, kLog2e, nm2); });
        s = s * __builtin_amdgcn_exp2f((m - mx) * kLog2e) + ((a[0] + a[1]) + (a[2] + a[3]));
        m = mx;
    };
    uint4 cur[U];
    request(cur, tid);
    if constexpr (Rounds > 1) {
        uint4 nxt[U];
        for (int i0 = tid; i0 < sp.nvec; i0 += U * TR) {
            request(nxt, i0 + U * TR);
            take(cur, i0);
#pragma unroll
            for (int u = 0; u < U; ++u) cur[u] = nxt[u];
        }
    } else {
        take(cur, tid);
    }
    // one maximum for the wavefront, then one rescaling and the sum (merging pairs takes two exponentials per step)
    float top = m;
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
    s = wave_sum(s * __builtin_amdgcn_exp2f((m - top) * kLog2e));
    m = top;
    if constexpr (TR > kWave) {
        __shared__ float sm[TR / kWave], ss[TR / kWave];
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) { sm[wave] = m; ss[wave] = s; }
        __syncthreads();
        m = sm[0];
        s = ss[0];
        for (int w = 1; w < TR / kWave; ++w) lse_merge(m, s, sm[w], ss[w]);
    }
    if (tid == 0) {
        part_max[seg * grid.rows + t] = m;
        part_sum[seg * grid.rows + t] = s;
        if (seg == 0) z_target[t] = zt;
    }
}

// d_logits[t][v] = g[t] * ([v == target[t]] - exp(z[t][v] - lse[t])) of one segment of a row (at most
// kGradGroup vectors per thread); rows whose scale is zero are written as zeros without being read.
// Vectors are aligned on the output side; the input's (the same boundaries unless the two arrays are
// offset against each other) may be unaligned.
template <typename T, int TR, bool Stream>
__global__ void __launch_bounds__(kRowThreads)
logits_row_grad_kernel(const T *__restrict__ logits, int64_t V, RowGrid grid, const int32_t *__restrict__ target,
                       const float *__restrict__ lse, const float *__restrict__ g, T *__restrict__ d_logits) {
    constexpr int N = Vec<T>::N, U = kGradGroup;
    const int64_t unit = group_unit<TR>();
    const int tid = threadIdx.x % TR;
    if (unit >= grid.units()) return;
    const uint32_t nseg = static_cast<uint32_t>(grid.nseg);
    const int64_t t = static_cast<uint32_t>(unit) / nseg, e0 = (static_cast<uint32_t>(unit) % nseg) * grid.seg_len;
    const T *p = logits + t * V + e0;
    T *out = d_logits + t * V + e0;
    const Span sp(out, static_cast<int>(V - e0 < grid.seg_len ? V - e0 : grid.seg_len));
    const float gt = g[t], ng = -gt, nl = -lse[t] * kLog2e;
    const int64_t yl = static_cast<int64_t>(target[t]) - e0;  // target's place in the segment
    const int y = yl >= 0 && yl < grid.seg_len ? static_cast<int>(yl) : -1;
    auto grad = [&](float x) { return ng * __builtin_amdgcn_exp2f(fmaf(x, kLog2e, nl)); };
    if (tid < sp.head + sp.tail) {
        const int e = tid < sp.head ? tid : tid + sp.nvec * N;
        Vec<T>::put(out + e, gt != 0.0f ? grad(Vec<T>::get(p + e)) + (e == y ? gt : 0.0f) : 0.0f);
    }
    const T *body = p + sp.head;
    uint4 *dst = reinterpret_cast<uint4 *>(out + sp.head);
    if (gt == 0.0f) {
        for (int i = tid; i < sp.nvec; i += TR) store16<Stream>(dst + i, make_uint4(0u, 0u, 0u, 0u));
        return;
    }
    const int yv = y >= sp.head ? (y - sp.head) / N : -1, yr = y >= sp.head ? (y - sp.head) % N : 0;
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (tid + u * TR < sp.nvec) v[u] = load16<Stream>(body + (tid + u * TR) * N);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int iv = tid + u * TR;
        if (iv >= sp.nvec) break;
        float x[N];
        Vec<T>::unpack(v[u], x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = grad(x[i]);
        if (iv == yv) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i == yr) x[i] += gt;
        }
        store16<Stream>(dst + iv, Vec<T>::pack(x));
    }
}

// (see row_grid for what narrow_eighths means)
constexpr int kLseNarrow = 5, kGradNarrow = 4;
static RowGrid row_grid(const spo_pg_desc *d, int group, int rounds, int narrow_eighths) {
    return row_grid(d->T, d->V, d->dtype, group, rounds, narrow_eighths);
}

// the forward goes down to one round per segment where two would leave compute units without their
// eight workgroups (256 x 151936 bf16: 17.4 against 18.0 us)
static RowGrid lse_grid(const spo_pg_desc *d) {
    const RowGrid g = row_grid(d, kLseGroup, kLseRounds, kLseNarrow);
    return g.units() >= 2048 ? g : row_grid(d, kLseGroup, 1, kLseNarrow);
}

static bool streams(const spo_pg_desc *d) {
    return d->T * d->V * (d->dtype == SPO_FP32 ? 4 : 2) > kStreamBytes;
}

struct LogitsFwdPlan {
    RowGrid grid;
    float *row_max, *row_sum, *z_target;
    FwdPartial *partials;
    uint32_t *done;
    int64_t nblk_tok;
    size_t bytes;
};

static LogitsFwdPlan plan_logits_fwd(const spo_pg_desc *d, void *ws) {
    LogitsFwdPlan p;
    const int64_t Tn = std::max<int64_t>(d->T, 1);
    p.nblk_tok = ceil_div(Tn, kTokThreads);
    p.grid = lse_grid(d);
    Arena a(ws);
    // room for rows of T and V cut into the shortest segments of either type (0.4 % of the logits' bytes): the segments
    // in use get longer with T and V, and room sized for the largest batch is to serve every smaller one
    const size_t room = static_cast<size_t>(Tn * ceil_div(d->V, kWave * kLseGroup * Vec<float>::N));
    p.row_max = a.take<float>(room);
    p.row_sum = a.take<float>(room);
    p.z_target = a.take<float>(Tn);
    p.partials = a.take<FwdPartial>(p.nblk_tok);
    p.done = a.take<uint32_t>(1);
    p.bytes = a.used;
    return p;
}

template <typename T, int TR, bool Stream>
static void launch_row_lse(const spo_pg_desc *d, const LogitsFwdPlan &p, hipStream_t s) {
    auto *kernel = p.grid.seg_len <= TR * kLseGroup * Vec<T>::N ? logits_row_lse_kernel<T, TR, 1, Stream>
                                                               : logits_row_lse_kernel<T, TR, kLseRounds, Stream>;
    kernel<<<p.grid.blocks(), kRowThreads, 0, s>>>(
        static_cast<const T *>(d->logits), d->V, p.grid, d->target, p.row_max, p.row_sum, p.z_target,
        p.done);
}
template <typename T>
static void launch_row_lse(const spo_pg_desc *d, const LogitsFwdPlan &p, hipStream_t s) {
    if (p.grid.per_wg > 1) streams(d) ? launch_row_lse<T, kWave, true>(d, p, s) : launch_row_lse<T, kWave, false>(d, p, s);
    else if (streams(d)) launch_row_lse<T, kRowThreads, true>(d, p, s);
    else launch_row_lse<T, kRowThreads, false>(d, p, s);
}

template <typename T, int TR, bool Stream>
static void launch_row_grad(const spo_pg_desc *d, const RowGrid &grid, const float *lse, const float *g, void *d_logits,
                            hipStream_t s) {
    logits_row_grad_kernel<T, TR, Stream><<<grid.blocks(), kRowThreads, 0, s>>>(
        static_cast<const T *>(d->logits), d->V, grid, d->target, lse, g, static_cast<T *>(d_logits));
}
template <typename T>
static void launch_row_grad(const spo_pg_desc *d, const float *lse, const float *g, void *d_logits, hipStream_t s) {
    const RowGrid grid = row_grid(d, kGradGroup, 1, kGradNarrow);
    if (grid.per_wg > 1) launch_row_grad<T, kWave, false>(d, grid, lse, g, d_logits, s);
    else if (streams(d)) launch_row_grad<T, kRowThreads, true>(d, grid, lse, g, d_logits, s);
    else launch_row_grad<T, kRowThreads, false>(d, grid, lse, g, d_logits, s);
}

int logits_fwd_workspace(const spo_pg_desc *d, size_t *bytes) {
    *bytes = plan_logits_fwd(d, nullptr).bytes;
    return SPO_OK;
}

int logits_fwd(const spo_pg_desc *d, float *loss, float *logp, float *lse, float *stats, void *ws,
               size_t ws_bytes, hipStream_t s) {
    const LogitsFwdPlan p = plan_logits_fwd(d, ws);
    if (ws_bytes < p.bytes) return SPO_EWORKSPACE;
    if (d->T > 0) {
        ScopedKernelTimer timer(kTimeLogitsFwd, s);
        if (d->dtype == SPO_BF16) launch_row_lse<bf16_t>(d, p, s);
        else launch_row_lse<float>(d, p, s);
    }
    const TokenShape tok = token_shape(p.grid.nseg, p.nblk_tok);
    token_loss_kernel<<<tok.blocks, tok.threads, 0, s>>>(
        p.row_max, p.row_sum, p.grid.nseg, tok.ways, d->T, p.z_target, token_inputs(d, 0, d->T), logp, lse, p.partials,
        TokenGrad{}, p.nblk_tok, p.nblk_tok, p.done, loss, stats);
    return launch_status();
}

struct LogitsBwdPlan {
    double *count;
    float *g;
    size_t bytes;
};

static LogitsBwdPlan plan_logits_bwd(const spo_pg_desc *d, void *ws) {
    LogitsBwdPlan p;
    Arena a(ws);
    p.count = a.take<double>(1);
    p.g = a.take<float>(std::max<int64_t>(d->T, 1));
    p.bytes = a.used;
    return p;
}

int logits_bwd_workspace(const spo_pg_desc *d, size_t *bytes) {
    *bytes = plan_logits_bwd(d, nullptr).bytes;
    return SPO_OK;
}

int logits_bwd(const spo_pg_desc *d, const float *logp, const float *lse, float grad_loss, void *d_logits,
               void *ws, size_t ws_bytes, hipStream_t s) {
    if (!d_logits) return SPO_ENULL;
    const LogitsBwdPlan p = plan_logits_bwd(d, ws);
    if (ws_bytes < p.bytes) return SPO_EWORKSPACE;
    if (d->T == 0) return SPO_OK;
    launch_grad_scale(d, logp, d->T, grad_loss, p.count, p.g, s);
    ScopedKernelTimer timer(kTimeLogitsBwd, s);
    if (d->dtype == SPO_BF16) launch_row_grad<bf16_t>(d, lse, p.g, d_logits, s);
    else launch_row_grad<float>(d, lse, p.g, d_logits, s);
    return launch_status();
}

}  // namespace spo
