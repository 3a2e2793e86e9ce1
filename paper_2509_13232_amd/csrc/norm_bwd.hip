// Normalisation of rows, backward (norm.hpp).
#include "gemm_core.hpp"
#include "norm.hpp"

namespace spo {

struct NormGrads {
    const float *mean, *rstd;
    const void *dy;
    int64_t dy_stride;
    void *dx;
    int dx_dtype;
    float *dw_parts, *db_parts;  // a row of partial sums per workgroup (of dy h / 2, of dy), or NULL
    int64_t part_stride;
};

// Those that share a row (L lanes, or with L = 0 the workgroup) take every so-manieth one, and ask for the next before they work on
// the one that they hold.  A thread keeps its columns' sums of dy h and dy over all of its rows, in registers or, where those do
// not suffice (InLds), in LDS; at the end those of a workgroup are added in order.  (h, off and mean_gh are halves here: half_from.)
// (InLds: W = 0, as many wavefronts as the row needs; one workgroup fills a compute unit, and what is asked for ahead would not fit
// its registers.)
template <typename TX, typename TY, int L, int W, int Eights, bool Bias, bool Stream>
__global__ void __launch_bounds__(L ? kThreads : W ? W * kWave : 1024) norm_bwd_kernel(NormArgs a, NormGrads g) {
    constexpr int E = kVector<TX, TY>, NV = Eights * 8 / E, kRows = L ? kThreads / (L ? L : 1) : 1;
    constexpr bool InLds = L == 0 && W == 0, HalfEarly = InLds && sizeof(TX) != sizeof(TY);
    __shared__ float scratch[2][L ? 1 : 3 * (W ? W : 16)];
    extern __shared__ __align__(16) float joined[];  // [2][cols, padded] of each wavefront (L), or of the workgroup (InLds)
    const int TR = L ? L : W ? W * kWave : static_cast<int>(blockDim.x), t = L ? static_cast<int>(threadIdx.x) % L : static_cast<int>(threadIdx.x);
    const int padded = (a.cols + 7) / 8 * 8;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kRows;
    int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + (L ? threadIdx.x / (L ? L : 1) : 0);
    RawE<E, TX> rx[NV], next_x[NV];
    RawE<E, TY> ry[NV], next_y[NV];
    float mu = 0.0f, rs = 0.0f, next_mu = 0.0f, next_rs = 0.0f;
    const auto get = [&](int64_t at, RawE<E, TX> (&x)[NV], RawE<E, TY> (&y)[NV], float &m, float &r) {
        const bool live = at < a.rows, past = at < a.rows - 1 && a.cols >= E;
        if (L == 0 && !live) return;
        const TX *px = static_cast<const TX *>(a.x) + at * a.x_stride;
        const TY *py = static_cast<const TY *>(g.dy) + at * g.dy_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TR + t) * E, some = live ? within_e<E>(c, a.cols) : 0;
            fetch<E, Stream>(x[k], px + c, some, past);
            fetch<E, Stream>(y[k], py + c, some, past);
        }
        m = a.layer && live ? g.mean[at] : 0.0f;
        if (HalfEarly) m = first_lane<kWave>(0.5f * m);  // (into a scalar register: 12288 columns from fp32 to bf16 297 us, so 287)
        r = live ? g.rstd[at] : 0.0f;
    };
    get(row, rx, ry, mu, rs);
    float w[NV][E], dw[NV][E], db[NV][E];
    if constexpr (InLds) {
        for (int c = static_cast<int>(threadIdx.x); c < 2 * padded; c += static_cast<int>(blockDim.x)) joined[c] = 0.0f;
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * TR + t) * E;
        if (a.w && !InLds) load_weights(w[k], a.w, a.w_dtype, c, within_e<E>(c, a.cols));
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (!a.w || InLds) w[k][i] = 1.0f;
            dw[k][i] = db[k][i] = 0.0f;
        }
    }
    const float inv_n = 1.0f / static_cast<float>(a.cols);
    int turn = 0;
    // whole wavefronts, and with L = 0 whole workgroups
    for (; row - (L ? threadIdx.x % kWave / (L ? L : 1) : 0) < a.rows; row += stride) {
        if constexpr (!InLds) get(row + stride, next_x, next_y, next_mu, next_rs);
        const bool live = row < a.rows;
        const float half_mu = HalfEarly ? mu : 0.5f * mu;
        float s[3] = {0.0f, 0.0f, 0.0f};  // of g h / 2, g, h / 2
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TR + t) * E, some = live ? within_e<E>(c, a.cols) : 0;
            float h[E], d[E];
            if constexpr (InLds) {  // (registers are short: masks cost less than a branch)
                floats_some(rx[k], h, some);
                floats_some(ry[k], d, some);
                if (a.w) load_weights(w[k], a.w, a.w_dtype, c, some);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float hi = i < some ? half_from(h[i], half_mu) * rs : 0.0f, gi = d[i] * w[k][i];
                    s[0] += gi * hi;
                    s[1] += gi;
                    s[2] += hi;
                }
            } else {
                floats(rx[k], h);
                floats(ry[k], d);
#pragma unroll
                for (int i = 0; i < E; ++i) h[i] = half_from(h[i], half_mu) * rs, d[i] *= w[k][i];
                if (__any(some < E))  // (few wavefronts)
#pragma unroll
                    for (int i = 0; i < E; ++i) h[i] = i < some ? h[i] : 0.0f, d[i] = i < some ? d[i] : 0.0f;
#pragma unroll
                for (int i = 0; i < E; ++i) s[0] += d[i] * h[i];
                if (a.layer)
#pragma unroll
                    for (int i = 0; i < E; ++i) s[1] += d[i], s[2] += h[i];
            }
        }
        float off = 0.0f, mean_g = 0.0f, mean_gh;
        if (a.layer) {
            row_sums<L, W, 3, float>(s, scratch[turn]);
            off = s[2] * inv_n;
            mean_g = s[1] * inv_n;
            mean_gh = s[0] * inv_n - off * mean_g;
        } else {
            float one[1] = {s[0]};
            row_sums<L, W, 1, float>(one, scratch[turn]);
            mean_gh = one[0] * inv_n;
        }
        turn ^= 1;
        const float of_g = -rs * mean_g, of_h = -4.0f * (rs * mean_gh);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TR + t) * E, some = live ? within_e<E>(c, a.cols) : 0;
            float h[E], d[E], dx[E], dyh[E];
            floats(rx[k], h);
            floats(ry[k], d);
            if (L && __any(some < E))  // (a row that is not there adds nothing; what lies behind the columns goes nowhere)
#pragma unroll
                for (int i = 0; i < E; ++i) h[i] = i < some ? h[i] : 0.0f, d[i] = i < some ? d[i] : 0.0f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float hi = fmaf(half_from(h[i], half_mu), rs, -off);
                dx[i] = fmaf(hi, of_h, fmaf(d[i] * w[k][i], rs, of_g));
                if constexpr (InLds) {
                    dyh[i] = d[i] * hi;
                } else {
                    dw[k][i] += d[i] * hi;
                    if (Bias) db[k][i] += d[i];
                }
            }
            if constexpr (InLds)
                if (some) {
#pragma unroll
                    for (int h4 = 0; h4 < E; h4 += 4) {
                        float4 *pw = reinterpret_cast<float4 *>(joined + c + h4), *pb = reinterpret_cast<float4 *>(joined + padded + c + h4);
                        float4 q = *pw;
                        q.x += dyh[h4], q.y += dyh[h4 + 1], q.z += dyh[h4 + 2], q.w += dyh[h4 + 3];
                        *pw = q;
                        if (Bias) {
                            q = *pb;
                            q.x += d[h4], q.y += d[h4 + 1], q.z += d[h4 + 2], q.w += d[h4 + 3];
                            *pb = q;
                        }
                    }
                }
            if (some && g.dx) {
                const int64_t at = row * a.cols + c;
                if (g.dx_dtype == SPO_FP32) store_e<Stream && E == 4>(static_cast<float *>(g.dx) + at, dx, some);
                else store_e<Stream>(static_cast<bf16_t *>(g.dx) + at, dx, some);
            }
            if constexpr (!InLds) rx[k] = next_x[k], ry[k] = next_y[k];
        }
        if constexpr (InLds) get(row + stride, rx, ry, mu, rs);
        else mu = next_mu, rs = next_rs;
    }
    if (!g.dw_parts && !g.db_parts) return;
    const int64_t part = blockIdx.x * g.part_stride;
    if constexpr (L == 0 && !InLds) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TR + t) * E, some = within_e<E>(c, a.cols);
            if (some && g.dw_parts) store_e<false>(g.dw_parts + part + c, dw[k], some);
            if (some && Bias) store_e<false>(g.db_parts + part + c, db[k], some);
        }
    } else {
        constexpr int kSets = L ? kThreads / kWave : 1;
        if constexpr (L) {
            const int wave = threadIdx.x / kWave;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
#pragma unroll
                for (int i = 0; i < E; ++i)
#pragma unroll
                    for (int o = L; o < kWave; o <<= 1) {
                        dw[k][i] += __shfl_xor(dw[k][i], o, kWave);
                        if (Bias) db[k][i] += __shfl_xor(db[k][i], o, kWave);
                    }
                const int c = (k * TR + t) * E, some = threadIdx.x % kWave < L ? within_e<E>(c, a.cols) : 0;
                store_e<false>(joined + wave * 2 * padded + c, dw[k], some);
                if (Bias) store_e<false>(joined + (wave * 2 + 1) * padded + c, db[k], some);
            }
        }
        __syncthreads();
        for (int c = static_cast<int>(threadIdx.x); c < a.cols; c += static_cast<int>(blockDim.x)) {
            float sw = 0.0f, sb = 0.0f;
#pragma unroll
            for (int i = 0; i < kSets; ++i) {
                sw += joined[i * 2 * padded + c];
                if (Bias) sb += joined[(i * 2 + 1) * padded + c];
            }
            if (g.dw_parts) g.dw_parts[part + c] = sw;
            if (Bias) g.db_parts[part + c] = sb;
        }
    }
}

// Rows that the registers of a workgroup do not hold beside the sums of their columns: the sums of a row first (13421 rows of 20000 in
// bf16: 2.9 TB/s of what is read once and written once; both passes read at the rate of a copy) ...
__global__ void __launch_bounds__(1024) norm_bwd_sums_kernel(NormArgs a, NormGrads g, int x_dtype, int dy_dtype, float *__restrict__ sums) {
    __shared__ float scratch[3 * 1024 / kWave];
    const int64_t row = flat_block();
    if (row >= a.rows) return;
    const float half_mu = a.layer ? 0.5f * g.mean[row] : 0.0f, rs = g.rstd[row];
    float s[3] = {0.0f, 0.0f, 0.0f};
    for (int c = static_cast<int>(threadIdx.x) * 8; c < a.cols; c += 8 * 1024) {
        const int some = within(c, a.cols);
        float h[8], d[8], w[8];
        load_typed(h, a.x, x_dtype, row * a.x_stride + c, some);
        load_typed(d, g.dy, dy_dtype, row * g.dy_stride + c, some);
        if (a.w) load_typed(w, a.w, a.w_dtype, c, some);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float hi = i < some ? half_from(h[i], half_mu) * rs : 0.0f, gi = a.w ? d[i] * w[i] : d[i];
            s[0] += hi;
            s[1] += gi;
            s[2] += gi * hi;
        }
    }
    lane_sums<kWave>(s);
    join_waves<16>(s, scratch);
    if (threadIdx.x == 0) {
        const float inv_n = 1.0f / static_cast<float>(a.cols);
        const float off = a.layer ? s[0] * inv_n : 0.0f, mean_g = a.layer ? s[1] * inv_n : 0.0f;
        sums[row * 3] = off;
        sums[row * 3 + 1] = mean_g;
        sums[row * 3 + 2] = s[2] * inv_n - off * mean_g;
    }
}
// ... then 2048 columns of every gridDim.y-th row per workgroup.
__global__ void __launch_bounds__(256) norm_bwd_cols_kernel(NormArgs a, NormGrads g, int x_dtype, int dy_dtype, const float *__restrict__ sums) {
    const int c = (static_cast<int>(blockIdx.x) * 256 + static_cast<int>(threadIdx.x)) * 8, some = within(c, a.cols);
    if (some == 0) return;
    float w[8], dw[8], db[8];
    if (a.w) load_typed(w, a.w, a.w_dtype, c, some);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (!a.w) w[i] = 1.0f;
        dw[i] = db[i] = 0.0f;
    }
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float half_mu = a.layer ? 0.5f * g.mean[row] : 0.0f, rs = g.rstd[row];
        const float off = sums[row * 3], mean_g = sums[row * 3 + 1], mean_gh = sums[row * 3 + 2];
        float h[8], d[8], dx[8];
        load_typed(h, a.x, x_dtype, row * a.x_stride + c, some);
        load_typed(d, g.dy, dy_dtype, row * g.dy_stride + c, some);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float hi = half_from(h[i], half_mu) * rs - off;
            dx[i] = rs * (d[i] * w[i] - mean_g - 4.0f * hi * mean_gh);
            dw[i] += d[i] * hi;
            db[i] += d[i];
        }
        if (g.dx) store_typed(g.dx, g.dx_dtype, row * a.cols + c, dx, some);
    }
    const int64_t at = static_cast<int64_t>(blockIdx.y) * g.part_stride + c;
    if (g.dw_parts) store_some(g.dw_parts + at, dw, some);
    if (g.db_parts) store_some(g.db_parts + at, db, some);
}

// Column sums of the partial rows: 64 columns per workgroup, four to a thread, 64 shares of the rows joined in a fixed order.
__global__ void __launch_bounds__(1024) norm_join_kernel(const float *__restrict__ dw_parts, const float *__restrict__ db_parts, int64_t part_stride, int parts,
                                                         int cols, void *__restrict__ dw, void *__restrict__ db, int dtype, int add) {
    __shared__ float sums[1024 / kWave][64];
    const float *of = blockIdx.y ? db_parts : dw_parts;
    void *to = blockIdx.y ? db : dw;
    if (!to) return;
    const int share = threadIdx.x / 16, four = threadIdx.x % 16 * 4;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = share; p < parts; p += 64) {  // (rows are padded to whole workgroups)
        const float4 v = *reinterpret_cast<const float4 *>(of + p * part_stride + blockIdx.x * 64 + four);
        s[0] += v.x, s[1] += v.y, s[2] += v.z, s[3] += v.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] += __shfl_xor(s[i], 16, kWave);
        s[i] += __shfl_xor(s[i], 32, kWave);
        if (threadIdx.x % kWave < 16) sums[threadIdx.x / kWave][four + i] = s[i];
    }
    __syncthreads();
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || c >= cols) return;
    float total = 0.0f;
    for (int i = 0; i < 1024 / kWave; ++i) total += sums[i][threadIdx.x];
    if (!blockIdx.y) total *= 2.0f;  // (of halves of h)
    if (dtype == SPO_FP32) static_cast<float *>(to)[c] = add ? static_cast<float *>(to)[c] + total : total;
    else static_cast<bf16_t *>(to)[c] = f32_to_bf16(total);
}

// ------------------------------------------------------------------------------------------------------------ host

// How many workgroups the backward has: as many as the chip holds at once, in whole numbers per compute unit (on one card, one, two and
// three of 8 wavefronts per unit: 65536 rows of 4096 in bf16 283, 271 and 311 us; 284780, rms, 1216 to 1258, 1251 to 1277 and
// 1327 to 1332).  Few rows: one to each group of lanes (713 rows of 1001: 5.9 us, two 7.4).
static int bwd_parts(int64_t rows, int64_t cols) {
    const int64_t eights = ceil_div(cols, 8);
    int64_t most, each = 1;
    if (cols > kRegisterCols) {
        most = kColumnParts;
    } else if (eights <= 2 * kWave) {
        most = eights <= kWave ? 4 * 256 : 2 * 256;
        each = kThreads / (eights > kWave ? kWave : lanes_of(eights));
    } else {
        most = eights <= 256 ? 4 * 256 : eights <= 512 ? 2 * 256 : 256;
    }
    return static_cast<int>(std::min<int64_t>(most, ceil_div(rows, each)));
}

constexpr int kLdsSums = 2 * kRegisterCols * static_cast<int>(sizeof(float));

template <typename TX, typename TY, int L, int W, int Eights, bool Bias>
static int bwd_rows(const NormArgs &a, const NormGrads &g, int parts, hipStream_t s) {
    constexpr bool InLds = L == 0 && W == 0;
    auto *kernel = past_cache<TX, TY>(a.rows, a.cols) ? norm_bwd_kernel<TX, TY, L, W, Eights, Bias, true> : norm_bwd_kernel<TX, TY, L, W, Eights, Bias, false>;
    const int padded = (a.cols + 7) / 8 * 8;
    const int lds = (InLds ? 2 : L ? 2 * kThreads / kWave : 0) * padded * static_cast<int>(sizeof(float));
    if (InLds)
        if (int rc = allow_lds(kernel, kLdsSums)) return rc;
    kernel<<<parts, L ? kThreads : W ? W * kWave : fours_of(ceil_div(a.cols, 8), Eights) * kWave, lds, s>>>(a, g);
    return SPO_OK;
}
template <typename TX, typename TY, bool Bias>
static int bwd_typed(const NormArgs &a, const NormGrads &g, int parts, hipStream_t s) {
    const int64_t eights = ceil_div(a.cols, 8);
    if (eights <= kWave)
        switch (lanes_of(eights)) {
            case 4: return bwd_rows<TX, TY, 4, 0, 1, Bias>(a, g, parts, s);
            case 8: return bwd_rows<TX, TY, 8, 0, 1, Bias>(a, g, parts, s);
            case 16: return bwd_rows<TX, TY, 16, 0, 1, Bias>(a, g, parts, s);
            case 32: return bwd_rows<TX, TY, 32, 0, 1, Bias>(a, g, parts, s);
            default: return bwd_rows<TX, TY, kWave, 0, 1, Bias>(a, g, parts, s);
        }
    if (eights <= 2 * kWave) return bwd_rows<TX, TY, kWave, 0, 2, Bias>(a, g, parts, s);
    if (eights <= 256) return bwd_rows<TX, TY, 0, 4, 1, Bias>(a, g, parts, s);
    if (eights <= 512) return bwd_rows<TX, TY, 0, 8, 1, Bias>(a, g, parts, s);
    if (eights <= 768) return bwd_rows<TX, TY, 0, 12, 1, Bias>(a, g, parts, s);
    if (eights <= 1024) return bwd_rows<TX, TY, 0, 16, 1, Bias>(a, g, parts, s);
    return bwd_rows<TX, TY, 0, 0, 2, Bias>(a, g, parts, s);
}
template <typename TX, typename TY>
static int bwd_typed(const NormArgs &a, const NormGrads &g, int parts, hipStream_t s) {
    return g.db_parts ? bwd_typed<TX, TY, true>(a, g, parts, s) : bwd_typed<TX, TY, false>(a, g, parts, s);
}

struct NormPlan {
    float *dw_parts, *db_parts, *sums;
    int64_t part_stride;
    size_t bytes;
};
// The size does not shrink with rows or cols: as many partial rows as any number of columns has with these rows.
static NormPlan plan_norm(int64_t rows, int64_t cols, void *ws) {
    NormPlan p{};
    Arena a(ws);
    p.part_stride = ceil_div(cols, 64) * 64;
    const size_t room = static_cast<size_t>(std::min<int64_t>(kParts, std::max<int64_t>(rows, 1))) * p.part_stride;
    p.dw_parts = a.take<float>(room);
    p.db_parts = a.take<float>(room);
    if (cols > kRegisterCols) p.sums = a.take<float>(static_cast<size_t>(rows) * 3);
    p.bytes = std::max<size_t>(a.used, 256);
    return p;
}

}  // namespace spo

using namespace spo;

extern "C" size_t spo_norm_bwd_workspace_bytes(const spo_norm_desc *d) {
    return validate(d) == SPO_OK ? plan_norm(d->rows, d->cols, nullptr).bytes : 0;
}

extern "C" int spo_norm_bwd(const spo_norm_desc *d, const float *mean, const float *rstd, const void *dy, int dy_dtype, int64_t dy_stride,
                            void *dx, int dx_dtype, void *d_weight, void *d_bias, int d_w_dtype, int accumulate, void *ws, size_t ws_bytes,
                            spo_stream_t stream) {
    if (int rc = validate(d)) return rc;
    if (!type_ok(dy_dtype) || (dx && !type_ok(dx_dtype)) || ((d_weight || d_bias) && !type_ok(d_w_dtype))) return SPO_EINVAL;
    if (accumulate && (d_weight || d_bias) && d_w_dtype != SPO_FP32) return SPO_EINVAL;
    if (dy_stride && dy_stride < d->cols) return SPO_EINVAL;
    if (dy_stride > int64_t(1) << 40) return SPO_ERANGE;
    if (d->rows && (!d->x || !dy || !rstd || (d->kind == SPO_NORM_LAYER && !mean))) return SPO_ENULL;
    if (!aligned_to(dy, dy_dtype) || (dx && !aligned_to(dx, dx_dtype)) || !aligned_to(d_weight, d_w_dtype) || !aligned_to(d_bias, d_w_dtype)) return SPO_EINVAL;
    if (!dx && !d_weight && !d_bias) return SPO_OK;
    if (!ws) return SPO_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(ws) % 256) return SPO_EINVAL;
    const NormPlan p = plan_norm(d->rows, d->cols, ws);
    if (ws_bytes < p.bytes) return SPO_EWORKSPACE;
    const NormArgs a = args_of(d);
    const NormGrads g{mean, rstd, dy, dy_stride ? dy_stride : d->cols, dx, dx_dtype, d_weight ? p.dw_parts : nullptr, d_bias ? p.db_parts : nullptr, p.part_stride};
    const hipStream_t s = as_stream(stream);
    const int parts = bwd_parts(d->rows, d->cols);
    if (d->rows && d->cols <= kRegisterCols) {
        const bool x32 = d->x_dtype == SPO_FP32, y32 = dy_dtype == SPO_FP32;
        int rc;
        if (x32 && y32) rc = bwd_typed<float, float>(a, g, parts, s);
        else if (x32) rc = bwd_typed<float, bf16_t>(a, g, parts, s);
        else if (y32) rc = bwd_typed<bf16_t, float>(a, g, parts, s);
        else rc = bwd_typed<bf16_t, bf16_t>(a, g, parts, s);
        if (rc) return rc;
    } else if (d->rows) {
        norm_bwd_sums_kernel<<<fold_grid(d->rows, 1024), 1024, 0, s>>>(a, g, d->x_dtype, dy_dtype, p.sums);
        norm_bwd_cols_kernel<<<dim3(static_cast<unsigned>(ceil_div(d->cols, 2048)), parts), 256, 0, s>>>(a, g, d->x_dtype, dy_dtype, p.sums);
    }
    if (d_weight || d_bias)  // (no rows: sums of nothing)
        norm_join_kernel<<<dim3(static_cast<unsigned>(ceil_div(d->cols, kWave)), 2), 1024, 0, s>>>(p.dw_parts, p.db_parts, p.part_stride, parts, static_cast<int>(d->cols),
                                                                                               d_weight, d_bias, d_w_dtype, accumulate);
    return launch_status();
}
