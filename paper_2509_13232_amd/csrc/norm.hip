// Normalisation of rows, forward and backward (the hidden states that a head reads, and the way back through them).
//
//   layer: mu = mean x, rstd = (mean (x - mu)^2 + eps)^-1/2, h = (x - mu) rstd;   rms: rstd = (mean x^2 + eps)^-1/2, h = x rstd
//   y = h w + b;  with g = dy w:  dx = rstd (g - mean g - h mean(g h)), rms without the mean of g;  dw = sum dy h,  db = sum dy
//
// A row is held in registers from its one read to its one write: by a wavefront, or by the wavefronts of a workgroup.
// The mean is rounded to fp32; rows far from zero lose digits of x - mu to that, all elements alike, so the sum of what is left
// (x - rounded mu) is taken as well and put right, in the backward from the row itself.
#include <algorithm>
#include <type_traits>

#include "vec8.hpp"

namespace spo {

constexpr int kMostCols = 65536;
constexpr int kParts = 512;        // most workgroups of the backward: each leaves one row of partial sums
constexpr int kColumnParts = 256;   // ... and of the one that takes rows by columns

struct NormArgs {
    const void *x;
    int64_t x_stride, rows;
    int cols, layer, w_dtype;
    const void *w, *b;
    float eps;
};

// Sums over a wavefront by moves between lanes: within rows of 16, then from row to row; the last lane's are everybody's.
template <int M>
__device__ __forceinline__ void wave_sums(float (&v)[M]) {
    const auto step = [&](auto control, auto rows) {
#pragma unroll
        for (int m = 0; m < M; ++m)
            v[m] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v[m]), decltype(control)::value, decltype(rows)::value, 0xf, false));
    };
    typedef std::integral_constant<int, 0xf> All;
    step(std::integral_constant<int, 0x111>{}, All{});  // from one lane below
    step(std::integral_constant<int, 0x112>{}, All{});
    step(std::integral_constant<int, 0x114>{}, All{});
    step(std::integral_constant<int, 0x118>{}, All{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});  // a row's last lane to the next row
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});  // the second row's last lane to the upper half
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v[m]), kWave - 1));
}
template <int M>
__device__ __forceinline__ void wave_sums(double (&v)[M]) {
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = wave_sum(v[m]);
}
// Sums over the TR threads that share a row, in a fixed order; every thread receives them.  TR > 64: all threads of the workgroup
// call this together; scratch holds M numbers per wavefront and is free again after the next such call with another scratch.
template <int TR, int M, typename T>
__device__ __forceinline__ void row_sums(T (&v)[M], T *scratch) {
    wave_sums(v);
    if constexpr (TR > kWave) {
        const int wave = threadIdx.x / kWave;
        if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
            for (int m = 0; m < M; ++m) scratch[wave * M + m] = v[m];
        __syncthreads();
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] = T(0);
        for (int i = 0; i < TR / kWave; ++i)
#pragma unroll
            for (int m = 0; m < M; ++m) v[m] += scratch[i * M + m];
    }
}

constexpr int kFwdThreads = 256;  // of a workgroup, where a wavefront has a row to itself
constexpr int threads_of(int TR) { return TR < kFwdThreads ? kFwdThreads : TR; }
constexpr float kSquaresLow = 1e-30f, kSquaresHigh = 1e38f;  // a variance below, sums of squares above: formed again in 64 bits
// Elements of a vector: 16 bytes of bf16; four where fp32 is among the arrays, so that a wavefront's loads are whole lines
// (17043 rows of 4096 from fp32 to bf16: 81 us with eight neighbours per thread).
template <typename TX, typename TY>
constexpr int kVector = sizeof(TX) == 2 && sizeof(TY) == 2 ? 8 : 4;

// Eights: eight elements per thread times this; the thread's k-th vector begins at column (k * TR + thread) * E.
template <typename TX, typename TY, int TR, int Eights, bool Stream>
__global__ void __launch_bounds__(threads_of(TR)) norm_fwd_kernel(NormArgs a, TY *y, int64_t y_stride, float *__restrict__ mean, float *__restrict__ rstd) {
    constexpr int E = kVector<TX, TY>, NV = Eights * 8 / E;
    constexpr int kWaves = threads_of(TR) / kWave;
    __shared__ double scratch[3][kWaves * 2];
    const int t = threadIdx.x % TR;
    const int64_t row = flat_block() * (threads_of(TR) / TR) + threadIdx.x / TR;
    if (row >= a.rows) return;  // (TR > 64: the workgroup's one row)
    const TX *x = static_cast<const TX *>(a.x) + row * a.x_stride;
    float v[NV][E];
    {
        RawE<E, TX> r[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TR + t) * E;
            fetch<E, Stream>(r[k], x + c, within_e<E>(c, a.cols));
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) floats(r[k], v[k]);
    }
    const float n = static_cast<float>(a.cols);
    float mu = 0.0f;
    if (a.layer) {
        float s[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) s[0] += v[k][i];
        row_sums<TR, 1, float>(s, reinterpret_cast<float *>(scratch[0]));
        mu = s[0] / n;
        if (!(fabsf(s[0]) <= 3e38f)) {  // the sum left fp32's range (or something in the row is not finite)
            double d[1] = {0.0};
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) d[0] += v[k][i];
            row_sums<TR, 1, double>(d, scratch[2]);
            mu = static_cast<float>(d[0] / a.cols);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int some = within_e<E>((k * TR + t) * E, a.cols);
#pragma unroll
            for (int i = 0; i < E; ++i) v[k][i] = i < some ? v[k][i] - mu : 0.0f;
        }
    }
    float s[2] = {0.0f, 0.0f};  // of what is left, and its squares
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < E; ++i) {
            s[0] += v[k][i];
            s[1] += v[k][i] * v[k][i];
        }
    row_sums<TR, 2, float>(s, reinterpret_cast<float *>(scratch[1]));
    const float off = a.layer ? s[0] / n : 0.0f;
    float var = s[1] / n - off * off;
    var = var < 0.0f ? 0.0f : var;
    float rs = 1.0f / sqrtf(var + a.eps);
    if (!(s[1] <= kSquaresHigh && var + a.eps >= kSquaresLow)) {
        double d[1] = {0.0};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < E; ++i) d[0] += static_cast<double>(v[k][i]) * static_cast<double>(v[k][i]);
        row_sums<TR, 1, double>(d, scratch[2]);
        rs = static_cast<float>(1.0 / sqrt(d[0] / a.cols - static_cast<double>(off) * off + a.eps));
    }
    if (t == 0) {
        if (mean && a.layer) mean[row] = mu;
        if (rstd) rstd[row] = rs;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * TR + t) * E, some = within_e<E>(c, a.cols);
        if (some == 0) continue;
#pragma unroll
        for (int i = 0; i < E; ++i) v[k][i] = (v[k][i] - off) * rs;
        float p[E];
        if (a.w) {
            load_weights(p, a.w, a.w_dtype, c, some);
#pragma unroll
            for (int i = 0; i < E; ++i) v[k][i] *= p[i];
        }
        if (a.b) {
            load_weights(p, a.b, a.w_dtype, c, some);
#pragma unroll
            for (int i = 0; i < E; ++i) v[k][i] += p[i];
        }
        store_e<Stream>(y + row * y_stride + c, v[k], some);
    }
}

struct NormGrads {
    const float *mean, *rstd;
    const void *dy;
    int64_t dy_stride;
    void *dx;
    int dx_dtype;
    float *dw_parts, *db_parts;  // a row of partial sums per workgroup, or NULL
    int64_t part_stride;
};

// A group of TR threads takes every so-manieth row; it asks for the next one before it works on the one that it holds.  A thread
// keeps its columns' sums of dy h and dy over all of its rows; wavefronts that have rows to themselves add theirs in order at the end.
constexpr int groups_of(int TR) { return TR == kWave ? 4 : 1; }
template <typename TX, typename TY, int TR, int Eights, bool Bias, bool Stream>
__global__ void __launch_bounds__(TR * groups_of(TR)) norm_bwd_kernel(NormArgs a, NormGrads g) {
    constexpr int E = kVector<TX, TY>, NV = Eights * 8 / E, kGroups = groups_of(TR);
    __shared__ float scratch[2][3 * TR * kGroups / kWave];
    extern __shared__ float joined[];  // [kGroups][2][cols], where a workgroup has several groups
    const int t = threadIdx.x % TR, group = threadIdx.x / TR;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kGroups;
    int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    RawE<E, TX> rx[NV], next_x[NV];
    RawE<E, TY> ry[NV], next_y[NV];
    float mu = 0.0f, rs = 0.0f, next_mu = 0.0f, next_rs = 0.0f;
    const auto get = [&](int64_t at, RawE<E, TX> (&x)[NV], RawE<E, TY> (&y)[NV], float &m, float &r) {
        if (at >= a.rows) return;
        const TX *px = static_cast<const TX *>(a.x) + at * a.x_stride;
        const TY *py = static_cast<const TY *>(g.dy) + at * g.dy_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TR + t) * E, some = within_e<E>(c, a.cols);
            fetch<E, Stream>(x[k], px + c, some);
            fetch<E, Stream>(y[k], py + c, some);
        }
        if (a.layer) m = g.mean[at];
        r = g.rstd[at];
    };
    get(row, rx, ry, mu, rs);
    float w[NV][E], dw[NV][E], db[NV][E];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * TR + t) * E;
        if (a.w) load_weights(w[k], a.w, a.w_dtype, c, within_e<E>(c, a.cols));
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (!a.w) w[k][i] = 1.0f;
            dw[k][i] = db[k][i] = 0.0f;
        }
    }
    const float inv_n = 1.0f / static_cast<float>(a.cols);
    int turn = 0;
    for (; row < a.rows; row += stride) {  // (TR > 64: the same rows for all of the workgroup)
        get(row + stride, next_x, next_y, next_mu, next_rs);
        float s[3] = {0.0f, 0.0f, 0.0f};  // of g h, g, h
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int some = within_e<E>((k * TR + t) * E, a.cols);
            float h[E], d[E];
            floats(rx[k], h);
            floats(ry[k], d);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float hi = i < some ? (h[i] - mu) * rs : 0.0f, gi = d[i] * w[k][i];
                s[0] += gi * hi;
                s[1] += gi;
                s[2] += hi;
            }
        }
        float off = 0.0f, mean_g = 0.0f, mean_gh;
        if (a.layer) {
            row_sums<TR, 3, float>(s, scratch[turn]);
            off = s[2] * inv_n;
            mean_g = s[1] * inv_n;
            mean_gh = s[0] * inv_n - off * mean_g;
        } else {
            float one[1] = {s[0]};
            row_sums<TR, 1, float>(one, scratch[turn]);
            mean_gh = one[0] * inv_n;
        }
        turn ^= 1;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TR + t) * E, some = within_e<E>(c, a.cols);
            float h[E], d[E], dx[E];
            floats(rx[k], h);
            floats(ry[k], d);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float hi = (h[i] - mu) * rs - off;
                dx[i] = rs * (d[i] * w[k][i] - mean_g - hi * mean_gh);
                dw[k][i] += d[i] * hi;
                if (Bias) db[k][i] += d[i];
            }
            if (some && g.dx) {
                const int64_t at = row * a.cols + c;
                if (g.dx_dtype == SPO_FP32) store_e<Stream && E == 4>(static_cast<float *>(g.dx) + at, dx, some);
                else store_e<Stream>(static_cast<bf16_t *>(g.dx) + at, dx, some);
            }
            rx[k] = next_x[k];
            ry[k] = next_y[k];
        }
        mu = next_mu;
        rs = next_rs;
    }
    if (!g.dw_parts && !g.db_parts) return;
    const int64_t part = blockIdx.x * g.part_stride;
    if constexpr (kGroups > 1) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TR + t) * E, some = within_e<E>(c, a.cols);
            store_e<false>(joined + group * 2 * a.cols + c, dw[k], some);
            if (Bias) store_e<false>(joined + (group * 2 + 1) * a.cols + c, db[k], some);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += TR * kGroups) {
            float sw = 0.0f, sb = 0.0f;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                sw += joined[i * 2 * a.cols + c];
                if (Bias) sb += joined[(i * 2 + 1) * a.cols + c];
            }
            if (g.dw_parts) g.dw_parts[part + c] = sw;
            if (Bias) g.db_parts[part + c] = sb;
        }
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * TR + t) * E, some = within_e<E>(c, a.cols);
            if (some && g.dw_parts) store_e<false>(g.dw_parts + part + c, dw[k], some);
            if (some && Bias) store_e<false>(g.db_parts + part + c, db[k], some);
        }
    }
}

// Rows that the registers of a workgroup do not hold beside the sums of their columns: the sums of a row first ...
__global__ void __launch_bounds__(1024) norm_bwd_sums_kernel(NormArgs a, NormGrads g, int x_dtype, int dy_dtype, float *__restrict__ sums) {
    __shared__ float scratch[3 * 1024 / kWave];
    const int64_t row = flat_block();
    if (row >= a.rows) return;
    const float mu = a.layer ? g.mean[row] : 0.0f, rs = g.rstd[row];
    float s[3] = {0.0f, 0.0f, 0.0f};
    for (int c = static_cast<int>(threadIdx.x) * 8; c < a.cols; c += 8 * 1024) {
        const int some = within(c, a.cols);
        float h[8], d[8], w[8];
        load_typed(h, a.x, x_dtype, row * a.x_stride + c, some);
        load_typed(d, g.dy, dy_dtype, row * g.dy_stride + c, some);
        if (a.w) load_typed(w, a.w, a.w_dtype, c, some);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float hi = i < some ? (h[i] - mu) * rs : 0.0f, gi = a.w ? d[i] * w[i] : d[i];
            s[0] += hi;
            s[1] += gi;
            s[2] += gi * hi;
        }
    }
    row_sums<1024, 3, float>(s, scratch);
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
        const float mu = a.layer ? g.mean[row] : 0.0f, rs = g.rstd[row];
        const float off = sums[row * 3], mean_g = sums[row * 3 + 1], mean_gh = sums[row * 3 + 2];
        float h[8], d[8], dx[8];
        load_typed(h, a.x, x_dtype, row * a.x_stride + c, some);
        load_typed(d, g.dy, dy_dtype, row * g.dy_stride + c, some);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float hi = (h[i] - mu) * rs - off;
            dx[i] = rs * (d[i] * w[i] - mean_g - hi * mean_gh);
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
    if (dtype == SPO_FP32) static_cast<float *>(to)[c] = add ? static_cast<float *>(to)[c] + total : total;
    else static_cast<bf16_t *>(to)[c] = f32_to_bf16(total);
}

// ------------------------------------------------------------------------------------------------------------ host

// Arrays that the Infinity Cache does not hold take the non-temporal hint
template <typename TX, typename TY>
static bool past_cache(int64_t rows, int64_t cols) { return rows * cols * static_cast<int64_t>(sizeof(TX) + sizeof(TY)) > kStreamBytes; }

template <typename TX, typename TY, int TR, int Eights>
static void fwd_rows(const NormArgs &a, void *y, int64_t y_stride, float *mean, float *rstd, hipStream_t s) {
    auto *kernel = past_cache<TX, TY>(a.rows, a.cols) ? norm_fwd_kernel<TX, TY, TR, Eights, true> : norm_fwd_kernel<TX, TY, TR, Eights, false>;
    kernel<<<fold_grid(ceil_div(a.rows, threads_of(TR) / TR)), threads_of(TR), 0, s>>>(a, static_cast<TY *>(y), y_stride, mean, rstd);
}
template <typename TX, typename TY>
static void fwd_typed(const NormArgs &a, void *y, int64_t y_stride, float *mean, float *rstd, hipStream_t s) {
    if (a.cols <= 512) fwd_rows<TX, TY, 64, 1>(a, y, y_stride, mean, rstd, s);
    else if (a.cols <= 1024) fwd_rows<TX, TY, 64, 2>(a, y, y_stride, mean, rstd, s);
    else if (a.cols <= 2048) fwd_rows<TX, TY, 256, 1>(a, y, y_stride, mean, rstd, s);
    else if (a.cols <= 4096) fwd_rows<TX, TY, 256, 2>(a, y, y_stride, mean, rstd, s);
    else if (a.cols <= 8192) fwd_rows<TX, TY, 256, 4>(a, y, y_stride, mean, rstd, s);
    else if (a.cols <= 16384) fwd_rows<TX, TY, 1024, 2>(a, y, y_stride, mean, rstd, s);
    else fwd_rows<TX, TY, 1024, 8>(a, y, y_stride, mean, rstd, s);
}

constexpr int kRegisterCols = 16384;  // rows up to here are held by a workgroup of the backward

// How many workgroups there are.  Two per compute unit of 256 threads: 284780 rows of 4096 in bf16 1160 us, with 384 or 640 of them
// in all, which leave units idle in the last round, 1310 and 1328, with 1024 (three of which fit a unit) 1499.  Few rows: one each
// (713 rows of 1001: 7.4 us, two each 8.5, four 11.9).
static int bwd_parts(int64_t rows, int64_t cols) {
    if (cols > kRegisterCols) return static_cast<int>(std::min<int64_t>(kColumnParts, rows));
    const int groups = cols <= 1024 ? groups_of(kWave) : 1;
    return static_cast<int>(std::min<int64_t>(kParts, ceil_div(rows, groups)));
}

template <typename TX, typename TY, int TR, int Eights, bool Bias>
static void bwd_rows(const NormArgs &a, const NormGrads &g, int parts, hipStream_t s) {
    auto *kernel = past_cache<TX, TY>(a.rows, a.cols) ? norm_bwd_kernel<TX, TY, TR, Eights, Bias, true> : norm_bwd_kernel<TX, TY, TR, Eights, Bias, false>;
    const size_t lds = groups_of(TR) > 1 ? sizeof(float) * 2 * groups_of(TR) * a.cols : 0;
    kernel<<<parts, TR * groups_of(TR), lds, s>>>(a, g);
}
template <typename TX, typename TY, bool Bias>
static void bwd_typed(const NormArgs &a, const NormGrads &g, int parts, hipStream_t s) {
    if (a.cols <= 512) bwd_rows<TX, TY, 64, 1, Bias>(a, g, parts, s);
    else if (a.cols <= 1024) bwd_rows<TX, TY, 64, 2, Bias>(a, g, parts, s);
    else if (a.cols <= 2048) bwd_rows<TX, TY, 256, 1, Bias>(a, g, parts, s);
    else if (a.cols <= 4096) bwd_rows<TX, TY, 256, 2, Bias>(a, g, parts, s);
    else if (a.cols <= 8192) bwd_rows<TX, TY, 512, 2, Bias>(a, g, parts, s);
    else bwd_rows<TX, TY, 1024, 2, Bias>(a, g, parts, s);
}
template <typename TX, typename TY>
static void bwd_typed(const NormArgs &a, const NormGrads &g, int parts, hipStream_t s) {
    if (g.db_parts) bwd_typed<TX, TY, true>(a, g, parts, s);
    else bwd_typed<TX, TY, false>(a, g, parts, s);
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

static bool type_ok(int t) { return t == SPO_FP32 || t == SPO_BF16; }
static bool aligned_to(const void *p, int dtype) { return reinterpret_cast<uintptr_t>(p) % (dtype == SPO_FP32 ? 4 : 2) == 0; }

static int validate(const spo_norm_desc *d) {
    if (!d) return SPO_ENULL;
    if (d->struct_size != sizeof(spo_norm_desc)) return SPO_EINVAL;
    if (d->kind != SPO_NORM_LAYER && d->kind != SPO_NORM_RMS) return SPO_EINVAL;
    if (!type_ok(d->x_dtype) || !type_ok(d->y_dtype) || !type_ok(d->w_dtype)) return SPO_EINVAL;
    if (d->rows < 0 || d->cols < 1 || !(d->eps >= 0.0f)) return SPO_EINVAL;
    if (d->x_stride && d->x_stride < d->cols) return SPO_EINVAL;
    if (d->rows >= int64_t(1) << 31 || d->cols > kMostCols || d->x_stride > int64_t(1) << 40) return SPO_ERANGE;
    if (!aligned_to(d->x, d->x_dtype) || !aligned_to(d->weight, d->w_dtype) || !aligned_to(d->bias, d->w_dtype)) return SPO_EINVAL;
    return SPO_OK;
}
static NormArgs args_of(const spo_norm_desc *d) {
    return NormArgs{d->x, d->x_stride ? d->x_stride : d->cols, d->rows, static_cast<int>(d->cols), d->kind == SPO_NORM_LAYER, d->w_dtype,
                    d->weight, d->bias, d->eps};
}

extern "C" int spo_norm_fwd(const spo_norm_desc *d, void *y, int64_t y_stride, float *mean, float *rstd, spo_stream_t stream) {
    if (int rc = validate(d)) return rc;
    if (y_stride && y_stride < d->cols) return SPO_EINVAL;
    if (y_stride > int64_t(1) << 40) return SPO_ERANGE;
    if (d->rows == 0) return SPO_OK;
    if (!d->x || !y) return SPO_ENULL;
    if (!aligned_to(y, d->y_dtype)) return SPO_EINVAL;
    const NormArgs a = args_of(d);
    const int64_t ys = y_stride ? y_stride : d->cols;
    const hipStream_t s = as_stream(stream);
    const bool x32 = d->x_dtype == SPO_FP32, y32 = d->y_dtype == SPO_FP32;
    if (x32 && y32) fwd_typed<float, float>(a, y, ys, mean, rstd, s);
    else if (x32) fwd_typed<float, bf16_t>(a, y, ys, mean, rstd, s);
    else if (y32) fwd_typed<bf16_t, float>(a, y, ys, mean, rstd, s);
    else fwd_typed<bf16_t, bf16_t>(a, y, ys, mean, rstd, s);
    return launch_status();
}

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
        if (x32 && y32) bwd_typed<float, float>(a, g, parts, s);
        else if (x32) bwd_typed<float, bf16_t>(a, g, parts, s);
        else if (y32) bwd_typed<bf16_t, float>(a, g, parts, s);
        else bwd_typed<bf16_t, bf16_t>(a, g, parts, s);
    } else if (d->rows) {
        norm_bwd_sums_kernel<<<fold_grid(d->rows), 1024, 0, s>>>(a, g, d->x_dtype, dy_dtype, p.sums);
        norm_bwd_cols_kernel<<<dim3(static_cast<unsigned>(ceil_div(d->cols, 2048)), parts), 256, 0, s>>>(a, g, d->x_dtype, dy_dtype, p.sums);
    }
    if (d_weight || d_bias)  // (no rows: sums of nothing)
        norm_join_kernel<<<dim3(static_cast<unsigned>(ceil_div(d->cols, kWave)), 2), 1024, 0, s>>>(p.dw_parts, p.db_parts, p.part_stride, parts, static_cast<int>(d->cols),
                                                                                               d_weight, d_bias, d_w_dtype, accumulate);
    return launch_status();
}
