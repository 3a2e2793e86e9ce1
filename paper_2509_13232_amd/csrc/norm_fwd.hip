// Normalisation of rows, forward (norm.hpp).
#include "norm.hpp"

namespace spo {

// Those that share a row (L lanes, or with L = 0 the workgroup) hold R rows: two side by side where their registers suffice and rows
// are many; weight and bias are read once for both, and their sums cross the lanes together.  One row and two, layer and rms: in bf16
// 131072 rows of 2048 227 -> 181 and 196 -> 169 us, 1342177 of 200 279 -> 211 and 234 -> 184, 65536 of 4096 192 -> 185 and 171 -> 177, 268435
// of 1000 201 and 190 -> 197; in fp32, whose wavefronts hold half as much, 32768 of 4096 186 -> 179 and 177, 65536 of 2048 184 -> 181 and
// 169 -> 178, 671088 of 200 215 -> 222 and 207 -> 226.  713 rows of 1001, which are there at once: 4.2 -> 5.2.
// Eights: eight elements per thread times this.  The k-th vector of the t-th of TR threads begins at column (k * TR + t) * E.
// Instructions count beside the bytes: with divisions, masks for all and an epilogue of four instructions per element, 262144 rows of
// 1024 took 188 us instead of 176, 131072 of 2048 210 instead of 185.  Registers, too, which the path of rows in 64 bits takes more of
// than the others: without the bounds on scalar ones 131072 rows of 2048 in bf16, rms, took 177 us instead of 168, 1342177 of 200
// 194 instead of 187; without those on vector ones 345476 of 777 234 instead of 220.  (fp32 needs more of these and does not gain.)
template <typename TX, typename TY, int L, int Eights, int R>
constexpr int kFwdWaves = R == 1 || kVector<TX, TY> == 4 ? 4 : Eights == 1 ? 8 : L ? 6 : 5;  // per SIMD, at least
template <typename TX, typename TY, int L, int W, int Eights, int R, bool Stream>
__global__ void __attribute__((amdgpu_num_sgpr(80))) __launch_bounds__(L ? kThreads : W * kWave, (kFwdWaves<TX, TY, L, Eights, R>))
    norm_fwd_kernel(NormArgs a, TY *y, int64_t y_stride, float *__restrict__ mean, float *__restrict__ rstd, int64_t apart) {
    constexpr int E = kVector<TX, TY>, NV = Eights * 8 / E, kRows = L ? kThreads / (L ? L : 1) : 1;
    __shared__ float scratch[2][L ? 1 : 2 * R * W];
    __shared__ double wide[R][L ? 1 : 2 * W];
    constexpr int TR = L ? L : W * kWave;
    const int t = L ? static_cast<int>(threadIdx.x) % L : static_cast<int>(threadIdx.x);
    const int64_t first = flat_block() * kRows + (L ? threadIdx.x / (L ? L : 1) : 0);
    if (L == 0 && first >= a.rows) return;
    const auto row_of = [&](int r) { return first + r * apart; };
    const auto some_of = [&](int r, int k) { return row_of(r) < a.rows ? within_e<E>((k * TR + t) * E, a.cols) : 0; };
    const auto past_of = [&](int r) { return row_of(r) < a.rows - 1 && a.cols >= E; };  // (the next row's elements may be read)
    const auto x_of = [&](int r) { return static_cast<const TX *>(a.x) + row_of(r) * a.x_stride; };
    float v[R][NV][E], base[R];
    // x - base
    const auto differences = [&](int r, const RawE<E, TX> (&raw)[NV]) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int some = some_of(r, k);
            floats(raw[k], v[r][k]);
#pragma unroll
            for (int i = 0; i < E; ++i) v[r][k][i] -= base[r];
            if (__any(some < E))  // (few wavefronts)
#pragma unroll
                for (int i = 0; i < E; ++i) v[r][k][i] = i < some ? v[r][k][i] : 0.0f;
        }
    };
    {
        RawE<E, TX> raw[R][NV], head[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int k = 0; k < NV; ++k) fetch<E, Stream>(raw[r][k], x_of(r) + (k * TR + t) * E, some_of(r, k), past_of(r));
            if (L == 0 && a.layer) fetch<E, false>(head[r], x_of(r), row_of(r) < a.rows ? within_e<E>(0, a.cols) : 0, past_of(r));
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            base[r] = 0.0f;
            if (a.layer) {
                const int some = row_of(r) < a.rows ? within_e<E>(0, a.cols) : 0;
                const float share = some == E ? 1.0f / E : __builtin_amdgcn_rcpf(static_cast<float>(max(some, 1)));  // (any pivot will do)
                float f[E];
                floats_some(L ? raw[r][0] : head[r], f, some);
#pragma unroll
                for (int i = 0; i < E; ++i) base[r] += f[i] * share;
                if constexpr (L) base[r] = first_lane<L>(base[r]);
            }
            differences(r, raw[r]);
        }
    }
    float off[R], var[R], squares[R], rs[R];
    const auto sum_up = [&](float *where) {
        float s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            s[2 * r] = s[2 * r + 1] = 0.0f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    s[2 * r] += v[r][k][i];
                    s[2 * r + 1] += v[r][k][i] * v[r][k][i];
                }
        }
        row_sums<L, W, 2 * R, float>(s, where);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            off[r] = a.layer ? s[2 * r] * a.inv_n : 0.0f;
            squares[r] = s[2 * r + 1];
            var[r] = squares[r] * a.inv_n - off[r] * off[r];
            var[r] = var[r] < 0.0f ? 0.0f : var[r];
        }
    };
    sum_up(scratch[0]);
    bool far = false;
#pragma unroll
    for (int r = 0; r < R; ++r) far |= off[r] * off[r] > 4.0f * var[r];
    if (any_row<L>(far)) {  // such rows about their mean; the others of the wavefront get what they had
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (off[r] * off[r] > 4.0f * var[r]) base[r] += off[r];
            RawE<E, TX> raw[NV];
#pragma unroll
            for (int k = 0; k < NV; ++k) fetch<E, false>(raw[k], x_of(r) + (k * TR + t) * E, some_of(r, k), past_of(r));
            differences(r, raw);
        }
        sum_up(scratch[1]);
    }
    // Squares or differences that left fp32's range, where the comparison above says nothing, or so small a variance
    bool odd[R], any_odd = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        rs[r] = __builtin_amdgcn_rsqf(var[r] + a.eps);  // (off by a place at most)
        odd[r] = !(squares[r] <= kSquaresHigh && var[r] + a.eps >= kSquaresLow);
        any_odd |= odd[r];
    }
    if (any_row<L>(any_odd)) {
        // Such rows once more from memory, in 64 bits, element by element; the others of the wavefront along with them, as below.  The
        // pivot lies within sqrt(cols / E) <= 128 deviations of the mean, as the mean of E of the row's elements does: one exchange keeps all
        // digits that matter, 2^-53 128^2 being 2e-12.
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool there = row_of(r) < a.rows;
            const TX *const x = x_of(r);
            double d[2] = {0.0, 0.0};
            const double pivot = __builtin_amdgcn_fmed3f(base[r], -kLargest, kLargest);  // (a row that holds an infinity has no finite sum either way)
            if (there && odd[r])
#pragma unroll 1
                for (int c = t; c < a.cols; c += TR) {
                    const double from_pivot = static_cast<double>(Vec<TX>::get(x + c)) - pivot;
                    d[0] += from_pivot;
                    d[1] = fma(from_pivot, from_pivot, d[1]);
                }
            row_sums<L, W, 2, double>(d, wide[r]);
            if (!there) continue;
            // (true divisions: of equal elements beside the pivot they give no variance at all)
            const double o = a.layer ? d[0] / a.cols : 0.0, mu = pivot + o, spread = d[1] / a.cols - o * o, gain = 1.0 / sqrt((spread < 0.0 ? 0.0 : spread) + a.eps);
            if (t == 0 && mean && a.layer) mean[row_of(r)] = odd[r] ? static_cast<float>(mu) : base[r] + off[r];
            if (t == 0 && rstd) rstd[row_of(r)] = odd[r] ? static_cast<float>(gain) : rs[r];
#pragma unroll 1
            for (int c = t; c < a.cols; c += TR) {
                const float f = Vec<TX>::get(x + c);
                const float h = odd[r] ? static_cast<float>((static_cast<double>(f) - mu) * gain) : fmaf(f - base[r], rs[r], -off[r] * rs[r]);
                store_one(y + row_of(r) * y_stride + c, fmaf(h, a.w ? load_weight(a.w, a.w_dtype, c) : 1.0f, a.b ? load_weight(a.b, a.w_dtype, c) : 0.0f));
            }
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (t == 0 && row_of(r) < a.rows) {
            if (mean && a.layer) mean[row_of(r)] = base[r] + off[r];
            if (rstd) rstd[row_of(r)] = rs[r];
        }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * TR + t) * E, inside = within_e<E>(c, a.cols);
        float w[E], b[E];
#pragma unroll
        for (int i = 0; i < E; ++i) w[i] = 1.0f, b[i] = 0.0f;
        if (a.w) load_weights(w, a.w, a.w_dtype, c, inside);
        if (a.b) load_weights(b, a.b, a.w_dtype, c, inside);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int some = some_of(r, k);
            if (some == 0) continue;
            const float shift = -off[r] * rs[r];  // (of two deviations at most, so that its rounding is small beside h's bound)
#pragma unroll
            for (int i = 0; i < E; ++i) v[r][k][i] = fmaf(fmaf(v[r][k][i], rs[r], shift), w[i], b[i]);
            store_e<Stream>(y + row_of(r) * y_stride + c, v[r][k], some);
        }
    }
}

// ------------------------------------------------------------------------------------------------------------ host

template <typename TX, typename TY, int L, int W, int Eights, int R, bool Stream>
static void fwd_launch(const NormArgs &a, void *y, int64_t y_stride, float *mean, float *rstd, hipStream_t s) {
    constexpr int kRows = L ? kThreads / (L ? L : 1) : 1;
    const dim3 grid = fold_grid(ceil_div(ceil_div(a.rows, kRows), R), L ? kThreads : W * kWave);
    norm_fwd_kernel<TX, TY, L, W, Eights, R, Stream><<<grid, L ? kThreads : W * kWave, 0, s>>>(a, static_cast<TY *>(y), y_stride, mean, rstd,
                                                                                          static_cast<int64_t>(grid.x) * grid.y * kRows);
}
template <typename TX, typename TY, int L, int W, int Eights>
static void fwd_rows(const NormArgs &a, void *y, int64_t y_stride, float *mean, float *rstd, hipStream_t s) {
    constexpr int R = Eights <= 2 ? 2 : 1;
    if (R == 2 && a.rows <= kFwdBlocks * (L ? kThreads / (L ? L : 1) : 1)) return fwd_launch<TX, TY, L, W, Eights, 1, false>(a, y, y_stride, mean, rstd, s);
    if (past_cache<TX, TY>(a.rows, a.cols)) fwd_launch<TX, TY, L, W, Eights, R, true>(a, y, y_stride, mean, rstd, s);
    else fwd_launch<TX, TY, L, W, Eights, R, false>(a, y, y_stride, mean, rstd, s);
}
template <typename TX, typename TY>
static void fwd_typed(const NormArgs &a, void *y, int64_t y_stride, float *mean, float *rstd, hipStream_t s) {
    const int64_t eights = ceil_div(a.cols, 8);
    if (eights <= kWave)
        switch (lanes_of(eights)) {
            case 4: return fwd_rows<TX, TY, 4, 0, 1>(a, y, y_stride, mean, rstd, s);
            case 8: return fwd_rows<TX, TY, 8, 0, 1>(a, y, y_stride, mean, rstd, s);
            case 16: return fwd_rows<TX, TY, 16, 0, 1>(a, y, y_stride, mean, rstd, s);
            case 32: return fwd_rows<TX, TY, 32, 0, 1>(a, y, y_stride, mean, rstd, s);
            default: return fwd_rows<TX, TY, kWave, 0, 1>(a, y, y_stride, mean, rstd, s);
        }
    if (eights <= 2 * kWave) return fwd_rows<TX, TY, kWave, 0, 2>(a, y, y_stride, mean, rstd, s);
    if (eights <= kLaneEights) return fwd_rows<TX, TY, kWave, 0, 3>(a, y, y_stride, mean, rstd, s);
    if (eights <= 256) return fwd_rows<TX, TY, 0, 4, 1>(a, y, y_stride, mean, rstd, s);
    if (eights <= 512) return fwd_rows<TX, TY, 0, 4, 2>(a, y, y_stride, mean, rstd, s);
    if (eights <= 1024) return fwd_rows<TX, TY, 0, 4, 4>(a, y, y_stride, mean, rstd, s);
    if (eights <= 2048) return fwd_rows<TX, TY, 0, 8, 4>(a, y, y_stride, mean, rstd, s);
    if (eights <= 12 * 4 * kWave) return fwd_rows<TX, TY, 0, 12, 4>(a, y, y_stride, mean, rstd, s);
    if (eights <= 4096) return fwd_rows<TX, TY, 0, 16, 4>(a, y, y_stride, mean, rstd, s);
    fwd_rows<TX, TY, 0, 16, 8>(a, y, y_stride, mean, rstd, s);
}

}  // namespace spo

using namespace spo;

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
