// Normalisation of rows, forward and backward (the hidden states that a head reads, and the way back through them).
//
//   layer: mu = mean x, rstd = (mean (x - mu)^2 + eps)^-1/2, h = (x - mu) rstd;   rms: rstd = (mean x^2 + eps)^-1/2, h = x rstd
//   y = h w + b;  with g = dy w:  dx = rstd (g - mean g - h mean(g h)), rms without the mean of g;  dw = sum dy h,  db = sum dy
//
// Bound by HBM.  A row is held in registers from its one read to its one write: by 4 to 64 lanes of a wavefront (rows of up to
// 1536 elements in the forward, 1024 in the backward), or by 4 to 16 wavefronts of a workgroup.  Registers end at 32768 elements in the
// forward (beyond, some of a row waits in scratch memory: 4096 rows of 65536 in bf16 4.7 TB/s, 2048 in fp32 2.7) and at 16384 in the
// backward, which reads longer rows twice (2.9 to 3.2).  (284780 rows of 4096 in bf16: forward 751-785 us, 6.1 TB/s, backward
// 1180-1290 from card to card, 5.4 to 5.9; 17043 rows of 4096 from fp32 to bf16: forward 74, 5.7; 8192 of 1024, which the caches hold:
// 9.6 and 14.4.  One row: 2.6 us, a launch and its chain of loads and sums.)
//
// The forward takes its sums about a pivot, the mean of the row's first elements: one exchange between the lanes gives mean and
// variance.  Where the pivot was off by more than two deviations the row is read once more and summed about its mean, so that no
// digits are lost; where squares or differences leave fp32's range, it is read once more in 64 bits.  The backward has the mean as
// fp32; what rounding it took off is common to all elements of a row and small, but not beside the deviations of rows far from zero,
// so that the sum of (x - mean) rstd is taken along and put right.
#pragma once

#include <algorithm>

#include "vec8.hpp"

namespace spo {

constexpr int kMostCols = 65536;
constexpr int kParts = 1024;         // most workgroups of the backward: each leaves one row of partial sums
constexpr int kColumnParts = 256;    // ... and of the one that takes rows by columns
constexpr int kRegisterCols = 16384; // rows up to here are held by a workgroup of the backward
constexpr int kLaneEights = 192;     // rows of up to so many eights are held by lanes of one wavefront, in the forward
constexpr int kFwdBlocks = 2048;     // workgroups of the forward that are there before one holds two rows
constexpr int kThreads = 256;        // of a workgroup whose wavefronts have rows to themselves

struct NormArgs {
    const void *x;
    int64_t x_stride, rows;
    int cols, layer, w_dtype;
    const void *w, *b;
    float eps, inv_n;  // 1 / cols
};

template <int M, typename Move>
__device__ __forceinline__ void add_moved(float (&v)[M], Move move) {
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] += __int_as_float(move(__float_as_int(v[m])));
}
// Sums over L neighbouring lanes by moves between them; every lane receives them.  All lanes of the wavefront call this.
template <int L, int M>
__device__ __forceinline__ void lane_sums(float (&v)[M]) {
    if constexpr (L == kWave) {  // within rows of 16, then from row to row; the last lane's are everybody's
        add_moved(v, [](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false); });  // from one lane below
        add_moved(v, [](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false); });
        add_moved(v, [](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false); });
        add_moved(v, [](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false); });
        add_moved(v, [](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false); });  // a row's last lane to the next row
        add_moved(v, [](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false); });  // the second row's to the upper half
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v[m]), kWave - 1));
    } else {
        add_moved(v, [](int x) { return __builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true); });  // lanes in pairs,
        add_moved(v, [](int x) { return __builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true); });  // pairs in fours,
        if constexpr (L >= 8) add_moved(v, [](int x) { return __builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true); });   // fours in eights,
        if constexpr (L >= 16) add_moved(v, [](int x) { return __builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true); });  // eights in rows
        if constexpr (L >= 32) add_moved(v, [](int x) { return __shfl_xor(x, 16, kWave); });
    }
}
template <int L, int M>
__device__ __forceinline__ void lane_sums(double (&v)[M]) {
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) v[m] += __shfl_xor(v[m], o, kWave);
}
// ... and over the W wavefronts of the workgroup (0: as many as there are), all threads of which call this together, in order.
// scratch: M numbers per wavefront, free again after the next such call with another scratch.
template <int W, int M, typename T>
__device__ __forceinline__ void join_waves(T (&v)[M], T *scratch) {
    if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
        for (int m = 0; m < M; ++m) scratch[threadIdx.x / kWave * M + m] = v[m];
    __syncthreads();
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = T(0);
    const auto add = [&](int i) {
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] += scratch[i * M + m];
    };
    if constexpr (W > 0 && W <= 8) {
#pragma unroll
        for (int i = 0; i < W; ++i) add(i);
    } else {
        const int waves = W ? W : static_cast<int>(blockDim.x) / kWave;
        for (int i = 0; i < waves; ++i) add(i);
    }
}
// The value of the first of L neighbouring lanes, for all of them.
template <int L>
__device__ __forceinline__ float first_lane(float v) {
    const int x = __float_as_int(v);
    if constexpr (L == kWave) return __int_as_float(__builtin_amdgcn_readfirstlane(x));
    else if constexpr (L == 4) return __int_as_float(__builtin_amdgcn_mov_dpp(x, 0x00, 0xf, 0xf, true));
    else return __shfl(v, static_cast<int>(threadIdx.x) & ~(L - 1) & (kWave - 1), kWave);
}
// Sums over the L lanes that share a row, or with L = 0 over the W wavefronts of the workgroup.
template <int L, int W, int M, typename T>
__device__ __forceinline__ void row_sums(T (&v)[M], T *scratch) {
    lane_sums<L == 0 ? kWave : L>(v);
    if constexpr (L == 0) join_waves<W>(v, scratch);
}
// Whether any row that this wavefront holds asks for more: the same for all threads of a row.
template <int L>
__device__ __forceinline__ bool any_row(bool one) { return L == 0 ? one : __any(one) != 0; }

constexpr float kSquaresLow = 1e-30f, kSquaresHigh = 1e38f;  // a variance below, sums of squares above: formed again in 64 bits
constexpr float kLargest = 3.402823466e38f;
// Half of x - mean, of half the mean: finite for all finite rows.  The backward works with halves of h and doubles what it makes of them;
// but for subnormal numbers that changes no rounding.
__device__ __forceinline__ float half_from(float x, float half_mean) { return fmaf(x, 0.5f, -half_mean); }
// Elements of a vector: 16 bytes of bf16; four where fp32 is among the arrays, so that a wavefront's loads are whole lines
// (17043 rows of 4096 from fp32 to bf16: 78 us, with eight neighbours per thread 81).
template <typename TX, typename TY>
constexpr int kVector = sizeof(TX) == 2 && sizeof(TY) == 2 ? 8 : 4;

// Arrays that the Infinity Cache does not hold take the non-temporal hint
template <typename TX, typename TY>
static bool past_cache(int64_t rows, int64_t cols) { return rows * cols * static_cast<int64_t>(sizeof(TX) + sizeof(TY)) > kStreamBytes; }

// Lanes that hold a row of so many eights, one each (or two or three, with all lanes of a wavefront).  Rows of fewer than 24 elements leave
// lanes idle (16777216 rows of 16 in bf16: 3.7 TB/s, of 9: 1.8).  And wavefronts of a workgroup that holds a row and its sums in LDS, in
// fours, as they are dealt to the SIMDs of a compute unit (backward in bf16 with a bias, in fours and as many as the row needs: 19173 rows of
// 14000 403 and 427 us, 20971 of 12800 402 and 405, 29826 of 9000 480 and 461).
static int lanes_of(int64_t eights) { return eights <= 4 ? 4 : eights <= 8 ? 8 : eights <= 16 ? 16 : eights <= 32 ? 32 : kWave; }
static int fours_of(int64_t eights, int each) { return static_cast<int>(ceil_div(eights, each * 4 * kWave)) * 4; }

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
                    d->weight, d->bias, d->eps, 1.0f / static_cast<float>(d->cols)};
}

}  // namespace spo
