// Orthogonalised updates: X <- U / |U|, then `steps` times A = X X^T, B = b A + c A A, X <- a X + B X (on the other side for
// matrices with more rows than columns), and the momentum step around it.
//
// Numbers.  The products run on fp16 matrix instructions (the rate of bf16, three bits more): every operand is scaled by a
// power of two to where fp16 is exact to 11 bits.  What this costs was found in 64 bits on gaussian, decaying and nearly
// low-rank matrices: small singular values grow by a (3.44) per step, and with them whatever was rounded in X; the rounding
// of A and B is not amplified.  So X is kept as a pair of halves (hi + lo / 2048, 22 bits), the term a X reads both, the
// products read hi alone: 2e-4 to 1.7e-3 after five steps (X in 11 bits: up to 2e-2; all of it in bf16: up to 0.16) for
// 4 bytes more per entry in the epilogue.  SPO_PRODUCTS_SPLIT keeps A and B as pairs too and forms
// hi hi + (hi lo + lo hi) / 2048 in every product: 3e-7 to 5e-6, three times the matrix instructions.
//
// Every matrix in the workspace has its sides rounded up to a step of the contraction (64), zero beyond the true ones: the
// main loop of gemm_core.hpp then has no ends to look after.
#include <algorithm>

#include "gemm_core.hpp"
#include "tile_choice.hpp"

namespace spo {

typedef Tile<256, 256, 2, 4, _Float16> OL;
typedef Tile<128, 128, 2, 2, _Float16> OS;

constexpr float kLoScale = 2048.0f;   // lo parts are held that much larger: as far above fp16's smallest numbers as hi parts
constexpr float kGramScale = 256.0f;  // A and B: their entries stay below about 10

typedef uint16_t half_t;  // raw IEEE half bits

__device__ __forceinline__ float half_value(uint32_t bits) { return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits))); }
__device__ __forceinline__ uint32_t half_bits(float v) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v)); }

// eight consecutive values of an output row, as the parts they are stored in
struct Eight {
    float v[8];
    __device__ __forceinline__ void split(uint4 &hi, uint4 &lo) const {
        uint32_t h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t h0 = half_bits(v[2 * i]), h1 = half_bits(v[2 * i + 1]);
            h[i] = h0 | h1 << 16;
            l[i] = half_bits((v[2 * i] - half_value(h0)) * kLoScale) | half_bits((v[2 * i + 1] - half_value(h1)) * kLoScale) << 16;
        }
        hi = make_uint4(h[0], h[1], h[2], h[3]);
        lo = make_uint4(l[0], l[1], l[2], l[3]);
    }
    // += beta * (hi + lo / 2048)
    __device__ __forceinline__ void add(float beta, const uint4 &hi, const uint4 &lo) {
        const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int sh = 16 * (i & 1);
            v[i] = fmaf(beta, fmaf(half_value(l[i / 2] >> sh & 0xffffu), 1.0f / kLoScale, half_value(h[i / 2] >> sh & 0xffffu)), v[i]);
        }
    }
};

// A stack of matrices in the workspace: `pairs` two planes (hi, lo) of rows x ld halves, else one.
struct Stack {
    half_t *base;
    int64_t ld, plane, step;  // elements: of a row, of a plane, from one matrix to the next
    __host__ __device__ half_t *of(int64_t i) const { return base + i * step; }
};

// Where the last product goes: out = value, or the weights' update W = keep W - rate value.
struct OrthOut {
    void *out;       // NULL: not the last product
    int dtype, update;
    int64_t ld, step;
    float keep, rate;
};

struct OrthProduct {
    Stack a, b, d, out;   // d.base NULL: no addend
    int64_t M, N, Mp, Np; // true and padded sides of the output
    int64_t batch;
    int KT, split;        // split: products of pairs
    float alpha, beta;    // value = alpha * (A B) + beta * D
    int d_lo, out_lo;     // D has, the output gets, a lo plane
    OrthOut last;
};

typedef uint32_t u32x4a2_t __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4a4_t __attribute__((ext_vector_type(4), aligned(4)));

// n (1..8) consecutive elements of a caller's array, from index `at` on
__device__ __forceinline__ void load_values(const void *p, int dtype, int64_t at, int n, float (&x)[8]) {
    if (dtype == SPO_FP32) {
        const float *q = static_cast<const float *>(p) + at;
        if (n == 8) {
            const f32x4a4_t u = *reinterpret_cast<const f32x4a4_t *>(q), v = *reinterpret_cast<const f32x4a4_t *>(q + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = u[i]; x[4 + i] = v[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < n ? q[i] : 0.0f;
        }
        return;
    }
    const bf16_t *q = static_cast<const bf16_t *>(p) + at;
    if (n == 8) {
        const u32x4a2_t u = *reinterpret_cast<const u32x4a2_t *>(q);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < n ? bf16_to_f32(q[i]) : 0.0f;
    }
}
__device__ __forceinline__ void store_values(void *p, int dtype, int64_t at, int n, const float (&x)[8]) {
    if (dtype == SPO_FP32) {
        float *q = static_cast<float *>(p) + at;
        if (n == 8) {
            *reinterpret_cast<f32x4a4_t *>(q) = f32x4a4_t{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<f32x4a4_t *>(q + 4) = f32x4a4_t{x[4], x[5], x[6], x[7]};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) q[i] = x[i];
        }
        return;
    }
    bf16_t *q = static_cast<bf16_t *>(p) + at;
    if (n == 8) {
        *reinterpret_cast<u32x4a2_t *>(q) = u32x4a2_t{pack_bf16x2_rn(x[0], x[1]), pack_bf16x2_rn(x[2], x[3]), pack_bf16x2_rn(x[4], x[5]),
                                                      pack_bf16x2_rn(x[6], x[7])};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) q[i] = f32_to_bf16(x[i]);
    }
}

// eight values of row m from column n on, on their way out of the last product
__device__ __forceinline__ void store_last(const OrthOut &o, int64_t matrix, int64_t m, int64_t n, int64_t N, Eight &e) {
    const int count = N - n < 8 ? static_cast<int>(N - n) : 8;
    if (count <= 0) return;
    const int64_t at = matrix * o.step + m * o.ld + n;
    if (o.update) {
        float w[8];
        load_values(o.out, o.dtype, at, count, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = fmaf(-o.rate, e.v[i], o.keep * w[i]);
    }
    store_values(o.out, o.dtype, at, count, e.v);
}

template <typename TT>
__device__ __forceinline__ void store_product(typename TT::Acc &acc, const OrthProduct &p, int64_t matrix, int64_t m0, int64_t n0) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));  // not to be traced: nothing derived from it is to live through the main loop
    const int grp = lane >> 4, col = lane & 15;
    const half_t *d = p.d.base ? p.d.of(matrix) : nullptr;
    half_t *out = p.out.base ? p.out.of(matrix) : nullptr;
#pragma unroll
    for (int i = 0; i < TT::FM; ++i) {
        const int64_t m = m0 + TT::wave_m0() + i * TT::MI + col;
#pragma unroll
        for (int j = 0; j < TT::FN; j += 2) {
            // after an exchange between neighbouring lane groups a lane holds eight consecutive columns of its row
            Eight e;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint32_t x = __float_as_uint(acc[i][j][r]), y = __float_as_uint(acc[i][j + 1][r]);
                swap_lane_groups(x, y);
                e.v[r] = __uint_as_float(x) * p.alpha;
                e.v[4 + r] = __uint_as_float(y) * p.alpha;
            }
            const int64_t n = n0 + TT::wave_n0() + j * TT::MI + (grp & 1) * TT::MI + (grp & 2) * 4;
            if (m >= p.Mp || n >= p.Np) continue;
            if (d) {
                const uint4 hi = *reinterpret_cast<const uint4 *>(d + m * p.d.ld + n);
                const uint4 lo = p.d_lo ? *reinterpret_cast<const uint4 *>(d + p.d.plane + m * p.d.ld + n) : make_uint4(0u, 0u, 0u, 0u);
                e.add(p.beta, hi, lo);
            }
            if (p.last.out) {
                if (m < p.M) store_last(p.last, matrix, m, n, p.N, e);
                continue;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (m >= p.M || n + k >= p.N) e.v[k] = 0.0f;
            uint4 hi, lo;
            e.split(hi, lo);
            *reinterpret_cast<uint4 *>(out + m * p.out.ld + n) = hi;
            if (p.out_lo) *reinterpret_cast<uint4 *>(out + p.out.plane + m * p.out.ld + n) = lo;
        }
    }
}

// value = alpha * sum_k A(m,k) B(n,k) + beta * D for every matrix of a stack.  ACols, BCols: the operand has the contraction
// index as its row index.
template <typename TT, bool ACols, bool BCols, bool Split>
__global__ void __launch_bounds__(TT::NT, 2)
orth_product_kernel(OrthProduct p) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const TileOrder ord(ceil_div(p.Mp, TT::BM), ceil_div(p.Np, TT::BN));
    const uint32_t tiles = static_cast<uint32_t>(ord.tiles());
    uint32_t i;
    if (!TileOrder::item(blockIdx.x, static_cast<uint32_t>(tiles * p.batch), i)) return;
    const int64_t matrix = i / tiles;
    int64_t tm, tn;
    ord.at(i % tiles, tm, tn);
    const int64_t m0 = tm * TT::BM, n0 = tn * TT::BN;
    const half_t *a = p.a.of(matrix), *b = p.b.of(matrix);
    auto A = [&](int lo) { return typename TT::Operand{reinterpret_cast<const char *>(a + lo * p.a.plane), p.a.ld * 2, m0, p.Mp, 0}; };
    auto B = [&](int lo) { return typename TT::Operand{reinterpret_cast<const char *>(b + lo * p.b.plane), p.b.ld * 2, n0, p.Np, 0}; };
    typename TT::Acc acc;
    TT::zero(acc);
    if constexpr (Split) {
        TT::template mainloop<ACols, BCols, true>(A(0), B(1), p.KT, lds, acc);
        TT::template mainloop<ACols, BCols, true>(A(1), B(0), p.KT, lds, acc);
#pragma unroll
        for (int x = 0; x < TT::FM; ++x)
#pragma unroll
            for (int y = 0; y < TT::FN; ++y) acc[x][y] *= 1.0f / kLoScale;
    }
    TT::template mainloop<ACols, BCols, true>(A(0), B(0), p.KT, lds, acc);
    store_product<TT>(acc, p, matrix, m0, n0);
}

// ----------------------------------------------------------------------------
// before the products: momentum, norm, scaling
// ----------------------------------------------------------------------------
struct OrthInput {
    const void *G;
    int dtype;
    int64_t stride, step;      // elements from row to row, from matrix to matrix
    float *momentum;           // NULL: U = G
    float mu;
    int nesterov;
    int64_t rows, cols;
    float eps;
};
constexpr int kNormParts = 256;  // most workgroups per matrix, and threads that join their sums

// U of eight entries from column c on; First: M <- mu M + G on the way (otherwise M is as it was left by that)
template <bool First>
__device__ __forceinline__ void load_update(const OrthInput &in, int64_t matrix, int64_t r, int64_t c, float (&u)[8]) {
    const int count = in.cols - c < 8 ? static_cast<int>(in.cols - c) : 8;
    load_values(in.G, in.dtype, matrix * in.step + r * in.stride + c, count, u);
    if (!in.momentum) return;
    const int64_t at = (matrix * in.rows + r) * in.cols + c;
    float m[8];
    load_values(in.momentum, SPO_FP32, at, count, m);
    if (First) {
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = fmaf(in.mu, m[i], u[i]);
        store_values(in.momentum, SPO_FP32, at, count, m);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = in.nesterov ? fmaf(in.mu, m[i], u[i]) : m[i];
}

// part[matrix][workgroup] = sum of squares of its share of U
__global__ void __launch_bounds__(256) orth_norm_kernel(OrthInput in, double *__restrict__ part) {
    __shared__ double scratch[4];
    const int64_t matrix = blockIdx.y, per_row = ceil_div(in.cols, 8), n = in.rows * per_row;
    double sum = 0.0;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
        float u[8], s = 0.0f;
        load_update<true>(in, matrix, i / per_row, i % per_row * 8, u);
#pragma unroll
        for (int k = 0; k < 8; ++k) s = fmaf(u[k], u[k], s);
        sum += s;
    }
    sum = block_sum(sum, scratch);
    if (threadIdx.x == 0) part[matrix * gridDim.x + blockIdx.x] = sum;
}

// X = scale * U / (|U| + eps) as pairs of halves, zero in the padding; with last.out: U / (|U| + eps) goes there (no steps)
__global__ void __launch_bounds__(256) orth_scale_kernel(OrthInput in, const double *__restrict__ part, int parts, float scale, Stack X,
                                                         int64_t rows_p, OrthOut last) {
    __shared__ double scratch[4];
    const int64_t matrix = blockIdx.y;
    const double norm = sqrt(block_sum(static_cast<int>(threadIdx.x) < parts ? part[matrix * parts + threadIdx.x] : 0.0, scratch));
    const double whole = norm + static_cast<double>(in.eps);
    const float f = whole > 0.0 ? static_cast<float>((last.out ? 1.0 : scale) / whole) : whole == 0.0 ? 0.0f : __builtin_nanf("");
    const int64_t per_row = X.ld / 8, n = rows_p * per_row;
    half_t *x = X.of(matrix);
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t r = i / per_row, c = i % per_row * 8;
        Eight e;
#pragma unroll
        for (int k = 0; k < 8; ++k) e.v[k] = 0.0f;
        const bool inside = r < in.rows && c < in.cols;
        if (inside) {
            load_update<false>(in, matrix, r, c, e.v);
#pragma unroll
            for (int k = 0; k < 8; ++k) e.v[k] *= f;
        }
        if (last.out) {
            if (inside) store_last(last, matrix, r, c, in.cols, e);
            continue;
        }
        uint4 hi, lo;
        e.split(hi, lo);
        *reinterpret_cast<uint4 *>(x + r * X.ld + c) = hi;
        *reinterpret_cast<uint4 *>(x + X.plane + r * X.ld + c) = lo;
    }
}

// ----------------------------------------------------------------------------
// host side
// ----------------------------------------------------------------------------
static int64_t padded(int64_t n) { return ceil_div(n, kBK) * kBK; }

struct OrthPlan {
    int64_t rp, cp, k, kp;  // padded sides, the smaller side and the same padded
    int parts;
    double *norm;
    Stack X[2], A, B;
    float x_scale;
    size_t bytes;
};

static OrthPlan plan_orth(const spo_orth_desc *d, void *ws) {
    OrthPlan p;
    p.rp = padded(d->rows);
    p.cp = padded(d->cols);
    p.k = std::min(d->rows, d->cols);
    p.kp = padded(p.k);
    // X's entries are about 1 / sqrt(longer side) once its singular values are near one
    p.x_scale = 1.0f;
    for (int64_t n = std::max(d->rows, d->cols); n > 1; n /= 4) p.x_scale *= 2.0f;
    const int64_t vectors = d->rows * ceil_div(d->cols, 8);
    p.parts = static_cast<int>(std::min<int64_t>(kNormParts, ceil_div(vectors, 256 * 4)));
    Arena a(ws);
    p.norm = a.take<double>(static_cast<size_t>(d->batch) * kNormParts);
    auto stack = [&](int64_t rows, int64_t ld) {
        Stack s{nullptr, ld, rows * ld, 2 * rows * ld};
        s.base = a.take<half_t>(static_cast<size_t>(d->batch) * 2 * rows * ld);
        return s;
    };
    p.X[0] = stack(p.rp, p.cp);
    p.X[1] = stack(p.rp, p.cp);
    p.A = stack(p.kp, p.kp);
    p.B = stack(p.kp, p.kp);
    p.bytes = a.used;
    return p;
}

template <typename TT, bool ACols, bool BCols, bool Split>
static int launch_product(const OrthProduct &p, hipStream_t s) {
    auto *kernel = orth_product_kernel<TT, ACols, BCols, Split>;
    if (int rc = allow_lds(kernel, TT::LDS_BYTES)) return rc;
    const int64_t items = ceil_div(p.Mp, TT::BM) * ceil_div(p.Np, TT::BN) * p.batch;
    kernel<<<static_cast<unsigned>(TileOrder::blocks(items)), TT::NT, TT::LDS_BYTES, s>>>(p);
    return SPO_OK;
}
template <bool ACols, bool BCols>
static int launch_product(const OrthProduct &p, hipStream_t s) {
    const bool small = tiles_over(p.Mp, false) * tiles_over(p.Np, false) * p.batch < kChipCUs * 3 / 4;
    if (small) return p.split ? launch_product<OS, ACols, BCols, true>(p, s) : launch_product<OS, ACols, BCols, false>(p, s);
    return p.split ? launch_product<OL, ACols, BCols, true>(p, s) : launch_product<OL, ACols, BCols, false>(p, s);
}

static int run_orth(const spo_orth_desc *d, const OrthInput &in, OrthOut last, void *ws, size_t ws_bytes, hipStream_t s) {
    const OrthPlan p = plan_orth(d, ws);
    if (ws_bytes < p.bytes) return SPO_EWORKSPACE;
    const dim3 parts(static_cast<unsigned>(p.parts), static_cast<unsigned>(d->batch));
    orth_norm_kernel<<<parts, 256, 0, s>>>(in, p.norm);
    const int64_t vectors = p.rp * p.cp / 8;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(1024, ceil_div(vectors, 256))), static_cast<unsigned>(d->batch));
    orth_scale_kernel<<<grid, 256, 0, s>>>(in, p.norm, p.parts, p.x_scale, p.X[0], p.rp, d->steps ? OrthOut{} : last);
    // Where the smaller side is one step of the contraction, launches are all that counts, and so few roundings do not
    // average out (one of 1 x 1: 4e-3): always pairs.
    const bool tall = d->rows > d->cols, split = d->products == SPO_PRODUCTS_SPLIT || p.k <= kBK;
    for (int i = 0; i < d->steps; ++i) {
        const Stack &X = p.X[i & 1], &Xn = p.X[(i + 1) & 1];
        OrthProduct q{};
        q.batch = d->batch;
        q.split = split;
        q.d_lo = q.out_lo = split;
        // A = X X^T (X^T X)
        q.a = q.b = X;
        q.out = p.A;
        q.M = q.N = p.k;
        q.Mp = q.Np = p.kp;
        q.KT = static_cast<int>((tall ? p.rp : p.cp) / kBK);
        q.alpha = kGramScale / (p.x_scale * p.x_scale);
        if (int rc = tall ? launch_product<true, true>(q, s) : launch_product<false, false>(q, s)) return rc;
        // B = b A + c A A; both are symmetric, so rows serve as columns
        q.a = q.b = q.d = p.A;
        q.out = p.B;
        q.KT = static_cast<int>(p.kp / kBK);
        q.alpha = d->c / kGramScale;
        q.beta = d->b;
        if (int rc = launch_product<false, false>(q, s)) return rc;
        // X <- a X + B X (X B)
        q.a = tall ? X : p.B;
        q.b = tall ? p.B : X;
        q.d = X;
        q.d_lo = q.out_lo = 1;
        q.out = Xn;
        q.M = d->rows;
        q.N = d->cols;
        q.Mp = p.rp;
        q.Np = p.cp;
        q.alpha = 1.0f / kGramScale;
        q.beta = d->a;
        if (i == d->steps - 1) {
            q.alpha /= p.x_scale;
            q.beta /= p.x_scale;
            q.last = last;
        }
        if (int rc = tall ? launch_product<false, false>(q, s) : launch_product<false, true>(q, s)) return rc;
    }
    return launch_status();
}

}  // namespace spo

using namespace spo;

static int validate(const spo_orth_desc *d) {
    if (!d) return SPO_ENULL;
    if (d->struct_size != sizeof(spo_orth_desc)) return SPO_EINVAL;
    if (d->batch < 1 || d->rows < 1 || d->cols < 1 || d->steps < 0) return SPO_EINVAL;
    if (d->products != SPO_PRODUCTS_FP16 && d->products != SPO_PRODUCTS_SPLIT) return SPO_EINVAL;
    if (!(d->eps >= 0.0f)) return SPO_EINVAL;
    if (d->batch > 65535 || d->rows > 65536 || d->cols > 65536 || d->steps > 64) return SPO_ERANGE;
    return SPO_OK;
}
static bool type_ok(int t) { return t == SPO_FP32 || t == SPO_BF16; }
static bool aligned_to(const void *p, int dtype) { return reinterpret_cast<uintptr_t>(p) % (dtype == SPO_FP32 ? 4 : 2) == 0; }
static int check_ws(void *ws) {
    if (!ws) return SPO_EWORKSPACE;
    return reinterpret_cast<uintptr_t>(ws) % 256 != 0 ? SPO_EINVAL : SPO_OK;
}

extern "C" size_t spo_orthogonalize_workspace_bytes(const spo_orth_desc *d) {
    return validate(d) == SPO_OK ? plan_orth(d, nullptr).bytes : 0;
}

extern "C" int spo_orthogonalize(const spo_orth_desc *d, const void *G, int g_dtype, int64_t g_stride, int64_t g_batch_stride,
                                 void *out, int out_dtype, void *ws, size_t ws_bytes, spo_stream_t stream) {
    int rc = validate(d);
    if (rc) return rc;
    if (!G || !out) return SPO_ENULL;
    if (!type_ok(g_dtype) || !type_ok(out_dtype) || !aligned_to(G, g_dtype) || !aligned_to(out, out_dtype)) return SPO_EINVAL;
    if ((g_stride && g_stride < d->cols) || g_batch_stride < 0) return SPO_EINVAL;
    if ((rc = check_ws(ws))) return rc;
    OrthInput in{};
    in.G = G;
    in.dtype = g_dtype;
    in.stride = g_stride ? g_stride : d->cols;
    in.step = g_batch_stride ? g_batch_stride : d->rows * in.stride;
    in.rows = d->rows;
    in.cols = d->cols;
    in.eps = d->eps;
    return run_orth(d, in, OrthOut{out, out_dtype, 0, d->cols, d->rows * d->cols, 0.0f, 0.0f}, ws, ws_bytes, as_stream(stream));
}

extern "C" int spo_muon_update(const spo_orth_desc *d, void *W, int w_dtype, float *momentum, const void *grad, int g_dtype, float mu,
                               int nesterov, float lr, float weight_decay, float scale, void *ws, size_t ws_bytes, spo_stream_t stream) {
    int rc = validate(d);
    if (rc) return rc;
    if (!W || !momentum || !grad) return SPO_ENULL;
    if (!type_ok(w_dtype) || !type_ok(g_dtype) || !aligned_to(W, w_dtype) || !aligned_to(grad, g_dtype) || !aligned_to(momentum, SPO_FP32))
        return SPO_EINVAL;
    if (!(mu >= 0.0f && mu < 1.0f) || !(lr >= 0.0f) || !(weight_decay >= 0.0f) || !(scale == scale)) return SPO_EINVAL;
    if ((rc = check_ws(ws))) return rc;
    OrthInput in{};
    in.G = grad;
    in.dtype = g_dtype;
    in.stride = d->cols;
    in.step = d->rows * d->cols;
    in.momentum = momentum;
    in.mu = mu;
    in.nesterov = nesterov ? 1 : 0;
    in.rows = d->rows;
    in.cols = d->cols;
    in.eps = d->eps;
    const float keep = static_cast<float>(1.0 - static_cast<double>(lr) * weight_decay);
    return run_orth(d, in, OrthOut{W, w_dtype, 1, d->cols, d->rows * d->cols, keep, lr * scale}, ws, ws_bytes, as_stream(stream));
}
