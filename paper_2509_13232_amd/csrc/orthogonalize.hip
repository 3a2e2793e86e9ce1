// Orthogonalised updates: X <- U / |U|, then `steps` times A = X X^T, B = b A + c A A, X <- a X + B X, and the momentum step
// around it.  Matrices with more rows than columns are worked on transposed: on their way into X, and on their way out of the
// last product.
//
// Numbers.  The products run on fp16 matrix instructions (the rate of bf16, three bits more): every operand is scaled by a
// power of two to where fp16 is exact to 11 bits.  What this costs was found in 64 bits on gaussian, decaying and nearly
// low-rank matrices: small singular values grow by a (3.44) per step, and with them whatever was rounded in X; the rounding
// of A and B is not amplified.  So X is kept as a pair of halves (hi + lo / 2048, 22 bits), the term a X reads both, the
// products read hi alone: 2e-4 to 1.7e-3 after five steps (X in 11 bits: up to 2e-2; all of it in bf16: up to 0.16) for
// 4 bytes more per entry in the epilogue.  Most of what is left comes from the diagonals of A and B, which lie near the mean
// of the squared singular values, s = |X|_F^2 / k, and near b s + c s^2.  So what is stored is A' = A - s I and
// B' = c A' A' + (b + 2 c s) A', and X <- (a + b s + c s^2) X + B' X: the same polynomial, 7e-5 to 7.2e-4
// from sides of 128 on, 9.4e-4 at 66 x 66.
// SPO_PRODUCTS_SPLIT keeps A and B as pairs too and forms
// hi hi + (hi lo + lo hi) / 2048 in every product: 3e-7 to 3.4e-6, three times the matrix instructions.
//
// Every matrix in the workspace has its sides rounded up to a step of the contraction (64), zero beyond the true ones: the
// main loop of gemm_core.hpp then has no ends to look after.
#include <algorithm>

#include "gemm_core.hpp"
#include "orth_choice.hpp"

namespace spo {

// Tiles that the wavefronts of a workgroup share; symmetric products also take the middle ones.
typedef Tile<256, 256, 2, 4, 16, true> OL;
typedef Tile<192, 192, 4, 2, 16, true> OM;
typedef Tile<128, 128, 2, 2, 16, true> OS;

constexpr float kLoScale = 2048.0f;   // lo parts are held that much larger: as far above fp16's smallest numbers as hi parts
constexpr float kGramScale = 256.0f;  // A and B: their entries stay below about 10

typedef uint16_t half_t;  // raw IEEE half bits

// eight consecutive values of an output row, as the parts they are stored in
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
struct Eight {
    float v[8];
    // (written so that a pair takes five instructions: one conversion, and a mixed multiply-add for each difference and lo part)
    __device__ __forceinline__ void split(uint4 &hi, uint4 &lo) const {
        uint32_t h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f16x2_t p = __builtin_convertvector((f32x2_t{v[2 * i], v[2 * i + 1]}), f16x2_t);
            const float a = fmaf(static_cast<float>(p.x), -1.0f, v[2 * i]), b = fmaf(static_cast<float>(p.y), -1.0f, v[2 * i + 1]);
            const f16x2_t q = {static_cast<_Float16>(a * kLoScale), static_cast<_Float16>(b * kLoScale)};
            h[i] = __builtin_bit_cast(uint32_t, p);
            l[i] = __builtin_bit_cast(uint32_t, q);
        }
        hi = make_uint4(h[0], h[1], h[2], h[3]);
        lo = make_uint4(l[0], l[1], l[2], l[3]);
    }
    // += beta * (hi + lo / 2048)
    __device__ __forceinline__ void add(float beta, const uint4 &hi, const uint4 &lo) {
        const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f16x2_t p = __builtin_bit_cast(f16x2_t, h[i]), q = __builtin_bit_cast(f16x2_t, l[i]);
            v[2 * i] = fmaf(beta, fmaf(static_cast<float>(q.x), 1.0f / kLoScale, static_cast<float>(p.x)), v[2 * i]);
            v[2 * i + 1] = fmaf(beta, fmaf(static_cast<float>(q.y), 1.0f / kLoScale, static_cast<float>(p.y)), v[2 * i + 1]);
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
    int dtype, update, across;  // across: X is the output's transpose
    int64_t ld, step;
    float keep, rate;
};

struct OrthProduct {
    Stack a, b, d, out;   // d.base NULL: no addend
    int64_t M, N, Mp, Np; // true and padded sides of the output
    int64_t batch;
    int KT, split;        // split: products of pairs
    int symmetric;        // only tiles on and below the diagonal are formed, each stored on both sides
    float alpha;          // value = alpha * (A B) + beta * D, beta = c[0] + s (c[1] + s c[2])
    float c[3];
    int d_lo, out_lo;     // D has, the output gets, a lo plane
    // Of each matrix the mean s of X's squared singular values: the product of X and its transpose forms it from the partial
    // sums of X's squares (n_sq of them, times sq_scale), takes it off its diagonal and leaves it in shift; the others read it.
    const float *sq;
    int n_sq;
    float sq_scale;
    float *shift;
    float *sq_out;        // [matrix][tile][wavefront] sums of squares of what is stored, NULL: not asked for
    OrthOut last;
};

// s of a matrix (see OrthProduct) in two parts: every wavefront's sum into scratch (NT / 64 floats), and, after a barrier, their
// total for every thread.
template <int NT>
__device__ __forceinline__ float begin_shift(const OrthProduct &p, int64_t matrix, float *scratch) {
    if (!p.n_sq) return p.shift[matrix];
    float sum = 0.0f;
    for (int i = threadIdx.x; i < p.n_sq; i += NT) sum += p.sq[matrix * p.n_sq + i];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x / kWave] = sum;
    return 0.0f;
}
template <int NT>
__device__ __forceinline__ float end_shift(const OrthProduct &p, int64_t matrix, const float *scratch, float begun, bool first_tile) {
    if (!p.n_sq) return begun;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) sum += scratch[w];
    sum *= p.sq_scale;
    if (first_tile && threadIdx.x == 0) p.shift[matrix] = sum;
    return sum;
}
__device__ __forceinline__ float beta_of(const OrthProduct &p, float s) { return p.c[0] + s * (p.c[1] + s * p.c[2]); }
// a wavefront's sum of squares (one by one: no barrier)
template <int NT>
__device__ __forceinline__ void store_squares(const OrthProduct &p, int64_t matrix, uint32_t tiles, uint32_t tile, float sum) {
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) p.sq_out[(matrix * tiles + tile) * (NT / kWave) + threadIdx.x / kWave] = sum;
}

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

// eight values of row m of X from column n on (N: X's columns), on their way out of the last product
__device__ __forceinline__ void store_last(const OrthOut &o, int64_t matrix, int64_t m, int64_t n, int64_t N, Eight &e) {
    const int count = N - n < 8 ? static_cast<int>(N - n) : 8;
    if (count <= 0) return;
    if (o.across) {  // (neighbouring lanes hold neighbouring m)
        const int64_t first = matrix * o.step + n * o.ld + m;
        if (o.dtype == SPO_FP32) {
            float *q = static_cast<float *>(o.out) + first;
            float w[8];
            if (o.update)
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = q[(i < count ? i : 0) * o.ld];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) q[i * o.ld] = o.update ? fmaf(-o.rate, e.v[i], o.keep * w[i]) : e.v[i];
        } else {
            bf16_t *q = static_cast<bf16_t *>(o.out) + first;
            bf16_t w[8];
            if (o.update)
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = q[(i < count ? i : 0) * o.ld];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) q[i * o.ld] = f32_to_bf16(o.update ? fmaf(-o.rate, e.v[i], o.keep * bf16_to_f32(w[i])) : e.v[i]);
        }
        return;
    }
    const int64_t at = matrix * o.step + m * o.ld + n;
    if (o.update) {
        float w[8];
        load_values(o.out, o.dtype, at, count, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = fmaf(-o.rate, e.v[i], o.keep * w[i]);
    }
    store_values(o.out, o.dtype, at, count, e.v);
}

// The tiles of a product in the order of their ids: those of TileOrder, or of a symmetric product (n x n tiles) the rows of the
// lower triangle one after the other.
struct OrthTiles {
    int64_t nM, nN, count;
    bool symmetric;
    __host__ __device__ OrthTiles(int64_t M, int64_t N, int64_t edge, bool sym)
        : nM(ceil_div(M, edge)), nN(ceil_div(N, edge)), count(orth_tiles(M, N, edge, sym)), symmetric(sym) {}
    __host__ __device__ int64_t tiles() const { return count; }
    __device__ __forceinline__ void at(uint32_t i, int64_t &tm, int64_t &tn) const {
        if (!symmetric) return TileOrder(nM, nN).at(i, tm, tn);
        uint32_t r = static_cast<uint32_t>((sqrtf(8.0f * static_cast<float>(i) + 1.0f) - 1.0f) * 0.5f);  // to one off
        while (r * (r + 1) / 2 > i) --r;
        while ((r + 1) * (r + 2) / 2 <= i) ++r;
        tm = r;
        tn = i - r * (r + 1) / 2;
    }
};

// `shift` off the diagonal of a tile on it
__device__ __forceinline__ void off_diagonal(float shift, int m, int n, Eight &e) {
#pragma unroll
    for (int k = 0; k < 8; ++k) e.v[k] -= m == n + k ? shift : 0.0f;
}
__device__ __forceinline__ void clear_padding(const OrthProduct &p, int64_t m, int64_t n, Eight &e) {
    if (m < p.M && n + 8 <= p.N) return;
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (m >= p.M || n + k >= p.N) e.v[k] = 0.0f;
}

template <typename TT> constexpr int kTurnPitch = TT::BM + 8;  // halves
template <typename TT> constexpr int kOrthLds = TT::LDS_BYTES > TT::BN * kTurnPitch<TT> * 2 ? TT::LDS_BYTES : TT::BN * kTurnPitch<TT> * 2;

// A finished tile, straight from the accumulators; of a symmetric product also its mirror image, which is turned in LDS, a
// plane at a time (Plane: 0 the hi parts and all that goes straight out, 1 the mirror image's lo parts).  Returns the sum of
// squares of what this thread stored (not of symmetric products).
template <typename TT, int Plane, bool Mirror>
__device__ __forceinline__ float store_product(typename TT::Acc &acc, const OrthProduct &p, float shift, int64_t matrix, int64_t m0, int64_t n0,
                                               char *lds) {
    const float beta = beta_of(p, shift), diagonal = Mirror && p.n_sq && m0 == n0 ? shift * kGramScale : 0.0f;
    float squares = 0.0f;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));  // not to be traced: nothing derived from it is to live through the main loop
    const int grp = lane >> 4, col = lane & 15;
    const bool mirror = Mirror && p.symmetric && m0 != n0;
    if (Plane == 1 && !mirror) return 0.0f;
    // places inside the tile: in 32 bits (rows are at most 65600 halves)
    const int d_ld = static_cast<int>(p.d.ld), out_ld = static_cast<int>(p.out.ld);
    const half_t *d = p.d.base ? p.d.of(matrix) + m0 * p.d.ld + n0 : nullptr, *d_lo_plane = d + p.d.plane;
    half_t *out = p.out.of(matrix) + m0 * p.out.ld + n0, *out_lo_plane = out + p.out.plane;
    const int rows = static_cast<int>(p.M - m0), cols = static_cast<int>(p.N - n0);            // true sides, from the tile's corner
    const int rows_p = static_cast<int>(p.Mp - m0), cols_p = static_cast<int>(p.Np - n0);      // padded ones, multiples of 64
    half_t *turn = reinterpret_cast<half_t *>(lds);
    // The addend of the next sixteen rows is requested before this sixteen are worked on.
    constexpr int C = TT::FN / 2;
    uint4 d_hi[2][C], d_lo[2][C];
    auto row = [&](int i) { return TT::wave_m0() + i * TT::MI + col; };
    auto column = [&](int j) { return TT::wave_n0() + 2 * j * TT::MI + (grp & 1) * TT::MI + (grp & 2) * 4; };
    auto request = [&](int i) {
        const int m = row(i);
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int n = column(j), at = (m < rows_p ? m : 0) * d_ld + (n < cols_p ? n : 0);  // always a load
            d_hi[i & 1][j] = *reinterpret_cast<const uint4 *>(d + at);
            d_lo[i & 1][j] = p.d_lo ? *reinterpret_cast<const uint4 *>(d_lo_plane + at) : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    if (d) request(0);
    if (mirror) __syncthreads();  // operands, or the other plane, are no longer read
    const bool inside = TT::wave_m0() + TT::WM <= rows && TT::wave_n0() + TT::WN <= cols;  // of the wavefront's part, all
#pragma unroll
    for (int i = 0; i < TT::FM; ++i) {
        if (d && i + 1 < TT::FM) request(i + 1);
#pragma unroll
        for (int j = 0; j < C; ++j) {
            // after an exchange between neighbouring lane groups a lane holds eight consecutive columns of its row
            Eight e;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint32_t x = __float_as_uint(acc[i][2 * j][r]), y = __float_as_uint(acc[i][2 * j + 1][r]);
                swap_lane_groups(x, y);
                e.v[r] = __uint_as_float(x) * p.alpha;
                e.v[4 + r] = __uint_as_float(y) * p.alpha;
            }
            const int m = row(i), n = column(j);
            if (d) e.add(beta, d_hi[i & 1][j], d_lo[i & 1][j]);
            if (Mirror && diagonal != 0.0f) off_diagonal(diagonal, m, n, e);
            if (!inside)
#pragma unroll
                for (int k = 0; k < 8; ++k) e.v[k] = m < rows && n + k < cols ? e.v[k] : 0.0f;
            if (!Mirror)
#pragma unroll
                for (int k = 0; k < 8; ++k) squares = fmaf(e.v[k], e.v[k], squares);
            uint4 hi, lo;
            e.split(hi, lo);
            if (inside || (m < rows_p && n < cols_p)) {
                if (Plane == 0) {
                    *reinterpret_cast<uint4 *>(out + (m * out_ld + n)) = hi;
                    if (p.out_lo) *reinterpret_cast<uint4 *>(out_lo_plane + (m * out_ld + n)) = lo;
                }
                if (mirror) {
                    const uint4 q = Plane ? lo : hi;
                    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int k = 0; k < 8; ++k) turn[(n + k) * kTurnPitch<TT> + m] = static_cast<half_t>(w[k / 2] >> (16 * (k & 1)));
                }
            }
        }
    }
    if (!mirror) return squares;
    __syncthreads();
    half_t *image = p.out.of(matrix) + n0 * p.out.ld + m0 + Plane * p.out.plane;
    for (int i = threadIdx.x; i < TT::BN * TT::BM / 8; i += TT::NT) {
        const int r = i / (TT::BM / 8), c = i % (TT::BM / 8) * 8;
        if (r < cols_p && c < rows_p)
            *reinterpret_cast<uint4 *>(image + (r * out_ld + c)) = *reinterpret_cast<const uint4 *>(turn + r * kTurnPitch<TT> + c);
    }
    return squares;
}

// A finished tile of the last product: a wavefront's part in LDS, 64 rows at a time, and from there in whole lines of the
// output's rows, whichever way these run.  (Out of the accumulators this code, once per block, spilled all of them.)
constexpr int kLastPitch = 64 + 4;  // floats
template <typename TT> constexpr int kLastLds = TT::NWAVE * 64 * kLastPitch * 4;
template <typename TT>
__device__ __forceinline__ void store_last_product(const typename TT::Acc &acc, const OrthProduct &p, float beta, int64_t matrix, int64_t m0, int64_t n0,
                                                   char *lds) {
    static_assert(TT::WN == 64 && TT::WM % 64 == 0, "parts of 64 x 64");
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    float *part = reinterpret_cast<float *>(lds) + TT::wave_id() * 64 * kLastPitch;
    const half_t *d = p.d.of(matrix);
    __syncthreads();  // operands are no longer read; from here on every wavefront by itself
#pragma unroll
    for (int half = 0; half < TT::WM / 64; ++half) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < TT::FN; ++j)
                *reinterpret_cast<f32x4_t *>(part + (i * 16 + (lane & 15)) * kLastPitch + j * 16 + 4 * (lane >> 4)) = acc[half * 4 + i][j];
        __builtin_amdgcn_wave_barrier();
        const int64_t mp = m0 + TT::wave_m0() + half * 64, np = n0 + TT::wave_n0();
        constexpr int U = 2;  // runs of eight values per lane that are worked on at a time, their loads together
        for (int u0 = lane; u0 < 64 * 64 / 8; u0 += U * kWave) {
            uint4 hi[U], lo[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int u = u0 + i * kWave;
                const int64_t m = mp + u / 8, n = np + u % 8 * 8;
                const half_t *q = d + (m < p.Mp ? m : p.Mp - 1) * p.d.ld + (n < p.Np ? n : p.Np - 8);
                hi[i] = *reinterpret_cast<const uint4 *>(q);
                lo[i] = *reinterpret_cast<const uint4 *>(q + p.d.plane);
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int u = u0 + i * kWave, r = u / 8, c = u % 8 * 8;
                f32x4_t *q = reinterpret_cast<f32x4_t *>(part + r * kLastPitch + c);
                const f32x4_t x = q[0], y = q[1];
                Eight e;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    e.v[k] = x[k] * p.alpha;
                    e.v[4 + k] = y[k] * p.alpha;
                }
                e.add(beta, hi[i], lo[i]);
                if (p.last.across) {
                    q[0] = f32x4_t{e.v[0], e.v[1], e.v[2], e.v[3]};
                    q[1] = f32x4_t{e.v[4], e.v[5], e.v[6], e.v[7]};
                } else if (mp + r < p.M) {
                    store_last(p.last, matrix, mp + r, np + c, p.N, e);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
        if (p.last.across && mp + lane < p.M)  // a row per lane: whole lines of the output's rows
            for (int c = 0; c < 64; c += 8) {
                const f32x4_t *q = reinterpret_cast<const f32x4_t *>(part + lane * kLastPitch + c);
                const f32x4_t x = q[0], y = q[1];
                Eight e;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    e.v[k] = x[k];
                    e.v[4 + k] = y[k];
                }
                store_last(p.last, matrix, mp + lane, np + c, p.N, e);
            }
        __builtin_amdgcn_wave_barrier();
    }
}

// value = alpha * sum_k A(m,k) B(n,k) + beta * D for every matrix of a stack; rows of A lie along k, those of B too or
// (BCols) its columns.  Bound by the matrix cores where the contraction is long, then by what the ends of a tile read and
// write: at 4096 x 4096 x 4096 the symmetric products take 70-75 us (69 GFLOP: 0.95 PFLOP/s), the one that updates X 118
// (137 GFLOP, 1.16 PFLOP/s, with 134 MB of X in and out); at four of 1024 x 4096 x 1024 it takes 51 (34 GFLOP, again 134 MB).
template <typename TT, bool BCols, bool Split, bool Last>
__global__ void __launch_bounds__(TT::NT, 2)
orth_product_kernel(OrthProduct p) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const OrthTiles ord(p.Mp, p.Np, TT::BM, p.symmetric);
    const uint32_t tiles = static_cast<uint32_t>(ord.tiles());
    uint32_t i;
    if (!TileOrder::item(blockIdx.x, static_cast<uint32_t>(tiles * p.batch), i)) return;
    const int64_t matrix = i / tiles;
    int64_t tm, tn;
    ord.at(i % tiles, tm, tn);
    const int64_t m0 = tm * TT::BM, n0 = tn * TT::BN;
    __shared__ float scratch[TT::NWAVE];
    const float begun = begin_shift<TT::NT>(p, matrix, scratch);
    const half_t *a = p.a.of(matrix), *b = p.b.of(matrix);
    auto A = [&](int lo) { return typename TT::Operand{reinterpret_cast<const char *>(a + lo * p.a.plane), p.a.ld * 2, m0, p.Mp, 0}; };
    auto B = [&](int lo) { return typename TT::Operand{reinterpret_cast<const char *>(b + lo * p.b.plane), p.b.ld * 2, n0, p.Np, 0}; };
    typename TT::Acc acc;
    TT::zero(acc);
    if constexpr (Split) {
        TT::template mainloop<false, BCols, true>(A(0), B(1), p.KT, lds, acc);
        TT::template mainloop<false, BCols, true>(A(1), B(0), p.KT, lds, acc);
#pragma unroll
        for (int x = 0; x < TT::FM; ++x)
#pragma unroll
            for (int y = 0; y < TT::FN; ++y) acc[x][y] *= 1.0f / kLoScale;
    }
    TT::template mainloop<false, BCols, true>(A(0), B(0), p.KT, lds, acc);
    // (the main loop has barriers)
    const float shift = end_shift<TT::NT>(p, matrix, scratch, begun, m0 == 0 && n0 == 0);
    if constexpr (Last) return store_last_product<TT>(acc, p, beta_of(p, shift), matrix, m0, n0, lds);
    // (symmetric products have both operands along k)
    const float squares = store_product<TT, 0, !BCols>(acc, p, shift, matrix, m0, n0, lds);
    if constexpr (Split && !BCols) store_product<TT, 1, true>(acc, p, shift, matrix, m0, n0, lds);
    if constexpr (BCols)
        if (p.sq_out) store_squares<TT::NT>(p, matrix, tiles, i % tiles, squares);
}

// ----------------------------------------------------------------------------
// products with few tiles: every wavefront its own share of the contraction
// ----------------------------------------------------------------------------
// Tiles of 64 x 64, four wavefronts, each of which forms the whole tile over every fourth step of 64; their sums are added in
// order at the end.  What bounds a small product is the way of its operands: a step of the main loop above cannot be
// shorter than one round trip to the L2s (0.57 us), here each wavefront has a stage of its own, waits for nobody, and eight
// steps are on their way per compute unit (two workgroups; with two stages per wavefront and one workgroup no product was
// faster); a wavefront reads 16 KB of LDS per 32 matrix instructions (tiles shared between wavefronts: twice that).  The
// sides of all matrices are multiples of 64, so nothing here has an end to look after.
constexpr int kFewEdge = 64, kFewWaves = 4, kFewThreads = kFewWaves * kWave;
constexpr int kFewPanel = kFewEdge * kRowBytes;  // bytes: 64 rows of an operand (of one plane)
constexpr int kFewPitch = kFewEdge + 4;              // floats, of a wavefront's sums
constexpr int kFewSums = kFewEdge * kFewPitch * 4;
constexpr int few_stage(bool pairs) { return (pairs ? 4 : 2) * kFewPanel; }
constexpr int few_lds(bool pairs) { return kFewWaves * (few_stage(pairs) > kFewSums ? few_stage(pairs) : kFewSums); }

// Pairs: a stage holds both planes of both operands, read once for the three products; one workgroup per compute unit then.
// (Two workgroups, each product with a stage of its own: 704 x 704 x 47 steps 31 us instead of 25, 1024 x 1024 x 16 14.6
// instead of 14.0, 1536 x 1536 x 24 symmetric 33 either way.)
template <bool BCols, bool Pairs>
__global__ void __launch_bounds__(kFewThreads, Pairs ? 1 : 2)
orth_few_kernel(OrthProduct p) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    typedef Tile<256, 256, 2, 4, 16, true> T;  // its transfers and instruction
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef short v8s __attribute__((ext_vector_type(8)));
    constexpr int E = kFewEdge, F = E / 16, ROWS = kRowBytes;
    const OrthTiles ord(p.Mp, p.Np, E, p.symmetric);
    const uint32_t tiles = static_cast<uint32_t>(ord.tiles());
    uint32_t item;
    if (!TileOrder::item(blockIdx.x, static_cast<uint32_t>(tiles * p.batch), item)) return;
    const int64_t matrix = item / tiles;
    int64_t tm, tn;
    ord.at(item % tiles, tm, tn);
    const int64_t m0 = tm * E, n0 = tn * E;
    const int lane = threadIdx.x & 63, wave = T::wave_id();

    // transfers: instruction i of an operand brings rows 8 i .. 8 i + 7 of its stage, lane l the chunk that belongs at its place
    const int64_t lda = p.a.ld * 2, ldb = p.b.ld * 2;
    const char *a = reinterpret_cast<const char *>(p.a.of(matrix)) + m0 * lda;
    const char *b = reinterpret_cast<const char *>(p.b.of(matrix)) + (BCols ? n0 * 2 : n0 * ldb);
    const int64_t step_a = ROWS, step_b = BCols ? E * ldb : ROWS;
    constexpr int PLANES = Pairs ? 2 : 1;
    const char *stage = lds + wave * few_stage(Pairs);  // panels: A (hi, lo), B (hi, lo)
    const uint32_t ring = T::lds_address(stage);
    auto cols_swizzle = [](int r) { return (r & 3) << 1; };  // columns along k: pieces of four rows on distinct banks
    uint32_t off_a[2], off_b[2];  // of rows 0..7 and 8..15 of sixteen
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = 8 * h + (lane >> 3), c = lane & 7;
        off_a[h] = static_cast<uint32_t>((lane >> 3) * lda) + static_cast<uint32_t>((c ^ swz(r)) * 16);
        off_b[h] = static_cast<uint32_t>((lane >> 3) * ldb) + static_cast<uint32_t>((c ^ (BCols ? cols_swizzle(r) : swz(r))) * 16);
    }
    const int mine = (p.KT - wave + kFewWaves - 1) / kFewWaves;  // steps of this wavefront
    auto request = [&](int j) {
        const int kt = wave + kFewWaves * j;
        const uint32_t to = __builtin_amdgcn_readfirstlane(ring);
#pragma unroll
        for (int plane = 0; plane < PLANES; ++plane) {
            const char *ga = T::uniform(a + plane * p.a.plane * 2 + kt * step_a), *gb = T::uniform(b + plane * p.b.plane * 2 + kt * step_b);
#pragma unroll
            for (int i = 0; i < 8; ++i) T::dma(ga + i * 8 * lda, off_a[i & 1], to + plane * kFewPanel + i * 1024);
#pragma unroll
            for (int i = 0; i < 8; ++i) T::dma(gb + i * 8 * ldb, off_b[i & 1], to + (PLANES + plane) * kFewPanel + i * 1024);
        }
    };
    typename T::AccBlock acc[F][F], cross[Pairs ? F : 1][Pairs ? F : 1];  // cross: hi lo + lo hi
#pragma unroll
    for (int x = 0; x < F; ++x)
#pragma unroll
        for (int y = 0; y < F; ++y) {
            acc[x][y] = typename T::AccBlock{0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (Pairs) cross[x][y] = acc[x][y];
        }
    if (mine > 0) request(0);
    __shared__ float scratch[kFewWaves];
    // meanwhile: s, and the addend of the two runs of eight values that this thread will store
    const float begun = begin_shift<kFewThreads>(p, matrix, scratch);
    constexpr int U = E * E / 8 / kFewThreads;
    const half_t *d = p.d.base ? p.d.of(matrix) : nullptr;
    uint4 d_hi[U], d_lo[U];
    // (values that go out across: neighbouring lanes on neighbouring rows)
    auto run_row = [&](int i) { return p.last.across ? (i * kFewThreads + static_cast<int>(threadIdx.x)) % E : (i * kFewThreads + static_cast<int>(threadIdx.x)) / (E / 8); };
    auto run_col = [&](int i) { return 8 * (p.last.across ? (i * kFewThreads + static_cast<int>(threadIdx.x)) / E : (i * kFewThreads + static_cast<int>(threadIdx.x)) % (E / 8)); };
    if (d)
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const half_t *q = d + (m0 + run_row(i)) * p.d.ld + n0 + run_col(i);
            d_hi[i] = *reinterpret_cast<const uint4 *>(q);
            d_lo[i] = p.d_lo ? *reinterpret_cast<const uint4 *>(q + p.d.plane) : make_uint4(0u, 0u, 0u, 0u);
        }
    for (int j = 0; j < mine; ++j) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        bf16x8_t fa[PLANES][2][F], fb[PLANES][2][F];
#pragma unroll
        for (int plane = 0; plane < PLANES; ++plane)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const int chunk = ((4 * kk + (lane >> 4)) ^ swz(lane & 15)) * 16 + (lane & 15) * ROWS;
                const char *pa = stage + plane * kFewPanel, *pb = stage + (PLANES + plane) * kFewPanel;
#pragma unroll
                for (int f = 0; f < F; ++f) fa[plane][kk][f] = *reinterpret_cast<const bf16x8_t *>(pa + f * 16 * ROWS + chunk);
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    if constexpr (BCols) {  // see Tile::Side
                        const int row = 32 * kk + 8 * (lane >> 4) + ((lane & 15) >> 2), col = f * 16 + 4 * (lane & 3);
                        const uint32_t at = T::lds_address(pb) + row * ROWS + (((col >> 3) ^ cols_swizzle(row)) << 4) + ((col >> 2) & 1) * 8;
                        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s __attribute__((address_space(3))) *)(uintptr_t)at);
                        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s __attribute__((address_space(3))) *)(uintptr_t)(at + 4 * ROWS));
                        fb[plane][kk][f] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    } else {
                        fb[plane][kk][f] = *reinterpret_cast<const bf16x8_t *>(pb + f * 16 * ROWS + chunk);
                    }
                }
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage is in registers: its place may be written
        __builtin_amdgcn_sched_barrier(0);
        if (j + 1 < mine) request(j + 1);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int x = 0; x < F; ++x)
#pragma unroll
                for (int y = 0; y < F; ++y) {
                    acc[x][y] = T::template mfma<true>(fa[0][kk][x], fb[0][kk][y], acc[x][y]);
                    if constexpr (Pairs) {
                        cross[x][y] = T::template mfma<true>(fa[0][kk][x], fb[1][kk][y], cross[x][y]);
                        cross[x][y] = T::template mfma<true>(fa[1][kk][x], fb[0][kk][y], cross[x][y]);
                    }
                }
    }
    if constexpr (Pairs)
#pragma unroll
        for (int x = 0; x < F; ++x)
#pragma unroll
            for (int y = 0; y < F; ++y) acc[x][y] += cross[x][y] * (1.0f / kLoScale);
    // the wavefronts' sums in LDS: lane l holds row l % 16 and columns 4 (l / 16) .. of a block
    __syncthreads();
    float *sums = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int x = 0; x < F; ++x)
#pragma unroll
        for (int y = 0; y < F; ++y)
            *reinterpret_cast<f32x4_t *>(sums + (wave * E + x * 16 + (lane & 15)) * kFewPitch + y * 16 + 4 * (lane >> 4)) = acc[x][y];
    __syncthreads();
    const float shift = end_shift<kFewThreads>(p, matrix, scratch, begun, m0 == 0 && n0 == 0), beta = beta_of(p, shift);
    half_t *out = p.out.base ? p.out.of(matrix) : nullptr;
    const bool mirror = p.symmetric && m0 != n0;
    uint4 hi[U], lo[U];
    int row[U], at[U];
    float squares = 0.0f;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int r = row[i] = run_row(i), c = at[i] = run_col(i);
        Eight e;
#pragma unroll
        for (int k = 0; k < 8; ++k) e.v[k] = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
            const f32x4_t *q = reinterpret_cast<const f32x4_t *>(sums + (w * E + r) * kFewPitch + c);
            const f32x4_t x = q[0], y = q[1];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                e.v[k] += x[k];
                e.v[4 + k] += y[k];
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) e.v[k] *= p.alpha;
        const int64_t m = m0 + r, n = n0 + c;
        if (d) e.add(beta, d_hi[i], d_lo[i]);
        if (p.last.out) {
            if (m < p.M) store_last(p.last, matrix, m, n, p.N, e);
            continue;
        }
        if (p.n_sq && m0 == n0) off_diagonal(shift * kGramScale, r, c, e);
        clear_padding(p, m, n, e);
#pragma unroll
        for (int k = 0; k < 8; ++k) squares = fmaf(e.v[k], e.v[k], squares);
        e.split(hi[i], lo[i]);
        *reinterpret_cast<uint4 *>(out + m * p.out.ld + n) = hi[i];
        if (p.out_lo) *reinterpret_cast<uint4 *>(out + p.out.plane + m * p.out.ld + n) = lo[i];
    }
    if (p.sq_out) return store_squares<kFewThreads>(p, matrix, tiles, item % tiles, squares);
    if (!mirror) return;
    // the mirror image, turned in LDS (a pitch of 33 words: the writes of a wavefront on 32 different banks)
    constexpr int P = E + 2;
    half_t *turn = reinterpret_cast<half_t *>(lds);
    __syncthreads();  // the sums are no longer read
#pragma unroll
    for (int plane = 0; plane < 2; ++plane) {
        if (plane && !p.out_lo) break;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint4 q = plane ? lo[i] : hi[i];
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) turn[(plane * E + at[i] + k) * P + row[i]] = static_cast<half_t>(w[k / 2] >> (16 * (k & 1)));
        }
    }
    __syncthreads();
#pragma unroll
    for (int plane = 0; plane < 2; ++plane) {
        if (plane && !p.out_lo) break;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint32_t *q = reinterpret_cast<const uint32_t *>(turn + (plane * E + row[i]) * P + at[i]);
            *reinterpret_cast<uint4 *>(out + plane * p.out.plane + (n0 + row[i]) * p.out.ld + m0 + at[i]) = make_uint4(q[0], q[1], q[2], q[3]);
        }
    }
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
constexpr int kNormParts = 1024;  // most workgroups per matrix; 256 threads join their sums

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

// part[matrix][workgroup] = sum of squares of its share of U; the momentum is written on the way.  Bound by HBM: four of
// 4096 x 1024 with momentum 168 MB in 29.8 us = 5.6 TB/s.
__global__ void __launch_bounds__(256) orth_norm_kernel(OrthInput in, double *__restrict__ part) {
    __shared__ double scratch[4];
    const int64_t matrix = blockIdx.y;
    const uint32_t per_row = static_cast<uint32_t>(ceil_div(in.cols, 8)), n = static_cast<uint32_t>(in.rows) * per_row;  // (2^29 at most)
    double sum = 0.0;
#pragma unroll 2
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
        float u[8];
        load_update<true>(in, matrix, i / per_row, i % per_row * 8, u);
        double s[2] = {0.0, 0.0};  // (in 64 bits: any fp32 entry's square is a number there)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k & 1] = fma(static_cast<double>(u[k]), static_cast<double>(u[k]), s[k & 1]);
        sum += s[0] + s[1];
    }
    sum = block_sum(sum, scratch);
    if (threadIdx.x == 0) part[matrix * gridDim.x + blockIdx.x] = sum;
}

// scale / (|U| + eps), 0 for a matrix of zeros, NaN for one with an infinity or a NaN; by a whole workgroup
// sq (NULL: not): the sum of X's squares.
__device__ __forceinline__ double scale_of(const OrthInput &in, const double *part, int parts, int64_t matrix, float scale, double *scratch, float *sq) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) sum += part[matrix * parts + i];
    const double norm = sqrt(block_sum(sum, scratch));
    const double whole = norm + static_cast<double>(in.eps);
    const double f = whole == 0.0 ? 0.0 : whole < __builtin_inf() ? scale / whole : __builtin_nan("");
    if (sq && blockIdx.x == 0 && threadIdx.x == 0) sq[matrix] = static_cast<float>((norm * f) * (norm * f));
    return f;
}

// X = scale * U / (|U| + eps) as pairs of halves, zero in the padding; with last.out: U / (|U| + eps) goes there (no steps).
// Every workgroup adds the parts of the norm up for itself, in the same order, while its first loads are on their way: one
// launch less.  4096 x 4096 in bf16: 101 MB in 20.5 us = 4.9 TB/s; small matrices 7 to 10 us, half of it the norm's chain.
__global__ void __launch_bounds__(256) orth_scale_kernel(OrthInput in, const double *__restrict__ part, int parts, float scale, Stack X,
                                                         int64_t rows_p, OrthOut last, float *__restrict__ sq) {
    __shared__ double scratch[4];
    const int64_t matrix = blockIdx.y;
    const uint32_t per_row = static_cast<uint32_t>(X.ld / 8), n = static_cast<uint32_t>(rows_p) * per_row, stride = gridDim.x * 256;
    auto load = [&](uint32_t i, float (&u)[8]) {
        const int64_t r = i / per_row, c = i % per_row * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) u[k] = 0.0f;
        if (i < n && r < in.rows && c < in.cols) load_update<false>(in, matrix, r, c, u);
    };
    uint32_t i = blockIdx.x * 256 + threadIdx.x;
    float u[8];
    load(i, u);  // on their way while the norm is formed
    const double f = scale_of(in, part, parts, matrix, last.out ? 1.0f : scale, scratch, sq);
    half_t *x = X.of(matrix);
    while (i < n) {
        const int64_t r = i / per_row, c = i % per_row * 8;
        Eight e;
#pragma unroll
        for (int k = 0; k < 8; ++k) e.v[k] = static_cast<float>(u[k] * f);
        i += stride;
        load(i, u);
        if (last.out) {
            if (r < in.rows && c < in.cols) store_last(last, matrix, r, c, in.cols, e);
            continue;
        }
        uint4 hi, lo;
        e.split(hi, lo);
        *reinterpret_cast<uint4 *>(x + r * X.ld + c) = hi;
        *reinterpret_cast<uint4 *>(x + X.plane + r * X.ld + c) = lo;
    }
}

// The same for matrices with more rows than columns: X gets their transpose, 64 x 64 entries by a workgroup through LDS.  Four of
// 4096 x 1024 with momentum: 168 MB in 32.6 us = 5.2 TB/s.
__global__ void __launch_bounds__(256) orth_scale_turned_kernel(OrthInput in, const double *__restrict__ part, int parts, float scale, Stack X,
                                                                unsigned across, float *__restrict__ sq) {
    __shared__ double scratch[4];
    __shared__ float turn[64][65];
    const int64_t matrix = blockIdx.y;
    const int64_t r0 = blockIdx.x % across * 64, c0 = blockIdx.x / across * 64;  // of U; across: tiles along X's rows
    float v[2][8] = {};
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // on their way while the norm is formed
        const int u = i * 256 + threadIdx.x, r = u / 8, c = u % 8 * 8;
        if (r0 + r < in.rows && c0 + c < in.cols) load_update<false>(in, matrix, r0 + r, c0 + c, v[i]);
    }
    const double f = scale_of(in, part, parts, matrix, scale, scratch, sq);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int u = i * 256 + threadIdx.x, r = u / 8, c = u % 8 * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) turn[r][c + k] = static_cast<float>(v[i][k] * f);
    }
    __syncthreads();
    half_t *x = X.of(matrix);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int u = i * 256 + threadIdx.x, r = u / 8, c = u % 8 * 8;  // of X
        Eight e;
#pragma unroll
        for (int k = 0; k < 8; ++k) e.v[k] = turn[c + k][r];
        uint4 hi, lo;
        e.split(hi, lo);
        *reinterpret_cast<uint4 *>(x + (c0 + r) * X.ld + r0 + c) = hi;
        *reinterpret_cast<uint4 *>(x + X.plane + (c0 + r) * X.ld + r0 + c) = lo;
    }
}

// ----------------------------------------------------------------------------
// host side
// ----------------------------------------------------------------------------
static_assert(kStep == kBK, "steps of the main loop");

struct OrthPlan {
    int64_t k, L, kp, Lp;  // the smaller and the larger side, and both padded: X is k x L
    int parts;
    double *norm;
    float *sq, *shift;     // see OrthProduct
    Stack X[2], A, B;
    float x_scale;
    size_t bytes;
};

static OrthPlan plan_orth(const spo_orth_desc *d, void *ws) {
    OrthPlan p;
    p.k = std::min(d->rows, d->cols);
    p.L = std::max(d->rows, d->cols);
    p.kp = padded(p.k);
    p.Lp = padded(p.L);
    // X's entries are about 1 / sqrt(longer side) once its singular values are near one
    p.x_scale = 1.0f;
    for (int64_t n = p.L; n > 1; n /= 4) p.x_scale *= 2.0f;
    const int64_t vectors = d->rows * ceil_div(d->cols, 8);
    p.parts = static_cast<int>(std::min<int64_t>(kNormParts, ceil_div(vectors, 256 * 2)));
    Arena a(ws);
    p.norm = a.take<double>(static_cast<size_t>(d->batch) * kNormParts);
    p.sq = a.take<float>(static_cast<size_t>(d->batch) * square_room(p.kp, p.Lp));
    p.shift = a.take<float>(d->batch);
    auto stack = [&](int64_t rows, int64_t ld) {
        Stack s{nullptr, ld, rows * ld, 2 * rows * ld};
        s.base = a.take<half_t>(static_cast<size_t>(d->batch) * 2 * rows * ld);
        return s;
    };
    p.X[0] = stack(p.kp, p.Lp);
    p.X[1] = stack(p.kp, p.Lp);
    p.A = stack(p.kp, p.kp);
    p.B = stack(p.kp, p.kp);
    p.bytes = a.used;
    return p;
}

template <typename TT, bool BCols, bool Split>
static int launch_tiles(const OrthProduct &p, hipStream_t s) {
    auto *kernel = orth_product_kernel<TT, BCols, Split, false>;
    int lds = kOrthLds<TT>;
    if constexpr (BCols)
        if (p.last.out) {
            kernel = orth_product_kernel<TT, BCols, Split, true>;
            lds = std::max(TT::LDS_BYTES, kLastLds<TT>);
        }
    if (int rc = allow_lds(kernel, lds)) return rc;
    const int64_t items = OrthTiles(p.Mp, p.Np, TT::BM, p.symmetric).tiles() * p.batch;
    kernel<<<static_cast<unsigned>(TileOrder::blocks(items)), TT::NT, lds, s>>>(p);
    return SPO_OK;
}
template <bool BCols, bool Pairs>
static int launch_few(const OrthProduct &p, hipStream_t s) {
    auto *kernel = orth_few_kernel<BCols, Pairs>;
    if (int rc = allow_lds(kernel, few_lds(Pairs))) return rc;
    const int64_t items = OrthTiles(p.Mp, p.Np, kFewEdge, p.symmetric).tiles() * p.batch;
    kernel<<<static_cast<unsigned>(TileOrder::blocks(items)), kFewThreads, few_lds(Pairs), s>>>(p);
    return SPO_OK;
}
template <typename TT, bool BCols>
static int launch_tiles(const OrthProduct &p, hipStream_t s) {
    return p.split ? launch_tiles<TT, BCols, true>(p, s) : launch_tiles<TT, BCols, false>(p, s);
}
static_assert(OS::BM == kOrthEdge[1] && OS::NWAVE == kOrthWaves[1] && OM::BM == kOrthEdge[2] && OM::NWAVE == kOrthWaves[2] &&
                  OL::BM == kOrthEdge[3] && OL::NWAVE == kOrthWaves[3] && kFewEdge == kOrthEdge[0] && kFewWaves == kOrthWaves[0],
              "orth_choice.hpp knows the kernels' tiles");
template <bool BCols>
static int launch_product(const OrthProduct &p, Kind kind, hipStream_t s) {
    if (kind == Kind::few) return p.split ? launch_few<BCols, true>(p, s) : launch_few<BCols, false>(p, s);
    if (kind == Kind::small) return launch_tiles<OS, BCols>(p, s);
    if constexpr (!BCols)  // (tiles of 192 take rows along the contraction only)
        if (kind == Kind::middle) return launch_tiles<OM, BCols>(p, s);
    return launch_tiles<OL, BCols>(p, s);
}

static int run_orth(const spo_orth_desc *d, const OrthInput &in, OrthOut last, void *ws, size_t ws_bytes, hipStream_t s) {
    const OrthPlan p = plan_orth(d, ws);
    if (ws_bytes < p.bytes) return SPO_EWORKSPACE;
    const bool tall = d->rows > d->cols;
    const unsigned batch = static_cast<unsigned>(d->batch);
    orth_norm_kernel<<<dim3(static_cast<unsigned>(p.parts), batch), 256, 0, s>>>(in, p.norm);
    if (tall && d->steps) {
        orth_scale_turned_kernel<<<dim3(static_cast<unsigned>(p.Lp / 64 * (p.kp / 64)), batch), 256, 0, s>>>(in, p.norm, p.parts, p.x_scale,
                                                                                                           p.X[0], static_cast<unsigned>(p.Lp / 64), p.sq);
    } else {
        const int64_t vectors = p.kp * p.Lp / 8;
        const int64_t x_rows = d->steps ? p.kp : d->rows;
        orth_scale_kernel<<<dim3(static_cast<unsigned>(std::min<int64_t>(1024, ceil_div(vectors, 256))), batch), 256, 0, s>>>(
            in, p.norm, p.parts, p.x_scale, p.X[0], x_rows, d->steps ? OrthOut{} : last, p.sq);
    }
    last.across = tall;
    const bool split = as_pairs(p.k, d->products == SPO_PRODUCTS_SPLIT);
    // A' = X X^T - s I
    OrthProduct gram{};
    gram.batch = d->batch;
    gram.split = gram.d_lo = gram.out_lo = split;
    gram.shift = p.shift;
    gram.symmetric = 1;
    gram.out = p.A;
    gram.M = gram.N = p.k;
    gram.Mp = gram.Np = p.kp;
    gram.KT = static_cast<int>(p.Lp / kBK);
    gram.alpha = kGramScale / (p.x_scale * p.x_scale);
    gram.sq = p.sq;
    gram.sq_scale = 1.0f / (p.x_scale * p.x_scale * static_cast<float>(p.k));
    // B' = (b + 2 c s) A' + c A' A'; A' is symmetric, so its rows serve as columns
    OrthProduct poly = gram;
    poly.n_sq = 0;
    poly.a = poly.b = poly.d = p.A;
    poly.out = p.B;
    poly.KT = static_cast<int>(p.kp / kBK);
    poly.alpha = d->c / kGramScale;
    poly.c[0] = d->b;
    poly.c[1] = 2.0f * d->c;
    // X <- (a + b s + c s^2) X + B' X
    OrthProduct update = poly;
    update.symmetric = 0;
    update.a = p.B;
    update.d_lo = update.out_lo = 1;
    update.N = p.L;
    update.Np = p.Lp;
    update.alpha = 1.0f / kGramScale;
    update.c[0] = d->a;
    update.c[1] = d->b;
    update.c[2] = d->c;
    update.sq_out = p.sq;
    const OrthKinds kinds = orth_kinds(p.kp, p.Lp, d->batch, split);
    for (int i = 0; i < d->steps; ++i) {
        const Stack &X = p.X[i & 1];
        gram.a = gram.b = X;
        gram.n_sq = i == 0 ? 1 : static_cast<int>(square_sums(p.kp, p.Lp, kinds.update));
        if (int rc = launch_product<false>(gram, kinds.gram, s)) return rc;
        if (int rc = launch_product<false>(poly, kinds.poly, s)) return rc;
        update.b = update.d = X;
        update.out = p.X[(i + 1) & 1];
        if (i == d->steps - 1) {
            update.alpha /= p.x_scale;
            for (float &c : update.c) c /= p.x_scale;
            update.sq_out = nullptr;
            update.last = last;
        }
        if (int rc = launch_product<true>(update, kinds.update, s)) return rc;
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
    return run_orth(d, in, OrthOut{out, out_dtype, 0, 0, d->cols, d->rows * d->cols, 0.0f, 0.0f}, ws, ws_bytes, as_stream(stream));
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
    return run_orth(d, in, OrthOut{W, w_dtype, 1, 0, d->cols, d->rows * d->cols, keep, lr * scale}, ws, ws_bytes, as_stream(stream));
}
