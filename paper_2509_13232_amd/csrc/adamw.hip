// AdamW over many tensors at once, the norm of their gradients, and the values of a state that is held in 8 bits.
//
//   g' = g min(1, max_norm / norm);  m <- b1 m + (1 - b1) g';  v <- b2 v + (1 - b2) g'^2;  r = sqrt v
//   p <- p - (lr / (1 - b1^t) m / (r / sqrt(1 - b2^t) + eps) + lr wd p)
//
// One pass over the elements, every one of which is read and written once: HBM.  What the kernels are told of the tensors
// travels in the launches' arguments, so a captured graph holds it and nothing is kept between calls.  Moments are chains of
// single roundings to fp32 (no contracted multiply-add): their codes in 8 bits have one answer on any machine.
#include <algorithm>
#include <cmath>
#include <limits>

#include "state8.hpp"
#include "vec8.hpp"

namespace spo {

constexpr int kThreads = 256;
constexpr int64_t kMostElements = int64_t(1) << 35, kMostTensors = int64_t(1) << 24;
constexpr size_t kTableBytes = 3840;  // of a launch's 4 KiB of arguments

struct Tensor32 {
    static constexpr int kChunk = kThreads * 4;  // elements that a workgroup takes: four per thread
    void *param;
    const void *grad;
    float *m, *v;
    bf16_t *copy;
    int64_t n;
    double decay;
    int32_t first, types;  // its first chunk of the launch; bit 0: param is bf16, bit 1: grad is bf16
};
struct Tensor8 {
    static constexpr int kChunk = kThreads * 8 * 4;  // four eights per thread
    void *param;
    const void *grad;
    uint8_t *m, *v;
    uint8_t *m_scale, *v_scale;
    bf16_t *copy;
    int64_t n;
    double decay;
    int32_t first, types;
};
struct TensorNorm {
    static constexpr int kChunk = kThreads * 8 * 2;
    const void *grad;
    int64_t n;
    int32_t first, types;
};
template <typename T>
struct Table {
    static constexpr int kMost = kTableBytes / sizeof(T);
    static_assert(kMost * (kMostElements / T::kChunk) < INT32_MAX, "chunks of a launch");
    T t[kMost];
    int32_t count, chunks;
    // the tensor of a chunk
    __device__ __forceinline__ int find(int chunk) const {
        int lo = 0, hi = count;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (t[mid].first <= chunk) lo = mid;
            else hi = mid;
        }
        return lo;
    }
};

// What a step's elements are told; on the device where the step's number or the rate is only known there.
struct AdamwStep {
    double lr;
    float rate, root_scale;  // lr / (1 - b1^t), (1 - b2^t)^-1/2
    uint32_t step;
};
struct AdamwScalars {
    float b1, c1, b2, c2, eps;  // c = 1 - b
    int rounding;
    const float *norm;
    float max_norm;
    AdamwStep step;
    const AdamwStep *on_device;  // or NULL: `step` holds
};

static __host__ __device__ AdamwStep step_of(double lr, double beta1, double beta2, int64_t t) {
    AdamwStep s;
    s.lr = lr;
    s.rate = static_cast<float>(lr / -expm1(static_cast<double>(t) * log(beta1)));
    s.root_scale = static_cast<float>(1.0 / sqrt(-expm1(static_cast<double>(t) * log(beta2))));
    s.step = static_cast<uint32_t>(t);
    return s;
}

__global__ void adamw_prepare_kernel(double lr, const float *lr_device, double beta1, double beta2, int64_t t, int64_t *t_device, const float *norm,
                                     AdamwStep *out) {
    if (t_device) {
        t = *t_device + 1;
        if (!norm || isfinite(*norm)) *t_device = t;  // (as the step's kernel decides whether anything moves)
    }
    *out = step_of(lr_device ? static_cast<double>(*lr_device) : lr, beta1, beta2, t);
}

__device__ __forceinline__ float first_moment(float m, float g, const AdamwScalars &a) {
#pragma clang fp contract(off)
    return m * a.b1 + g * a.c1;
}
__device__ __forceinline__ float second_moment(float v, float g, const AdamwScalars &a) {
#pragma clang fp contract(off)
    return v * a.b2 + g * g * a.c2;
}
template <int N>
__device__ __forceinline__ void new_weights(float (&p)[N], const float (&change)[N], float decay) {
    if (decay != 0.0f) {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] -= fmaf(p[i], decay, change[i]);
    } else {  // (an infinite weight stays)
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] -= change[i];
    }
}

// A weight's new value in its type, by the step's thresholds (state8.hpp) where that is asked for; what is not finite, to nearest.
__device__ __forceinline__ float by_threshold(float x, uint32_t turn) {
    const uint32_t u = __float_as_uint(x);
    return (u & 0x7f800000u) == 0x7f800000u ? x : __uint_as_float((u + (turn >> 16)) & 0xffff0000u);
}
template <int N>
__device__ __forceinline__ void thresholds(float (&x)[N], uint32_t step, uint32_t place) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = by_threshold(x[i], turn_at(turn_of(step, kTurnWeight), place + i));
}

struct Codes {
    uint32_t u[2];
};
__device__ __forceinline__ Codes load_codes(const uint8_t *p, int n) {
    Codes c;
    if (n >= 8) {
        typedef uint32_t V __attribute__((ext_vector_type(2), aligned(1)));
        const V v = *reinterpret_cast<const V *>(p);
        c.u[0] = v.x, c.u[1] = v.y;
        return c;
    }
    c.u[0] = c.u[1] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) c.u[i / 4] |= static_cast<uint32_t>(p[i]) << 8 * (i & 3);
    return c;
}
__device__ __forceinline__ void store_codes(uint8_t *p, const Codes &c, int n) {
    if (n >= 8) {
        typedef uint32_t V __attribute__((ext_vector_type(2), aligned(1)));
        *reinterpret_cast<V *>(p) = V{c.u[0], c.u[1]};
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = static_cast<uint8_t>(c.u[i / 4] >> 8 * (i & 3));
}
template <typename C>
__device__ __forceinline__ float code_at(const Codes &c, int i) { return C::unscaled(c.u[i / 4] >> 8 * (i & 3) & 0xff); }
template <typename C>
__device__ __forceinline__ void decode8(const Codes &c, uint32_t scale, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = ldexpf(code_at<C>(c, i), static_cast<int>(scale) - 15);
    if (__any(scale == kNotFinite)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = scale == kNotFinite ? __uint_as_float(0x7fc00000u) : x[i];
    }
}
// The largest of a value over eight neighbouring lanes, for all of them: lanes exchanged in fours, then the halves of eight.
__device__ __forceinline__ uint32_t max_of_eight_lanes(uint32_t v) {
    constexpr int kSwapPairs = 0xb1, kSwapTwos = 0x4e, kMirrorHalfRow = 0x141;
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), kSwapPairs, 0xf, 0xf, true)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), kSwapTwos, 0xf, 0xf, true)));
    return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), kMirrorHalfRow, 0xf, 0xf, true)));
}
// The codes of a thread's eight elements and the scale of their block, which eight neighbouring lanes hold together.
struct Coded {
    uint32_t word[8];  // (codes in the uppermost bytes)
    uint32_t top, scale;
    __device__ __forceinline__ Codes codes() const {
        Codes c;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            c.u[h] = __builtin_amdgcn_perm(word[4 * h + 1], word[4 * h], 0x0c0c0703) | __builtin_amdgcn_perm(word[4 * h + 3], word[4 * h + 2], 0x0c0c0703) << 16;
        return c;
    }
};
template <typename C>
__device__ __forceinline__ Coded encode8(const float (&x)[8], const uint32_t (&threshold)[8]) {
    Coded c;
    c.top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) c.top = max(c.top, C::magnitude(x[i]));
    c.top = max_of_eight_lanes(c.top);
    c.scale = C::scale(c.top);
#pragma unroll
    for (int i = 0; i < 8; ++i) c.word[i] = C::encode(x[i], c.scale, threshold[i]);
    return c;
}

// Roots and their codes.  The hardware's root is off by a place at most; a rounded one takes twice the instructions of all the
// rest of its code.  Its last place decides a code only where root and threshold together lie within a place of the next code
// (one value of 2^18), or the block's largest within a place of the next scale: then, and where a square is so small that the
// hardware's root is not good, the wavefront's roots are made again.  (Vector instructions per element of the whole kernel: 56.5 with
// rounded roots throughout, 47 so.)
__device__ __forceinline__ Coded encode_roots(const float (&v)[8], float (&root)[8], const uint32_t (&threshold)[8]) {
    constexpr uint32_t kSmall = 0x0f800000;  // 2^-96
    constexpr uint32_t kPlace = 1u << (24 - RootCode::kDrop);  // of a magnitude, in a code's word
    uint32_t least = 0xffffffffu, nearest = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        root[i] = __builtin_amdgcn_sqrtf(v[i]);
        least = min(least, __float_as_uint(v[i]) - 1u);  // (zero is none of the small ones)
    }
    Coded c = encode8<RootCode>(root, threshold);
#pragma unroll
    for (int i = 0; i < 8; ++i) nearest = min(nearest, (RootCode::word(root[i], c.scale, threshold[i]) + kPlace) << 8);
    const uint32_t to_scale = (c.top + (1u << RootCode::kDrop)) << 9;
    if (__any(least < kSmall || nearest <= kPlace << 8 || to_scale <= 1u << 9)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) root[i] = sqrtf(v[i]);
        c = encode8<RootCode>(root, threshold);
    }
    return c;
}

// What the elements of a workgroup share.
struct Shared {
    float factor, decay;
    AdamwStep step;
};

// 32-bit states: four elements per thread and no more, so that what is read and written at a time lies together (two fours per
// thread: 595 us instead of 551 for 151936 x 1024 in bf16, four 579; eights of neighbours, whose fp32 lines are asked for twice, 682).
template <typename TP, typename TG, bool Stream>
__device__ __forceinline__ void update32(const Tensor32 &t, int64_t begin, const AdamwScalars &a, const Shared &s) {
    const int64_t at = begin + threadIdx.x * 4;
    const int some = within4(at, t.n);
    if (!some) return;
    TP *const param = static_cast<TP *>(t.param) + at;
    float p[4], g[4], m[4], v[4], change[4];
    load4(p, param, some);
    load4(g, static_cast<const TG *>(t.grad) + at, some);
    load4<Stream>(m, t.m + at, some);
    load4<Stream>(v, t.v + at, some);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float gi = g[i] * s.factor;
        m[i] = first_moment(m[i], gi, a);
        v[i] = second_moment(v[i], gi, a);
        change[i] = m[i] / (sqrtf(v[i]) * s.step.root_scale + a.eps) * s.step.rate;
    }
    new_weights(p, change, s.decay);
    store4<Stream>(t.m + at, m, some);
    store4<Stream>(t.v + at, v, some);
    if (sizeof(TP) == 2 && a.rounding != SPO_ROUND_NEAREST) thresholds(p, s.step.step, static_cast<uint32_t>(at) % kStateBlock);
    store4(param, p, some);
    if (t.copy) store4(t.copy + at, p, some);
}

// 8-bit states.  Eight lanes hold a block, so that its scales are three moves between lanes away (151936 x 4096 in bf16: 1065-1126 us,
// 10 bytes per element at 5.6-5.9 TB/s).  Whole: the workgroup's elements are all there.  (Weights and gradients in fp32 take no
// non-temporal hint: both halves of a line are asked for, one after the other.)
template <typename TP, typename TG, bool Whole, bool Stream>
__device__ __forceinline__ void update8(const Tensor8 &t, int64_t begin, const AdamwScalars &a, const Shared &s) {
    const int64_t end = std::min<int64_t>(begin + Tensor8::kChunk, t.n);
    uint32_t first_threshold[8], root_threshold[8];  // a thread's places of a block stay the same
    const uint32_t place = threadIdx.x * 8 % kStateBlock;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        first_threshold[i] = FirstCode::threshold(turn_at(turn_of(s.step.step, kTurnFirst), place + i));
        root_threshold[i] = RootCode::threshold(turn_at(turn_of(s.step.step, kTurnRoot), place + i));
    }
    int64_t at = begin + threadIdx.x * 8;
    for (int64_t wave = at - threadIdx.x % kWave * 8; wave < end; wave += kThreads * 8, at += kThreads * 8) {  // whole wavefronts
        const int some = Whole ? 8 : within(at, t.n);
        Raw8<TP> raw_p;
        Raw8<TG> raw_g;
        load_some<Stream && sizeof(TP) == 2>(raw_p, static_cast<const TP *>(t.param) + at, some);
        load_some<Stream && sizeof(TG) == 2>(raw_g, static_cast<const TG *>(t.grad) + at, some);
        const Codes old_m = load_codes(t.m + at, some), old_v = load_codes(t.v + at, some);
        const uint32_t m_scale = some ? t.m_scale[at / kStateBlock] : 0, v_scale = some ? t.v_scale[at / kStateBlock] : 0;
        float p[8], g[8], m[8], v[8], root[8], change[8];
        raw_floats(raw_p, p);
        raw_floats(raw_g, g);
        if (s.factor != 1.0f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] *= s.factor;
        }
        decode8<FirstCode>(old_m, m_scale, m);
        decode8<RootCode>(old_v, v_scale, root);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = first_moment(m[i], g[i], a);
            v[i] = second_moment(root[i] * root[i], g[i], a);
        }
        const Coded first = encode8<FirstCode>(m, first_threshold), second = encode_roots(v, root, root_threshold);
        store_codes(t.m + at, first.codes(), some);
        store_codes(t.v + at, second.codes(), some);
        if (some && place == 0) {
            t.m_scale[at / kStateBlock] = static_cast<uint8_t>(first.scale);
            t.v_scale[at / kStateBlock] = static_cast<uint8_t>(second.scale);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)  // (a root is zero or 2^-75 and more: the reciprocal takes every such divisor)
            change[i] = m[i] * __builtin_amdgcn_rcpf(fmaf(root[i], s.step.root_scale, a.eps)) * s.step.rate;
        new_weights(p, change, s.decay);
        if (sizeof(TP) == 2 && a.rounding != SPO_ROUND_NEAREST) thresholds(p, s.step.step, place);
        store_some<Stream && sizeof(TP) == 2>(static_cast<TP *>(t.param) + at, p, some);
        if (t.copy) store_some<Stream>(t.copy + at, p, some);
    }
}
template <typename TP, typename TG, bool Stream>
__device__ __forceinline__ void update8(const Tensor8 &t, int64_t begin, const AdamwScalars &a, const Shared &s) {
    if (begin + Tensor8::kChunk <= t.n) update8<TP, TG, true, Stream>(t, begin, a, s);
    else update8<TP, TG, false, Stream>(t, begin, a, s);
}

template <typename TP, typename TG, bool Stream>
__device__ __forceinline__ void update(const Tensor32 &t, int64_t begin, const AdamwScalars &a, const Shared &s) { update32<TP, TG, Stream>(t, begin, a, s); }
template <typename TP, typename TG, bool Stream>
__device__ __forceinline__ void update(const Tensor8 &t, int64_t begin, const AdamwScalars &a, const Shared &s) { update8<TP, TG, Stream>(t, begin, a, s); }

template <typename T, bool Stream>
__global__ void __launch_bounds__(kThreads) adamw_kernel(Table<T> table, AdamwScalars a) {
    const int64_t block = flat_block();
    if (block >= table.chunks) return;
    Shared s;
    s.factor = 1.0f;
    if (a.norm) {
        const float norm = *a.norm;
        if (!isfinite(norm)) return;  // nothing moves
        if (norm > a.max_norm) s.factor = a.max_norm / norm;
    }
    s.step = a.on_device ? *a.on_device : a.step;
    const T t = table.t[table.find(static_cast<int>(block))];
    s.decay = static_cast<float>(s.step.lr * t.decay);
    const int64_t begin = (block - t.first) * T::kChunk;
    switch (t.types) {
        case 0: return update<float, float, Stream>(t, begin, a, s);
        case 1: return update<bf16_t, float, Stream>(t, begin, a, s);
        case 2: return update<float, bf16_t, Stream>(t, begin, a, s);
        default: return update<bf16_t, bf16_t, Stream>(t, begin, a, s);
    }
}

// --------------------------------------------------------------------------------------------- norm of the gradients
constexpr int kNormParts = 2048;  // workgroups of a launch

template <int N>
__device__ __forceinline__ double squares(const float (&g)[N], double sum) {
#pragma unroll
    for (int i = 0; i < N; ++i) sum = fma(static_cast<double>(g[i]), static_cast<double>(g[i]), sum);
    return sum;
}
// Squares of fp32 numbers are exact in 64 bits, and so nearly are their sums: the norm is the rounded true one.  (78 million gradients
// in bf16: 31 us where the Infinity Cache holds them; 44-49 behind a step that left it full of lines to be written back.)
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(Table<TensorNorm> table, double *__restrict__ parts) {
    __shared__ double scratch[kThreads / kWave];
    double sum = 0.0;
    for (int chunk = blockIdx.x; chunk < table.chunks; chunk += gridDim.x) {
        const TensorNorm t = table.t[table.find(chunk)];
        const int64_t begin = static_cast<int64_t>(chunk - t.first) * TensorNorm::kChunk;
        if (t.types & 2) {
            constexpr int kEights = TensorNorm::kChunk / kThreads / 8;
            Raw8<bf16_t> r[kEights];
#pragma unroll
            for (int k = 0; k < kEights; ++k) {
                const int64_t at = begin + (k * kThreads + threadIdx.x) * 8;
                load_some(r[k], static_cast<const bf16_t *>(t.grad) + at, within(at, t.n));
            }
#pragma unroll
            for (int k = 0; k < kEights; ++k) {
                float g[8];
                raw_floats(r[k], g);
                sum = squares(g, sum);
            }
        } else {
            constexpr int kFours = TensorNorm::kChunk / kThreads / 4;
            float g[kFours][4];
#pragma unroll
            for (int k = 0; k < kFours; ++k) {
                const int64_t at = begin + (k * kThreads + threadIdx.x) * 4;
                load4(g[k], static_cast<const float *>(t.grad) + at, within4(at, t.n));
            }
#pragma unroll
            for (int k = 0; k < kFours; ++k) sum = squares(g[k], sum);
        }
    }
    sum = block_sum(sum, scratch);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}
__global__ void __launch_bounds__(1024) grad_norm_join_kernel(const double *__restrict__ parts, int64_t n, float *__restrict__ norm) {
    __shared__ double scratch[1024 / kWave];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) sum += parts[i];
    sum = block_sum(sum, scratch);
    if (threadIdx.x == 0) *norm = static_cast<float>(sqrt(sum));
}

// ------------------------------------------------------------------------------------------- values of an 8-bit state
// HBM: 2 bytes read and 4 written per element (622 million: 592-613 us, 6.1-6.3 TB/s).
__global__ void __launch_bounds__(kThreads) state_values_kernel(const uint8_t *m, const uint8_t *m_scale, const uint8_t *v, const uint8_t *v_scale, int64_t n,
                                                                void *m_out, void *root_out, int dtype) {
    const int64_t at = (flat_block() * kThreads + threadIdx.x) * 8;
    const int some = within(at, n);
    if (!some) return;
    float x[8];
    if (m_out) {
        decode8<FirstCode>(load_codes(m + at, some), m_scale[at / kStateBlock], x);
        store_typed(m_out, dtype, at, x, some);
    }
    if (root_out) {
        decode8<RootCode>(load_codes(v + at, some), v_scale[at / kStateBlock], x);
        store_typed(root_out, dtype, at, x, some);
    }
}

// ------------------------------------------------------------------------------------------------------------ host

static void describe(Tensor32 &e, const spo_adamw_tensor &t) {
    e.m = static_cast<float *>(t.m);
    e.v = static_cast<float *>(t.v);
}
static void describe(Tensor8 &e, const spo_adamw_tensor &t) {
    e.m = static_cast<uint8_t *>(t.m);
    e.v = static_cast<uint8_t *>(t.v);
    e.m_scale = t.m_scale;
    e.v_scale = t.v_scale;
}
static void describe(TensorNorm &, const spo_adamw_tensor &) {}
template <typename T>
static void describe_weights(T &e, const spo_adamw_tensor &t) {
    e.param = t.param;
    e.copy = static_cast<bf16_t *>(t.copy);
    e.decay = t.weight_decay;
}
static void describe_weights(TensorNorm &, const spo_adamw_tensor &) {}

// Calls launch(table) for the tensors that have elements, as many at a time as a launch's arguments hold.
template <typename T, typename F>
static int in_tables(const spo_adamw_desc *d, F launch) {
    Table<T> table;
    table.count = table.chunks = 0;
    for (int64_t i = 0; i < d->count; ++i) {
        const spo_adamw_tensor &t = d->tensors[i];
        if (t.n == 0) continue;
        T &e = table.t[table.count++];
        describe(e, t);
        describe_weights(e, t);
        e.grad = t.grad;
        e.n = t.n;
        e.first = table.chunks;
        e.types = (t.param_dtype == SPO_BF16 ? 1 : 0) | (t.grad_dtype == SPO_BF16 ? 2 : 0);
        table.chunks += static_cast<int32_t>(ceil_div(t.n, T::kChunk));
        if (table.count == Table<T>::kMost) {
            if (int rc = launch(table)) return rc;
            table.count = table.chunks = 0;
        }
    }
    return table.count ? launch(table) : SPO_OK;
}

// Steps over more than the Infinity Cache holds take the non-temporal hint: in 32 bits for the moments (151936 x 1024 in bf16:
// 597 -> 551 us), in 8 bits for what is no code (151936 x 4096 in bf16: 1189 -> 1115 us).
static bool past_cache(const spo_adamw_desc *d, int64_t elements) { return elements > kStreamBytes / (d->state_bits == 32 ? 8 : 6); }

static int64_t elements_of(const spo_adamw_desc *d) {
    int64_t n = 0;
    for (int64_t i = 0; i < d->count; ++i) n += d->tensors[i].n;
    return n;
}

static int64_t norm_launches(const spo_adamw_desc *d) { return std::max<int64_t>(1, ceil_div(d->count, Table<TensorNorm>::kMost)); }

}  // namespace spo

using namespace spo;

static_assert(sizeof(Table<Tensor32>) + sizeof(AdamwScalars) <= 4096 && sizeof(Table<Tensor8>) + sizeof(AdamwScalars) <= 4096, "arguments of a launch");

static bool type_ok(int t) { return t == SPO_FP32 || t == SPO_BF16; }
static bool aligned_to(const void *p, int dtype) { return reinterpret_cast<uintptr_t>(p) % (dtype == SPO_FP32 ? 4 : 2) == 0; }

// `state`: moments and weights are looked at too
static int validate(const spo_adamw_desc *d, bool state) {
    if (!d) return SPO_ENULL;
    if (d->struct_size != sizeof(spo_adamw_desc)) return SPO_EINVAL;
    if (d->state_bits != 32 && d->state_bits != 8) return SPO_EINVAL;
    if (d->count < 0) return SPO_EINVAL;
    if (d->count > kMostTensors) return SPO_ERANGE;
    if (d->count && !d->tensors) return SPO_ENULL;
    for (int64_t i = 0; i < d->count; ++i) {
        const spo_adamw_tensor &t = d->tensors[i];
        if (t.n < 0 || !type_ok(t.grad_dtype)) return SPO_EINVAL;
        if (t.n > kMostElements) return SPO_ERANGE;
        if (t.n == 0) continue;
        if (!t.grad) return SPO_ENULL;
        if (!aligned_to(t.grad, t.grad_dtype)) return SPO_EINVAL;
        if (!state) continue;
        if (!type_ok(t.param_dtype) || !(t.weight_decay >= 0.0)) return SPO_EINVAL;
        if (!t.param || !t.m || !t.v || (d->state_bits == 8 && (!t.m_scale || !t.v_scale))) return SPO_ENULL;
        if (!aligned_to(t.param, t.param_dtype) || !aligned_to(t.copy, SPO_BF16)) return SPO_EINVAL;
        if (d->state_bits == 32 && (!aligned_to(t.m, SPO_FP32) || !aligned_to(t.v, SPO_FP32))) return SPO_EINVAL;
        if (t.copy && t.param_dtype != SPO_FP32) return SPO_EINVAL;
    }
    return SPO_OK;
}

extern "C" size_t spo_grad_norm_workspace_bytes(const spo_adamw_desc *d) {
    return d && d->struct_size == sizeof(spo_adamw_desc) && d->count >= 0 && d->count <= kMostTensors ? sizeof(double) * kNormParts * norm_launches(d) : 0;
}

extern "C" int spo_grad_norm(const spo_adamw_desc *d, float *norm, void *ws, size_t ws_bytes, spo_stream_t stream) {
    if (int rc = validate(d, false)) return rc;
    if (!norm) return SPO_ENULL;
    if (!ws) return SPO_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(ws) % 256 || !aligned_to(norm, SPO_FP32)) return SPO_EINVAL;
    if (ws_bytes < spo_grad_norm_workspace_bytes(d)) return SPO_EWORKSPACE;
    const hipStream_t s = as_stream(stream);
    double *parts = static_cast<double *>(ws);
    int64_t used = 0;
    const int rc = in_tables<TensorNorm>(d, [&](const Table<TensorNorm> &table) {
        const int groups = std::min(kNormParts, table.chunks);
        grad_norm_kernel<<<groups, kThreads, 0, s>>>(table, parts + used);
        used += groups;
        return SPO_OK;
    });
    if (rc) return rc;
    grad_norm_join_kernel<<<1, 1024, 0, s>>>(parts, used, norm);
    return launch_status();
}

extern "C" size_t spo_adamw_update_workspace_bytes(void) { return 256; }

extern "C" int spo_adamw_update(const spo_adamw_desc *d, double lr, const float *lr_device, double beta1, double beta2, double eps, int64_t step,
                                int64_t *step_device, const float *grad_norm, double max_norm, int rounding, void *ws, size_t ws_bytes,
                                spo_stream_t stream) {
    if (int rc = validate(d, true)) return rc;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0)) return SPO_EINVAL;
    if (!lr_device && !(lr >= 0.0)) return SPO_EINVAL;
    if (!step_device && step < 1) return SPO_EINVAL;
    if (grad_norm && !(max_norm >= 0.0)) return SPO_EINVAL;
    if (rounding != SPO_ROUND_NEAREST && rounding != SPO_ROUND_THRESHOLD) return SPO_EINVAL;
    if (reinterpret_cast<uintptr_t>(lr_device) % 4 || reinterpret_cast<uintptr_t>(step_device) % 8 || reinterpret_cast<uintptr_t>(grad_norm) % 4) return SPO_EINVAL;
    const bool on_device = lr_device || step_device;
    if (on_device) {
        if (!ws || ws_bytes < spo_adamw_update_workspace_bytes()) return SPO_EWORKSPACE;
        if (reinterpret_cast<uintptr_t>(ws) % 256) return SPO_EINVAL;
    }
    const int64_t elements = elements_of(d);
    if (elements == 0 && !step_device) return SPO_OK;
    const hipStream_t s = as_stream(stream);
    AdamwScalars a{};
    a.b1 = static_cast<float>(beta1);
    a.c1 = static_cast<float>(1.0 - beta1);
    a.b2 = static_cast<float>(beta2);
    a.c2 = static_cast<float>(1.0 - beta2);
    // an eps above zero stays there, so that moments of zero are no 0 / 0: in 8 bits where the hardware's reciprocal takes it
    a.eps = static_cast<float>(eps);
    if (eps > 0.0) a.eps = std::max(a.eps, d->state_bits == 8 ? std::numeric_limits<float>::min() : std::numeric_limits<float>::denorm_min());
    a.rounding = rounding;
    a.norm = grad_norm;
    a.max_norm = static_cast<float>(max_norm);
    if (on_device) {
        AdamwStep *out = static_cast<AdamwStep *>(ws);
        adamw_prepare_kernel<<<1, 1, 0, s>>>(lr, lr_device, beta1, beta2, step, step_device, grad_norm, out);
        a.on_device = out;
    } else {
        a.step = step_of(lr, beta1, beta2, step);
    }
    const auto launch = [&](auto *kernel) {
        return [=](const auto &table) {
            kernel<<<fold_grid(table.chunks), kThreads, 0, s>>>(table, a);
            return SPO_OK;
        };
    };
    const bool past = past_cache(d, elements);
    const int rc = d->state_bits == 32 ? (past ? in_tables<Tensor32>(d, launch(adamw_kernel<Tensor32, true>)) : in_tables<Tensor32>(d, launch(adamw_kernel<Tensor32, false>)))
                                       : (past ? in_tables<Tensor8>(d, launch(adamw_kernel<Tensor8, true>)) : in_tables<Tensor8>(d, launch(adamw_kernel<Tensor8, false>)));
    return rc ? rc : launch_status();
}

extern "C" int spo_adamw_state_values(const uint8_t *m, const uint8_t *v, const uint8_t *m_scale, const uint8_t *v_scale, int64_t n, void *m_out,
                                      void *root_out, int dtype, spo_stream_t stream) {
    if (n < 0 || !type_ok(dtype) || !aligned_to(m_out, dtype) || !aligned_to(root_out, dtype)) return SPO_EINVAL;
    if (n > kMostElements) return SPO_ERANGE;
    if (n == 0 || (!m_out && !root_out)) return SPO_OK;
    if ((m_out && (!m || !m_scale)) || (root_out && (!v || !v_scale))) return SPO_ENULL;
    state_values_kernel<<<fold_grid(ceil_div(n, kThreads * 8)), kThreads, 0, as_stream(stream)>>>(m, m_scale, v, v_scale, n, m_out, root_out, dtype);
    return launch_status();
}
