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

#include "state8.hpp"
#include "vec8.hpp"

namespace spo {

constexpr int kThreads = 256;
constexpr int kChunk = kThreads * 8 * 4;  // elements of a tensor that a workgroup takes
constexpr int64_t kMostElements = int64_t(1) << 36;
constexpr size_t kTableBytes = 3840;  // of a launch's 4 KiB of arguments

struct Tensor32 {
    void *param;
    const void *grad;
    float *m, *v;
    bf16_t *copy;
    int64_t n;
    double decay;
    int32_t first, types;  // its first chunk of the launch; bit 0: param is bf16, bit 1: grad is bf16
};
struct Tensor8 {
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
    const void *grad;
    int64_t n;
    int32_t first, types;
};
template <typename T>
struct Table {
    static constexpr int kMost = kTableBytes / sizeof(T);
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
    int32_t skip;
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
    s.skip = 0;
    return s;
}

__global__ void adamw_prepare_kernel(double lr, const float *lr_device, double beta1, double beta2, int64_t t, int64_t *t_device, const float *norm,
                                     AdamwStep *out) {
    const bool skip = norm && !isfinite(*norm);
    if (t_device) {
        t = *t_device + 1;
        if (!skip) *t_device = t;
    }
    *out = step_of(lr_device ? static_cast<double>(*lr_device) : lr, beta1, beta2, t);
    out->skip = skip;
}

// Eight elements of one tensor: their moments move on, their weights step.
struct Eight {
    float p[8], g[8];
};
__device__ __forceinline__ void weights(Eight &e, const float (&m)[8], const float (&root)[8], const AdamwScalars &a, const AdamwStep &s, float decay) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float change = m[i] / (root[i] * s.root_scale + a.eps) * s.rate;
        e.p[i] = e.p[i] - (change + (decay != 0.0f ? e.p[i] * decay : 0.0f));  // (an infinite weight without decay stays)
    }
}
__device__ __forceinline__ float first_moment(float m, float g, const AdamwScalars &a) {
#pragma clang fp contract(off)
    return m * a.b1 + g * a.c1;
}
__device__ __forceinline__ float second_moment(float v, float g, const AdamwScalars &a) {
#pragma clang fp contract(off)
    return v * a.b2 + g * g * a.c2;
}

// bf16 by the step's thresholds (state8.hpp); what is not finite, to nearest
__device__ __forceinline__ void store_by_threshold(bf16_t *p, const float (&x)[8], int n, uint32_t step, uint32_t place) {
    const uint32_t turn = turn_of(step, kTurnWeight);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = __float_as_uint(x[i]);
        const uint32_t up = (u + (turn_at(turn, place + i) >> 16)) & 0xffff0000u;
        y[i] = (u & 0x7f800000u) == 0x7f800000u ? x[i] : __uint_as_float(up);
    }
    store_some(p, y, n);
}

__device__ __forceinline__ void load_moments(const Tensor32 &t, int64_t at, int some, float (&m)[8], float (&v)[8]) {
    Raw8<float> r;
    load_some(r, t.m + at, some);
    raw_floats(r, m);
    load_some(r, t.v + at, some);
    raw_floats(r, v);
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
__device__ __forceinline__ void decode8(const Codes &c, uint32_t scale, float (&x)[8]) {
    const uint32_t nan = nan_of(scale);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = C::decode(c.u[i / 4] >> 8 * (i & 3) & 0xff, scale, nan);
}
// The scale of the block of which this thread holds eight elements (the eight neighbouring threads hold it together), and their codes.
template <typename C>
__device__ __forceinline__ Codes encode8(const float (&x)[8], uint32_t turn, uint32_t place, uint32_t &scale) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < kStateBlock / 8; o <<= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o, kWave)));
    scale = C::scale(top);
    Codes c = {{0, 0}};
#pragma unroll
    for (int i = 0; i < 8; ++i) c.u[i / 4] |= C::encode(x[i], scale, turn_at(turn, place + i)) << 8 * (i & 3);
    return c;
}

template <typename T, int kBits>
__global__ void __launch_bounds__(kThreads) adamw_kernel(Table<T> table, AdamwScalars a) {
    const int64_t block = flat_block();
    if (block >= table.chunks) return;
    float factor = 1.0f;
    if (a.norm) {
        const float norm = *a.norm;
        if (!isfinite(norm)) return;  // nothing moves
        if (norm > a.max_norm) factor = a.max_norm / norm;
    }
    const AdamwStep s = a.on_device ? *a.on_device : a.step;
    const int which = table.find(static_cast<int>(block));
    const T t = table.t[which];
    const float decay = static_cast<float>(s.lr * t.decay);
    const int64_t begin = (block - t.first) * kChunk, end = std::min<int64_t>(begin + kChunk, t.n);
    for (int64_t at = begin + threadIdx.x * 8; at - threadIdx.x % kWave * 8 < end; at += kThreads * 8) {  // whole wavefronts
        const int some = within(at, t.n);
        const uint32_t place = static_cast<uint32_t>(at) % kStateBlock;
        Eight e;
        float m[8], v[8], root[8];
        load_typed(e.p, t.param, t.types & 1 ? SPO_BF16 : SPO_FP32, at, some);
        load_typed(e.g, t.grad, t.types & 2 ? SPO_BF16 : SPO_FP32, at, some);
        uint32_t scale = 0;
        if constexpr (kBits == 32) {
            load_moments(t, at, some, m, v);
        } else {
            const int64_t b = at / kStateBlock;
            scale = some ? t.m_scale[b] : 0;
            decode8<FirstCode>(load_codes(t.m + at, some), scale, m);
            scale = some ? t.v_scale[b] : 0;
            decode8<RootCode>(load_codes(t.v + at, some), scale, root);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = root[i] * root[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float g = e.g[i] * factor;
            m[i] = first_moment(m[i], g, a);
            v[i] = second_moment(v[i], g, a);
            root[i] = sqrtf(v[i]);
        }
        weights(e, m, root, a, s, decay);
        if constexpr (kBits == 32) {
            store_some(t.m + at, m, some);
            store_some(t.v + at, v, some);
        } else {
            const int64_t b = at / kStateBlock;
            const Codes mc = encode8<FirstCode>(m, turn_of(s.step, kTurnFirst), place, scale);
            store_codes(t.m + at, mc, some);
            if (some && place == 0) t.m_scale[b] = static_cast<uint8_t>(scale);
            const Codes vc = encode8<RootCode>(root, turn_of(s.step, kTurnRoot), place, scale);
            store_codes(t.v + at, vc, some);
            if (some && place == 0) t.v_scale[b] = static_cast<uint8_t>(scale);
        }
        if (!(t.types & 1)) store_some(static_cast<float *>(t.param) + at, e.p, some);
        else if (a.rounding == SPO_ROUND_NEAREST) store_some(static_cast<bf16_t *>(t.param) + at, e.p, some);
        else store_by_threshold(static_cast<bf16_t *>(t.param) + at, e.p, some, s.step, place);
        if (t.copy) store_some(t.copy + at, e.p, some);
    }
}

// --------------------------------------------------------------------------------------------- norm of the gradients
constexpr int kNormParts = 2048;  // workgroups of a launch

// Squares of fp32 numbers are exact in 64 bits, and so nearly are their sums: the norm is the rounded true one.
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(Table<TensorNorm> table, double *__restrict__ parts) {
    __shared__ double scratch[kThreads / kWave];
    double sum = 0.0;
    for (int chunk = blockIdx.x; chunk < table.chunks; chunk += gridDim.x) {
        const TensorNorm t = table.t[table.find(chunk)];
        const int64_t begin = static_cast<int64_t>(chunk - t.first) * kChunk;
#pragma unroll
        for (int k = 0; k < kChunk / (kThreads * 8); ++k) {
            const int64_t at = begin + (k * kThreads + threadIdx.x) * 8;
            float g[8];
            load_typed(g, t.grad, t.types & 2 ? SPO_BF16 : SPO_FP32, at, within(at, t.n));
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fma(static_cast<double>(g[i]), static_cast<double>(g[i]), sum);
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
        table.chunks += static_cast<int32_t>(ceil_div(t.n, kChunk));  // (at most kMost 2^23 of them)
        if (table.count == Table<T>::kMost) {
            if (int rc = launch(table)) return rc;
            table.count = table.chunks = 0;
        }
    }
    return table.count ? launch(table) : SPO_OK;
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
    if (d->count > int64_t(1) << 24) return SPO_ERANGE;
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
    return d && d->struct_size == sizeof(spo_adamw_desc) && d->count >= 0 ? sizeof(double) * kNormParts * norm_launches(d) : 0;
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
    const hipStream_t s = as_stream(stream);
    AdamwScalars a{};
    a.b1 = static_cast<float>(beta1);
    a.c1 = static_cast<float>(1.0 - beta1);
    a.b2 = static_cast<float>(beta2);
    a.c2 = static_cast<float>(1.0 - beta2);
    a.eps = static_cast<float>(eps);
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
    const int rc = d->state_bits == 32 ? in_tables<Tensor32>(d, launch(adamw_kernel<Tensor32, 32>)) : in_tables<Tensor8>(d, launch(adamw_kernel<Tensor8, 8>));
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
