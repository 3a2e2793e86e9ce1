// Eight elements of a row or a flat array as floats and back, from any address that is aligned to the element; fewer where the
// array ends.
#pragma once

#include "row_stream.hpp"

namespace spo {

template <typename T> struct Raw8;  // eight elements as they lie in memory
template <> struct Raw8<bf16_t> { uint4 u[1]; };
template <> struct Raw8<float> { uint4 u[2]; };

template <bool Stream = false>
__device__ __forceinline__ void load_raw(Raw8<bf16_t> &r, const bf16_t *p) { r.u[0] = load16<Stream>(p); }
template <bool Stream = false>
__device__ __forceinline__ void load_raw(Raw8<float> &r, const float *p) {
    r.u[0] = load16<Stream>(p);
    r.u[1] = load16<Stream>(p + 4);
}
__device__ __forceinline__ void raw_floats(const Raw8<bf16_t> &r, float (&x)[8]) { Vec<bf16_t>::unpack(r.u[0], x); }
__device__ __forceinline__ void raw_floats(const Raw8<float> &r, float (&x)[8]) {
    const uint4 a = r.u[0], b = r.u[1];
    x[0] = __uint_as_float(a.x), x[1] = __uint_as_float(a.y), x[2] = __uint_as_float(a.z), x[3] = __uint_as_float(a.w);
    x[4] = __uint_as_float(b.x), x[5] = __uint_as_float(b.y), x[6] = __uint_as_float(b.z), x[7] = __uint_as_float(b.w);
}

// The first `n` (0 to 8) of eight elements, zeros for the others.
template <bool Stream = false>
__device__ __forceinline__ void load_some(Raw8<bf16_t> &r, const bf16_t *p, int n) {
    if (n >= 8) return load_raw<Stream>(r, p);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = i < n ? p[i] : 0u;
    r.u[0] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
}
template <bool Stream = false>
__device__ __forceinline__ void load_some(Raw8<float> &r, const float *p, int n) {
    if (n >= 8) return load_raw<Stream>(r, p);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = i < n ? __float_as_uint(p[i]) : 0u;
    r.u[0] = make_uint4(w[0], w[1], w[2], w[3]);
    r.u[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

template <bool Stream>
__device__ __forceinline__ void put16(void *p, const uint4 &u) {
    typedef u32x4_t V __attribute__((aligned(1)));
    const u32x4_t v = {u.x, u.y, u.z, u.w};
    if (Stream) __builtin_nontemporal_store(v, reinterpret_cast<V *>(p));
    else *reinterpret_cast<V *>(p) = v;
}
template <bool Stream = false>
__device__ __forceinline__ void store_some(bf16_t *p, const float (&x)[8], int n) {
    const uint4 u = Vec<bf16_t>::pack(x);
    if (n >= 8) return put16<Stream>(p, u);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = static_cast<bf16_t>(w[i / 2] >> 16 * (i & 1));
}
template <bool Stream = false>
__device__ __forceinline__ void store_some(float *p, const float (&x)[8], int n) {
    if (n >= 8) {
        put16<Stream>(p, make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])));
        put16<Stream>(p + 4, make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = x[i];
}

// Of a type that the kernel is told at run time (the same for all its threads): arrays that are small beside the others.
__device__ __forceinline__ void load_typed(float (&x)[8], const void *p, int dtype, int64_t at, int n) {
    if (dtype == SPO_FP32) {
        Raw8<float> r;
        load_some(r, static_cast<const float *>(p) + at, n);
        raw_floats(r, x);
    } else {
        Raw8<bf16_t> r;
        load_some(r, static_cast<const bf16_t *>(p) + at, n);
        raw_floats(r, x);
    }
}
template <bool Stream = false>
__device__ __forceinline__ void store_typed(void *p, int dtype, int64_t at, const float (&x)[8], int n) {
    if (dtype == SPO_FP32) store_some<Stream>(static_cast<float *>(p) + at, x, n);
    else store_some<Stream>(static_cast<bf16_t *>(p) + at, x, n);
}
__device__ __forceinline__ int within(int64_t at, int64_t n) { return at >= n ? 0 : n - at < 8 ? static_cast<int>(n - at) : 8; }

}  // namespace spo
