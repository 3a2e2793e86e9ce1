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

// Four elements: of fp32 a wavefront's are then whole lines.
__device__ __forceinline__ int within4(int64_t at, int64_t n) { return at >= n ? 0 : n - at < 4 ? static_cast<int>(n - at) : 4; }
template <bool Stream = false>
__device__ __forceinline__ void load4(float (&x)[4], const float *p, int n) {
    if (n >= 4) return Vec<float>::unpack(load16<Stream>(p), x);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = 0.0f;
    if (n <= 0) return;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < n) x[i] = p[i];
}
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void load4(float (&x)[4], const bf16_t *p, int n) {
    if (n >= 4) {
        typedef u32x2_t V __attribute__((aligned(2)));
        const u32x2_t v = *reinterpret_cast<const V *>(p);
        x[0] = __uint_as_float(v.x << 16), x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16), x[3] = __uint_as_float(v.y & 0xffff0000u);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = 0.0f;
    if (n <= 0) return;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < n) x[i] = bf16_to_f32(p[i]);
}
template <bool Stream = false>
__device__ __forceinline__ void store4(float *p, const float (&x)[4], int n) {
    if (n >= 4) return put16<Stream>(p, Vec<float>::pack(x));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) p[i] = x[i];
}
__device__ __forceinline__ void store4(bf16_t *p, const float (&x)[4], int n) {
    const u32x2_t v = {pack_bf16x2_rn(x[0], x[1]), pack_bf16x2_rn(x[2], x[3])};
    if (n >= 4) {
        typedef u32x2_t V __attribute__((aligned(2)));
        *reinterpret_cast<V *>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) p[i] = static_cast<bf16_t>((i < 2 ? v.x : v.y) >> 16 * (i & 1));
}

// E = 8 elements of bf16 or 4 of any type as they lie in memory, floats from them, and floats into memory.
template <int E, typename T> struct RawE { uint32_t u[E * sizeof(T) / 4]; };
template <int E, bool Stream, typename T>
__device__ __forceinline__ void fetch_whole(RawE<E, T> &r, const T *p) {
    static_assert(E * sizeof(T) == 16 || E * sizeof(T) == 8, "one load");
    if constexpr (E * sizeof(T) == 16) {
        const uint4 v = load16<Stream>(p);
        r.u[0] = v.x, r.u[1] = v.y, r.u[2] = v.z, r.u[3] = v.w;
    } else {
        typedef u32x2_t V __attribute__((aligned(2)));
        const u32x2_t v = Stream ? __builtin_nontemporal_load(reinterpret_cast<const V *>(p)) : *reinterpret_cast<const V *>(p);
        r.u[0] = v.x, r.u[1] = v.y;
    }
}
// The first n of them; the others are anything (floats_some leaves them out).  past: what lies behind the n may be read, too.
template <int E, bool Stream, typename T>
__device__ __forceinline__ void fetch(RawE<E, T> &r, const T *p, int n, bool past) {
    if (n >= E || (n > 0 && past)) return fetch_whole<E, Stream>(r, p);
    if (n <= 0) return;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if constexpr (sizeof(T) == 4) {
            r.u[i] = i < n ? __float_as_uint(p[i]) : 0u;
        } else {
            const uint32_t x = i < n ? static_cast<uint32_t>(p[i]) : 0u;
            r.u[i / 2] = i & 1 ? r.u[i / 2] | x << 16 : x;
        }
    }
}
template <int E, typename T>
__device__ __forceinline__ void floats(const RawE<E, T> &r, float (&x)[E]) {
#pragma unroll
    for (int i = 0; i < E; ++i)
        x[i] = __uint_as_float(sizeof(T) == 4 ? r.u[i] : i & 1 ? r.u[i / 2] & 0xffff0000u : r.u[i / 2] << 16);
}
template <int E, typename T>
__device__ __forceinline__ void floats_some(const RawE<E, T> &r, float (&x)[E], int n) {
    floats(r, x);
    if (n < E)
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = i < n ? x[i] : 0.0f;
}
// The first n (0 to E) of E elements, in as few stores as there are ones in n's binary digits.
template <bool Stream, int E>
__device__ __forceinline__ void store_e(float *p, const float (&x)[E], int n) {
    if (n >= E) {
#pragma unroll
        for (int h = 0; h < E; h += 4) {
            const float y[4] = {x[h], x[h + 1], x[h + 2], x[h + 3]};
            put16<Stream>(p + h, Vec<float>::pack(y));
        }
        return;
    }
    uint32_t u[3] = {__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2])};
    if constexpr (E == 8)
        if (n >= 4) {
            const float y[4] = {x[0], x[1], x[2], x[3]};
            put16<false>(p, Vec<float>::pack(y));
            u[0] = __float_as_uint(x[4]), u[1] = __float_as_uint(x[5]), u[2] = __float_as_uint(x[6]);
            p += 4, n -= 4;
        }
    if (n & 2) {
        typedef u32x2_t V2 __attribute__((aligned(4)));
        *reinterpret_cast<V2 *>(p) = u32x2_t{u[0], u[1]};
        p += 2;
        u[0] = u[2];
    }
    if (n & 1) *p = __uint_as_float(u[0]);
}
template <bool Stream, int E>
__device__ __forceinline__ void store_e(bf16_t *p, const float (&x)[E], int n) {
    uint32_t w[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) w[i] = pack_bf16x2_rn(x[2 * i], x[2 * i + 1]);
    typedef u32x2_t V2 __attribute__((aligned(2)));
    if (n >= E) {
        if constexpr (E == 8) {
            put16<Stream>(p, make_uint4(w[0], w[1], w[2], w[3]));
        } else {
            const u32x2_t v = {w[0], w[1]};
            if (Stream) __builtin_nontemporal_store(v, reinterpret_cast<V2 *>(p));
            else *reinterpret_cast<V2 *>(p) = v;
        }
        return;
    }
    uint32_t a = w[0], b = w[1];
    if constexpr (E == 8)
        if (n >= 4) {
            *reinterpret_cast<V2 *>(p) = u32x2_t{w[0], w[1]};
            a = w[2], b = w[3];
            p += 4, n -= 4;
        }
    if (n & 2) {
        typedef uint32_t V1 __attribute__((aligned(2)));
        *reinterpret_cast<V1 *>(p) = a;
        p += 2;
        a = b;
    }
    if (n & 1) *p = static_cast<bf16_t>(a);
}
// One element, rounded as those of store_e are
__device__ __forceinline__ void store_one(float *p, float x) { *p = x; }
__device__ __forceinline__ void store_one(bf16_t *p, float x) { *p = static_cast<bf16_t>(pack_bf16x2_rn(x, x)); }
template <int E>
__device__ __forceinline__ int within_e(int at, int n) { return at >= n ? 0 : n - at < E ? n - at : E; }
// Weights of a type that the kernel is told at run time; zeros behind the n-th.
__device__ __forceinline__ float load_weight(const void *p, int dtype, int at) {
    return dtype == SPO_FP32 ? static_cast<const float *>(p)[at] : bf16_to_f32(static_cast<const bf16_t *>(p)[at]);
}
template <int E>
__device__ __forceinline__ void load_weights(float (&x)[E], const void *p, int dtype, int at, int n) {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = 0.0f;
    if (n <= 0) return;
    if (dtype == SPO_FP32) {
#pragma unroll
        for (int h = 0; h < E; h += 4) {
            float y[4];
            load4(y, static_cast<const float *>(p) + at + h, n - h);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[h + i] = y[i];
        }
    } else {
        RawE<E, bf16_t> r;
        fetch<E, false>(r, static_cast<const bf16_t *>(p) + at, n, false);
        floats_some(r, x, n);
    }
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
__device__ __forceinline__ void store_typed(void *p, int dtype, int64_t at, const float (&x)[8], int n) {
    if (dtype == SPO_FP32) store_some(static_cast<float *>(p) + at, x, n);
    else store_some(static_cast<bf16_t *>(p) + at, x, n);
}
__device__ __forceinline__ int within(int64_t at, int64_t n) { return at >= n ? 0 : n - at < 8 ? static_cast<int>(n - at) : 8; }

}  // namespace spo
