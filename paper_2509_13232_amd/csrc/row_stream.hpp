// Streaming rows of logits: vectors of 16 bytes as floats and back, the aligned part of a row segment, and how rows are
// cut into segments that groups of threads work on.
#pragma once

#include "pg_common.hpp"

namespace spo {

constexpr int kRowThreads = 256;
constexpr int64_t kStreamBytes = int64_t(256) << 20;  // the Infinity Cache: larger arrays take the non-temporal hint
constexpr int kFewSegments = 8;                        // see row_grid

// 16 bytes of a row as floats and back
template <typename T> struct Vec;
template <> struct Vec<bf16_t> {
    static constexpr int N = 8;
    __device__ static __forceinline__ void unpack(const uint4 &u, float (&x)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[8]) {
        return make_uint4(pack_bf16x2_rn(x[0], x[1]), pack_bf16x2_rn(x[2], x[3]), pack_bf16x2_rn(x[4], x[5]),
                          pack_bf16x2_rn(x[6], x[7]));
    }
    __device__ static __forceinline__ float get(const bf16_t *p) { return bf16_to_f32(*p); }
    __device__ static __forceinline__ void put(bf16_t *p, float v) { *p = f32_to_bf16(v); }
};
template <> struct Vec<float> {
    static constexpr int N = 4;
    __device__ static __forceinline__ void unpack(const uint4 &u, float (&x)[4]) {
        x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
    }
    __device__ static __forceinline__ uint4 pack(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ static __forceinline__ float get(const float *p) { return *p; }
    __device__ static __forceinline__ void put(float *p, float v) { *p = v; }
};

// 16 bytes from an address that may only be aligned to the element (the hardware takes it), and to a
// 16-byte boundary; Stream: with the non-temporal hint
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <typename T> struct Unaligned16;
template <> struct Unaligned16<bf16_t> { typedef u32x4_t V __attribute__((aligned(2))); };
template <> struct Unaligned16<float> { typedef u32x4_t V __attribute__((aligned(4))); };

template <bool Stream, typename T>
__device__ __forceinline__ uint4 load16(const T *p) {
    const auto *q = reinterpret_cast<const typename Unaligned16<T>::V *>(p);
    const u32x4_t v = Stream ? __builtin_nontemporal_load(q) : *q;
    return make_uint4(v.x, v.y, v.z, v.w);
}
template <bool Stream>
__device__ __forceinline__ void store16(uint4 *p, const uint4 &u) {
    const u32x4_t v = {u.x, u.y, u.z, u.w};
    if (Stream) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t *>(p));
    else *reinterpret_cast<u32x4_t *>(p) = v;
}

// Elements [0, n) of a row segment as: a head of single elements up to the first 16-byte boundary,
// whole vectors, a tail of single elements.
struct Span {
    int head, nvec, tail;  // a segment has fewer than 2^31 elements
    template <typename T>
    __device__ __forceinline__ Span(const T *p, int n) {
        const int off = static_cast<int>((16 - reinterpret_cast<uintptr_t>(p) % 16) % 16 / sizeof(T));
        head = off < n ? off : n;
        nvec = (n - head) / Vec<T>::N;
        tail = n - head - nvec * Vec<T>::N;
    }
};

// Which part of which row a group of threads works on: `unit` counts (row, segment) pairs, the
// segments of a row next to each other.
struct RowGrid {
    int64_t rows, seg_len;  // elements per segment
    int nseg, per_wg;       // segments per row, (row, segment) pairs per workgroup
    __host__ __device__ uint32_t units() const { return static_cast<uint32_t>(rows * nseg); }  // < 2^32: of 4 KB segments, 16 TB
    __host__ dim3 blocks() const { return fold_grid(ceil_div(rows * nseg, per_wg)); }
};

// The unit of a group of TR threads, a value the compiler knows to be the same in a whole wavefront: its place and
// extent are then scalar arithmetic (30000 rows of 4104 in bf16: 66 -> 62 us).
template <int TR>
__device__ __forceinline__ int64_t group_unit() {
    if constexpr (TR == kRowThreads) return flat_block();
    else return flat_block() * (kRowThreads / TR) + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / TR);
}

// How the rows are cut: into segments of `rounds` rounds of `group` vectors per thread, of which a short rest is one
// more.  Where that would be one of few, all are made equal (8000 rows of 16392 in bf16 in segments of 16384 and 8:
// 68 us, in halves 50); where it is one of many, whole rounds are the better cut (8192 rows of 151936, loss and
// gradient in turn: 1200 us, in equal segments 1216).  Rows that give a workgroup little work go
// to single wavefronts, four to a workgroup: up to narrow_eighths eighths of a round (60000 rows of 4104 in bf16:
// a workgroup each 116 us, two wavefronts each 96; of 8192, a whole round, 84 against 97).
static inline RowGrid row_grid(int64_t T, int64_t V, int dtype, int group, int rounds, int narrow_eighths) {
    const int64_t n = dtype == SPO_FP32 ? 4 : 8;  // elements per vector
    RowGrid g;
    g.rows = T;
    const bool narrow = V * 8 <= kRowThreads * group * n * narrow_eighths;
    g.per_wg = narrow ? kRowThreads / kWave : 1;
    g.seg_len = (narrow ? kWave : kRowThreads) * group * n * rounds;
    g.nseg = static_cast<int>(ceil_div(V, g.seg_len));
    // of few segments, equal ones: at most as long as they were, so as many of them, none empty
    constexpr int64_t kLine = 64;  // elements: they start on cache lines when the row does
    if (g.nseg <= kFewSegments) g.seg_len = ceil_div(ceil_div(V, g.nseg), kLine) * kLine;
    return g;
}

}  // namespace spo
