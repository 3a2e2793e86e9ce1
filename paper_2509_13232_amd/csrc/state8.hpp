// Moments of an optimiser in 8 bits, in blocks of 64 elements that share a power of two.  Host and device; a test runs it on the host.
//
// A scale is the exponent field (15 to 254) that the block's largest magnitude has once no code is smaller than it; 255: the
// block holds something that is not finite, and all of it is NaN.  A code is the upper bits of a magnitude brought by the scale to
// where exponent fields run from 0 to 15, so codes have subnormals and zero, and both ways are a shift and an exact product:
//   signed   (first moment)            sign, 4 bits of exponent, 3 of mantissa;
//   unsigned (second moment's root)    4 bits of exponent, 4 of mantissa.  A root that is not zero does not become zero: beside a
//                                      first moment that is not, it would be divided by.
// What is held never has more digits than a bf16 number.
//
// Rounding: a value between two codes goes to the upper one if its place between them and the step's threshold reach one.  The
// threshold of a place of the block is (step * golden ratio + place * plastic number's power) mod 1: over steps it visits all of
// [0, 1) evenly (the discrepancy of n steps is of order log n / n), so what a moment changes by per step adds up.  Rounded to
// the nearest code a second moment would stand still: with beta2 = 0.999 a step moves its root by 5e-4, half a code is 3e-2.
#pragma once

#include <cmath>
#include <cstdint>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define SPO_BOTH __host__ __device__ __forceinline__
#else
#define SPO_BOTH inline
#endif

namespace spo {

constexpr int kStateBlock = 64;
constexpr uint32_t kNotFinite = 255;
constexpr uint32_t kPerStep = 0x9E3779B9u, kPerPlace = 0xC13FA9A9u;  // fractions of the golden and the plastic ratio, of 2^32
constexpr uint32_t kTurnFirst = 0u, kTurnRoot = 0x80000000u, kTurnWeight = 0x40000000u;  // where each array's thresholds begin

SPO_BOTH uint32_t float_bits(float x) {
    uint32_t u;
    __builtin_memcpy(&u, &x, 4);
    return u;
}
SPO_BOTH float bits_float(uint32_t u) {
    float x;
    __builtin_memcpy(&x, &u, 4);
    return x;
}

// The threshold of a place of the block: the upper bits of `turn` count.
SPO_BOTH uint32_t turn_of(uint32_t step, uint32_t start) { return step * kPerStep + start; }
SPO_BOTH uint32_t turn_at(uint32_t turn, uint32_t place) { return turn + place * kPerPlace; }

template <int Mantissa>
struct Code8 {
    static_assert(Mantissa == 3 || Mantissa == 4, "with a sign or without");
    static constexpr bool kSigned = Mantissa == 3;
    static constexpr int kDrop = 23 - Mantissa;

    // A value's part in its block's largest: as whole numbers magnitudes compare alike, and NaN is the largest.  A root has no sign, but a
    // NaN that takes its place may.
    SPO_BOTH static uint32_t magnitude(float x) { return kSigned ? float_bits(x) & 0x7fffffffu : float_bits(x); }
    // top: the block's largest
    SPO_BOTH static uint32_t scale(uint32_t top) {
        const uint32_t infinite = 0x7f800000u, e = ((top < infinite ? top : infinite) + ((1u << kDrop) - 1)) >> 23;  // (of NaNs with a sign the sum would wrap)
        return e < 15 ? 15 : e;
    }
    SPO_BOTH static uint32_t threshold(uint32_t turn) { return turn >> (32 - kDrop); }
    // A magnitude and its threshold, shifted so that the code they make is the uppermost byte.
    SPO_BOTH static uint32_t word(float x, uint32_t scale, uint32_t threshold) {
        return (float_bits(ldexpf(fabsf(x), 15 - static_cast<int>(scale))) + threshold) << (24 - kDrop);
    }
    // The code in the uppermost byte, anything below it.  (In a block that is not finite codes may be anything, too.)
    SPO_BOTH static uint32_t encode(float x, uint32_t scale, uint32_t threshold) {
        const uint32_t y = word(x, scale, threshold);
        if (kSigned) return float_bits(copysignf(bits_float(y), x));
        const uint32_t least = float_bits(x) < 1u << 24 ? float_bits(x) : 1u << 24;  // a root is zero or 2^-75 and more, which is past that
        return y > least ? y : least;
    }
    // What a code stands for, of scale 15: the code shifted to where the type's exponent and mantissa meet, and its sign.
    SPO_BOTH static float unscaled(uint32_t code) {
        const float size = bits_float((code & (kSigned ? 0x7f : 0xff)) << kDrop);
        return kSigned ? copysignf(size, bits_float(code << 24)) : size;
    }
    SPO_BOTH static float decode(uint32_t code, uint32_t scale) {
        if (scale == kNotFinite) return bits_float(0x7fc00000u);
        return ldexpf(unscaled(code), static_cast<int>(scale) - 15);
    }
};

typedef Code8<3> FirstCode;
typedef Code8<4> RootCode;

}  // namespace spo
