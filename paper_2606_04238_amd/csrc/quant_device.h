// The quantizer's steps that have to be bit for bit the same everywhere: the one
// rounding of a scale and the quotient of a number and a scale.
#pragma once

#include "qmlp_device.h"

namespace qmlp {

// fp64 -> binary16 bits, a single round-to-nearest-even (never through fp32).
// Built from the bit fields of the double.
__device__ __forceinline__ uint32_t f64_to_f16_bits(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t sign = (uint32_t)(b >> 48) & 0x8000u;
    const int e = (int)((b >> 52) & 0x7FF);
    const uint64_t frac = b & ((1ull << 52) - 1);
    if (e == 0x7FF)
        return frac ? 0x7E00u : (sign | 0x7C00u);
    if (e == 0)
        return sign;                       // fp64 subnormal: far below 2^-25
    const int E = e - 1023;                // value = 1.frac * 2^E
    if (E > 15)
        return sign | 0x7C00u;
    uint64_t keep, rest, halfway;
    int shift;
    uint64_t mant = (1ull << 52) | frac;   // 53-bit significand
    if (E >= -14) {
        shift = 42;                        // keep 11 bits (implicit one + 10)
    } else {
        shift = 42 + (-14 - E);            // subnormal: quantum 2^-24
        if (shift > 63)
            return sign;                   // below half the smallest subnormal
    }
    keep = mant >> shift;
    rest = mant & ((1ull << shift) - 1);
    halfway = 1ull << (shift - 1);
    if (rest > halfway || (rest == halfway && (keep & 1)))
        ++keep;
    if (E >= -14) {
        int he = E + 15;
        if (keep == 2048) {                // rounded up to the next binade
            keep = 1024;
            ++he;
        }
        if (he >= 31)
            return sign | 0x7C00u;
        return sign | ((uint32_t)he << 10) | (uint32_t)(keep - 1024);
    }
    return sign | (uint32_t)keep;          // keep == 1024 is 2^-14, still correct
}

__device__ __forceinline__ double f16_bits_to_f64(uint32_t h) { return (double)h2f(h); }

// rint(w / sd) for a positive binary16 scale sd, exactly as IEEE fp64 division
// followed by rint gives it, in fp32.  w has 24 significant bits and sd 11,
// so w / sd is either a half integer exactly or at least 2^-23 of itself
// away from one, and fp64 rounding never moves it onto one: the answer is the
// integer nearest to the true quotient, ties to even.  c = rint(w * r) with
// r = fl(1 / sd) is that integer or a neighbour (the quotient's magnitude is
// at most 1.5 * 15 + 1, so the product is off by less than 1e-5), and the
// remainder w - c sd is exact in fp32: it is a multiple of the smaller of the
// two operands' last places and no larger than sd.
__device__ __forceinline__ float div_rint(float w, float sd, float r) {
    float c = __builtin_rintf(w * r);
    const float rem = __builtin_fmaf(-c, sd, w);
    const float twice = 2.0f * __builtin_fabsf(rem);
    const float next = c + __builtin_copysignf(1.0f, rem);
    const bool odd = ((int)c & 1) != 0;
    return twice > sd || (twice == sd && odd) ? next : c;
}

}  // namespace qmlp
