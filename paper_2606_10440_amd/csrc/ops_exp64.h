// Exponentials in 64 bits, where which of two near values is higher, or on
// which side of a border one lies, must not depend on how it was computed.
// 64-bit fused operations run at the rate of 32-bit ones here.
#pragma once

#include "ops_common.h"

namespace simops {

// e^x for x <= 0: 2^n times the exponential's series at what is left, at most
// ln 2 / 2 in magnitude, up to r^12 / 12! (the next term is below 2^-53).
__device__ inline double exp64(double x) {
    x = x < -800. ? -800. : x;  // (0 then; a NaN stays)
    // the nearest whole number in the low bits of 1.5 2^52 and it
    const double magic = 6755399441055744., t = __builtin_fma(x, 1.4426950408889634, magic), n = t - magic;
    // ln 2 as 24 bits, by which n is multiplied exactly, and the rest
    const double r = __builtin_fma(n, 1.904654299957768e-09, __builtin_fma(n, -0.693147182464599609375, x));
    double p = __builtin_fma(r, 1. / 479001600., 1. / 39916800.);
    p = __builtin_fma(p, r, 1. / 3628800.);
    p = __builtin_fma(p, r, 1. / 362880.);
    p = __builtin_fma(p, r, 1. / 40320.);
    p = __builtin_fma(p, r, 1. / 5040.);
    p = __builtin_fma(p, r, 1. / 720.);
    p = __builtin_fma(p, r, 1. / 120.);
    p = __builtin_fma(p, r, 1. / 24.);
    p = __builtin_fma(p, r, 1. / 6.);
    p = __builtin_fma(p, r, .5);
    p = __builtin_fma(p, r, 1.);
    p = __builtin_fma(p, r, 1.);
    return __builtin_ldexp(p, (int)__builtin_bit_cast(uint64_t, t));
}

}  // namespace simops
