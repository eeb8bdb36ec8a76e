// rotary.hpp -- cosine and sine of rotary positions, and a rounding that leaves a
// further one as it would be (splice_tree.h, splice_pages.h).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#pragma clang fp contract(off)

namespace splice_dev {

// (cos, sin) of so many turns, times a factor.  To the nearest quarter turn,
// then the series of sine and cosine on [-pi / 4, pi / 4], whose first term
// left out is below 2^-33.
__device__ __forceinline__ double2 turned(double turns, double factor) {
    turns -= rint(turns);
    const double n = rint(4. * turns);
    const double x = (turns - 0.25 * n) * 6.28318530717958647693, y = x * x;
    double sn = 1. / 39916800., cs = -1. / 3628800.;
    sn = fma(-sn, y, 1. / 362880.);
    cs = fma(cs, y, 1. / 40320.);
    sn = fma(sn, y, -1. / 5040.);
    cs = fma(cs, y, -1. / 720.);
    sn = fma(sn, y, 1. / 120.);
    cs = fma(cs, y, 1. / 24.);
    sn = fma(sn, y, -1. / 6.);
    cs = fma(cs, y, -1. / 2.);
    sn = fma(sn * y, x, x);
    cs = fma(cs, y, 1.);
    const int k = (int)n & 3;   // quarters
    const double c = k & 1 ? sn : cs, s = k & 1 ? cs : sn;
    return make_double2((k == 1 || k == 2 ? -c : c) * factor, (k & 2 ? -s : s) * factor);
}

// x in 32 bits so that a further rounding, to an 8-bit code, is that of x
// itself: of the two floats beside an inexact x the one with an odd last bit.
__device__ __forceinline__ float odd_float(double x) {
    const float f = (float)x;
    const double rest = x - (double)f;
    uint32_t b = __float_as_uint(f);
    if ((rest > 0. || rest < 0.) && !(b & 1) && fabsf(f) < INFINITY) b += (rest > 0.) != (x < 0.) ? 1 : -1;
    return __uint_as_float(b);
}

}  // namespace splice_dev
