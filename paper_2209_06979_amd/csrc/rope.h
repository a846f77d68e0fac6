// Sine and cosine of position * frequency for positions that are far (internal, device).
#pragma once

#include <hip/hip_runtime.h>

// The angle is one product in double precision.  It is taken as quarter turns n + r, |r| <= 1/2: n from the product with 2/pi, r from the
// same product without its rounding (a fused multiply-add, and the part of 2/pi below a double), so that an angle of 10^6 is
// reduced to 10^-16 of a turn.  Beyond 2^52 the first product has no fraction left and r is up to some hundred turns (at 2^63): it is reduced once more, and
// what is left is within 2^-42 of a quarter turn.  Then the Taylor series of sine and cosine at |x| <= pi/4, in REAL: what is left out is below
// 2e-9 with the terms of float and below 1e-18 with those of double.  (In float, x is rounded after the reduction: 3e-8 at most.)
template <class REAL> struct SinCos { REAL s, c; };

template <class REAL> __device__ __forceinline__ SinCos<REAL> sin_cos_of(double position, double frequency)
{
    constexpr double TWO_OVER_PI = 0x1.45f306dc9c883p-1, BELOW = -0x1.6b01ec5417056p-55, HALF_PI = 0x1.921fb54442d18p0;
    const double angle = position * frequency, t = angle * TWO_OVER_PI, n = __builtin_rint(t);
    const double far = __builtin_fma(angle, TWO_OVER_PI, -n) + angle * BELOW, more = __builtin_rint(far), r = far - more;
    const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25)) + (int)more;
    const REAL x = (REAL)(r * HALF_PI), xx = x * x;
    REAL s, c;
    if constexpr (sizeof(REAL) == 4) {
        s = x + x * xx * (-1.f / 6 + xx * (1.f / 120 + xx * (-1.f / 5040 + xx * (1.f / 362880))));
        c = 1.f - 0.5f * xx + xx * xx * (1.f / 24 + xx * (-1.f / 720 + xx * (1.f / 40320 + xx * (-1.f / 3628800))));
    } else {
        s = x + x * xx * (-1.0 / 6 + xx * (1.0 / 120 + xx * (-1.0 / 5040 + xx * (1.0 / 362880 + xx * (-1.0 / 39916800 +
            xx * (1.0 / 6227020800 + xx * (-1.0 / 1307674368000 + xx * (1.0 / 355687428096000))))))));
        c = 1.0 - 0.5 * xx + xx * xx * (1.0 / 24 + xx * (-1.0 / 720 + xx * (1.0 / 40320 + xx * (-1.0 / 3628800 + xx * (1.0 / 479001600 +
            xx * (-1.0 / 87178291200 + xx * (1.0 / 20922789888000)))))));
    }
    SinCos<REAL> out;
    out.s = quarter & 1 ? c : s;
    out.c = quarter & 1 ? s : c;
    if (quarter & 2) out.s = -out.s;
    if ((quarter + 1) & 2) out.c = -out.c;
    return out;
}
