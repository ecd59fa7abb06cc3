// Frequencies of the rotation by (time, height, width): host code of the norm and rotation call.
#pragma once

#include <cmath>
#include <cstdint>

// Revolutions per unit of position of every pair, theta^(-2 i / dims[axis]) / (2 pi), as turns + rest.  64 bits alone are off by half of
// 2^-53 of the angle, which shows in a float's last bits from frame 2^28 on; the two parts are within 2^-57 of the first pair's.
// Repeated products of 64-bit fractions: pair i has i roundings of 2^-64, and i times the ratio's own, which is that of
// x = 2 i ln(theta) / dims in the exponent, so x e^-x times 2^-64.  A product instead of a power for every pair (3 us of a call), and 0.2 us
// more than products in 64 bits; powl for the ratio 1 us more.
inline void fc_rope_turns(double theta, const int32_t* dims, double* turns, float* rest) {
    const long double log_theta = log2l((long double)theta);
    for (int axis = 0, p = 0; axis < 3; ++axis) {
        if (dims[axis] == 0) continue;
        const long double ratio = exp2l(log_theta * -2.0L / dims[axis]);
        long double t = 0.159154943091895335768883763372514362L;      // 1 / (2 pi)
        for (int i = 0; i < dims[axis] / 2; ++i, ++p, t *= ratio) {
            turns[p] = (double)t;
            rest[p] = (float)(t - (long double)turns[p]);
        }
    }
}
