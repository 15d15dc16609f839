// Angles of the rotary embedding (rotary.hip, compact.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace revisit {

struct CosSin {
    float c, s;
};

// cos and sin of `quarters` quarter turns. An angle is counted in quarter turns
// in double (position times quarter turns per position), so that far positions
// keep their fraction: of it, nearest whole number away, at most half a quarter
// turn is left, and rounding that to fp32 moves the angle by at most 2^-26
// quarter turns. Its cos and sin are their Taylor sums to degree 10 and 9
// (remainders below 2e-9 at 45 degrees); the whole quarters swap and sign them.
__device__ __forceinline__ CosSin quarter_turns(double quarters) {
    const double whole = rint(quarters);
    const float x = (float)(quarters - whole) * 1.5707963267948966f;
    // whole mod 4, exact for any double
    const int n = (int)(whole - 4.0 * floor(whole * 0.25));
    const float z = x * x;
    const float s0 = x * (1.0f + z * (-1.0f / 6 + z * (1.0f / 120 + z * (-1.0f / 5040 + z * (1.0f / 362880)))));
    const float c0 = 1.0f + z * (-0.5f + z * (1.0f / 24 + z * (-1.0f / 720 + z * (1.0f / 40320 + z * (-1.0f / 3628800)))));
    const float s1 = (n & 1) ? c0 : s0;
    const float c1 = (n & 1) ? s0 : c0;
    return CosSin{((n + 1) & 2) ? -c1 : c1, (n & 2) ? -s1 : s1};
}

}  // namespace revisit
