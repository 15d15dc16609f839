// Angles of the rotary embedding (rotary.hip, compact.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace revisit {

struct CosSin {
    float c, s;
};

// cos and sin of `quarters` quarter turns. An angle is counted in quarter turns in double (position
// times quarter turns per position: off by 2^-52 of the angle at most), so that far positions keep
// their fraction; nearest whole number away, at most half a quarter turn is left of it. Its cos and
// sin are Taylor sums to degree 10 and 9 in double (remainders below 2e-9 at 45 degrees), rounded
// once to fp32 (2^-25); in fp32 throughout they were off by up to 1.1e-7. The whole
// quarters swap and sign them.
__device__ __forceinline__ CosSin quarter_turns(double quarters) {
    const double whole = rint(quarters);
    const double x = (quarters - whole) * 1.5707963267948966;
    // whole mod 4, exact for any double
    const int n = (int)(whole - 4.0 * floor(whole * 0.25));
    const double z = x * x;
    const float s0 = (float)(x * (1.0 + z * (-1.0 / 6 + z * (1.0 / 120 + z * (-1.0 / 5040 + z * (1.0 / 362880))))));
    const float c0 = (float)(1.0 + z * (-0.5 + z * (1.0 / 24 + z * (-1.0 / 720 + z * (1.0 / 40320 + z * (-1.0 / 3628800))))));
    const float s1 = (n & 1) ? c0 : s0;
    const float c1 = (n & 1) ? s0 : c0;
    return CosSin{((n + 1) & 2) ? -c1 : c1, (n & 2) ? -s1 : s1};
}

}  // namespace revisit
