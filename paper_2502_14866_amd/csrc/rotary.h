// Angles of rotary positions, for the kernels that turn rows.
#pragma once

#include "kernels.h"

namespace lserve {

// (scale cos, scale sin) of position times frequency: the angle in 64 bits, its whole turns dropped there, sine and cosine of the rest in 32.
__device__ __forceinline__ float2 turn_of(int position, double radians, float scale) {
    const double turns = (double)position * (radians * 0.15915494309189533577);
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    return make_float2(c * scale, s * scale);
}

}  // namespace lserve
