// Sine and cosine of position * frequency at any 64-bit position without loss: the frequency is held in turns, as a 64-bit
// binary fraction w = frac(frequency / 2 pi) * 2^64, so that the product modulo 2^64 is the angle modulo a turn exactly (the
// fraction's own rounding, 2^-64 of a turn, is all that the position multiplies).  An fp32 product would be off by position *
// frequency * 2^-24 radians: 0.06 at position 10^6.
#pragma once

#include <cmath>
#include <cstdint>

namespace clear {

inline uint64_t turns_of(double frequency)
{
    const long double turns = (long double)frequency / 6.283185307179586476925286766559L;
    const long double part = turns - std::floor(turns);
    return part >= 1.0L ? 0u : (uint64_t)std::ldexp(part, 64);
}

#ifdef __CUDACC__
// The quadrant comes off in whole numbers, so what is rounded to fp32 is at most an eighth of a turn (error below 2^-26 rad).
__device__ __forceinline__ void turn_sincos(int64_t position, uint64_t turns, float &s, float &c)
{
    const uint64_t t = (uint64_t)position * turns;
    const uint32_t quadrant = (uint32_t)((t + (1ull << 61)) >> 62);
    const int32_t rest = (int32_t)((uint32_t)(t >> 32) - (quadrant << 30));  // [-2^29, 2^29) of 2^32 a turn
    float sn, cs;
    sincospif((float)rest * 4.656612873077393e-10f, &sn, &cs);              // 2^-31: half turns
    const bool swap = quadrant & 1u;
    const float a = swap ? cs : sn, b = swap ? sn : cs;
    s = quadrant & 2u ? -a : a;
    c = (quadrant + 1u) & 2u ? -b : b;
}
#endif

}  // namespace clear
