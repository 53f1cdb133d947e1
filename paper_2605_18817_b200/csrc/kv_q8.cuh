// Rows of the key / value cache in 8 bits: a row of D values is D e4m3 codes and one byte s, x_i = code_i 2^(s - 127).
#pragma once
#include "mrp_internal.cuh"

namespace mrp {

constexpr uint32_t kQ8NaN = 255;           // the scale byte of a row with a value that is not finite
constexpr uint32_t kQ8Last = 247;          // the largest one else: the largest fp32 lies below 256 * 2^120

// Where rows of the pools and their scales lie (elements are bytes).
struct PoolQ8 {
    uint8_t *code[2], *scale[2];           // keys, values
};

// The scale byte of a row whose largest magnitude has the bits `top` (|x| as an integer; NaN above infinity above all others):
// 127 + E, E the smallest integer >= -127 with |x| <= 448 2^E = 1.75 * 2^(E + 8); 127 for zeros.
__device__ __forceinline__ uint32_t q8_scale(uint32_t top)
{
    if (top >= 0x7F800000u) return kQ8NaN;
    const int s = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u);
    return top == 0 ? 127u : (uint32_t)max(s, 0);
}
// 2^(127 - s) for s = 0 .. 247 (what a row is multiplied by before its codes are rounded)
__device__ __forceinline__ float q8_inverse(uint32_t s) { return __uint_as_float((254u - s) << 23); }
// 2^(s - 127), NaN for 255
__device__ __forceinline__ float q8_factor(uint32_t s)
{
    return __uint_as_float(s == kQ8NaN ? 0x7FC00000u : s == 0 ? 0x00400000u : s << 23);
}
// four values -> four codes, the first in the lowest byte; to nearest, ties to even
__device__ __forceinline__ uint32_t q8_codes(float a, float b, float c, float d)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | (uint32_t)hi << 16;
}
// two codes -> their values times f
__device__ __forceinline__ float2 q8_values(uint32_t two, float f)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&h));
    return make_float2(x.x * f, x.y * f);
}

}  // namespace mrp
