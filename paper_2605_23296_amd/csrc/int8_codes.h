// Codes of a row: q = 127 x / amax, rounded to the nearest integer, ties to even; scale = amax / 127.
#pragma once
#include <type_traits>

#include "common.h"

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

struct RowCodes {
    float inv;     // 127 / amax, not below it
    float amax;
    float up;      // what x and amax are multiplied with, so that 127 / amax is a number
    float scale;
};

// amax as bits.  Broken rows (infinity or NaN): codes 0, scale NaN; rows of zeros: codes 0, scale 0.
__device__ __forceinline__ RowCodes row_codes(uint32_t amax_bits) {
    RowCodes rc;
    const float amax = __uint_as_float(amax_bits);
    rc.scale = amax / 127.0f;
    rc.up = amax < 1e-30f ? 0x1p100f : 1.0f;
    rc.amax = amax * rc.up;
    rc.inv = 127.0f / rc.amax;
    // bf16 values x = X 2^s, amax = A 2^t with 8-bit X and A are a tie where 254 X = (2 j + 1) A 2^n, so where the prime 127 divides 2 j + 1 (j = 63: x = amax / 2) or
    // A (then 127 / amax is a power of two and the product exact).  The first is 63.5, which 127 / amax rounded down would put below; rounded up, the
    // product is 63.5 or more, hence 64.  Every other quotient is 2^-16 of itself or more away from a tie, the error here is 2^-22.
    if (fmaf(rc.inv, rc.amax, -127.0f) < 0.0f) rc.inv = __uint_as_float(__float_as_uint(rc.inv) + 1);
    if (amax_bits == 0) rc.inv = 0.0f;
    if (amax_bits >= 0x7f800000u) {
        rc.scale = __uint_as_float(0x7fc00000u);
        rc.inv = 0.0f;
        rc.up = 0.0f;
    }
    return rc;
}

// T: the type that the value was stored in
template <typename T>
__device__ __forceinline__ int code_of(float x, const RowCodes& rc) {
    const float xs = x * rc.up, t = xs * rc.inv;
    float c = rintf(t);
    // 24-bit values come closer to a tie than t's error (3e-5): those are decided by the quotient in 64 bits
    if (std::is_same<T, float>::value && fabsf(fabsf(t - c) - 0.5f) < 0x1p-14f) c = (float)rint((double)xs * 127.0 / (double)rc.amax);
    // (broken rows: infinity or NaN times 0 is NaN)
    return rc.up == 0.0f ? 0 : (int)c;
}

template <typename T>
__device__ __forceinline__ uint2 codes8(const float (&v)[8], const RowCodes& rc) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[h] |= (uint32_t)(code_of<T>(v[4 * h + j], rc) & 255) << (8 * j);
    }
    return make_uint2(w[0], w[1]);
}
