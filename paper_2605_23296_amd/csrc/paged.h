// The paged cache in 8 bits as its kernels see it: pages, E4M3 codes, E8M0 scales.
#pragma once
#include "common.h"

#define PAGED_MAX_REQUESTS 4096   // the plan keeps four numbers per request in LDS
#define PAGED_MAX_ROWS (1 << 26)  // rows of a step: a plan's threads and the units of an attention are counted in 32 bits
#define PAGED_GRAN 16             // rows of a granule: a 16-byte piece of a V row, never across pages

struct PagedView {
    uint8_t *k, *v, *ks, *vs;
    int32_t* table;
    int32_t n_pages, page_shift, max_pages, n_requests;
};

typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

// 2^(byte - 127) as a float (byte 0, which the library never writes, as 0)
__device__ __forceinline__ float e8m0(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

// two E4M3 codes (the low or the high half of w) times 2^n (given as a float) in bf16: exact
template <bool HI>
__device__ __forceinline__ bf16x2 codes_to_bf16(unsigned w, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI);
#else
    return bf16x2{};
#endif
}
// eight codes: one operand of a bf16 matrix instruction
__device__ __forceinline__ bf16x8 codes8_to_bf16(unsigned w0, unsigned w1, float scale) {
    const bf16x2 a = codes_to_bf16<false>(w0, scale), b = codes_to_bf16<true>(w0, scale);
    const bf16x2 c = codes_to_bf16<false>(w1, scale), d = codes_to_bf16<true>(w1, scale);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// four values to four E4M3 codes, to nearest, ties to even; NaN -> NaN
__device__ __forceinline__ unsigned to_codes4(float a, float b, float c, float d) {
#if defined(__HIP_DEVICE_COMPILE__)
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
#else
    return 0;
#endif
}
// four codes whose scale grows: their values times `down` (a power of two, at most 1), rounded again
__device__ __forceinline__ unsigned recode4(unsigned w, float down) {
#if defined(__HIP_DEVICE_COMPILE__)
    const floatx2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return to_codes4(a[0] * down, a[1] * down, b[0] * down, b[1] * down);
#else
    return 0;
#endif
}
// a mask of the first n bytes of a word (none for n <= 0, all for n >= 4)
__device__ __forceinline__ unsigned low_bytes(int n) { return n >= 4 ? 0xFFFFFFFFu : (1u << 8 * max(n, 0)) - 1u; }

// The largest size that is cached, 240 * 2^120: the next code at that scale, 256, is 2^128, which neither bf16 nor fp32 has.  The bits
// of a float (and, in the upper half, of a bf16).
#define TOP_BITS 0x7F700000u
#define TOP_BYTE 247   // its scale

// E8M0 byte of the least 2^e with amax <= 448 * 2^e = 1.75 * 2^(e + 8), at least 1; amax is finite and not negative
__device__ __forceinline__ int scale_byte(float amax) {
    const unsigned u = __builtin_bit_cast(unsigned, amax);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);   // (subnormals have e <= 1 whatever their bits)
    return max(e, 1);
}

// paged.hip
int paged_view(compact_ctx* ctx, const compact_paged_kv* kv, bool with_pages, PagedView* out);
