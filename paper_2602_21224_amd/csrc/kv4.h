// The 4-bit form of cached rows: 32 values along the head dimension share a power of two
// (one byte, its exponent plus 127; 255 stands for NaN) and are held as sign, two bits of
// exponent and one of mantissa each: 0, 0.5, 1, 1.5, 2, 3, 4, 6. gfx950 converts between
// these and bf16 two values at a time, scale included; every value is exact in bf16.
#pragma once

#include "tv_internal.h"

namespace tv {
namespace {

constexpr int kBlock4 = 32;            // values that share a scale

// The power of two of scale byte e as the conversions take it: its exponent field (0
// stands for 2^-127 there, 255 for NaN).
__device__ __forceinline__ float scale4(unsigned e) { return __uint_as_float(e << 23); }

// Values 2 SEL and 2 SEL + 1 of the eight codes in `x`.
template <int SEL>
__device__ __forceinline__ bf16x2 from4(unsigned x, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, SEL);
}
// The eight values of the codes in `x`.
__device__ __forceinline__ bf16x8 from4x8(unsigned x, float scale) {
    const bf16x2 a = from4<0>(x, scale), b = from4<1>(x, scale), c = from4<2>(x, scale), d = from4<3>(x, scale);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace
}  // namespace tv
