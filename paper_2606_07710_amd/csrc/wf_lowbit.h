// wf_lowbit.h -- device-side pieces of the low-bit formats (gfx950): e4m3
// cache elements and power-of-two scale bytes.  Internal header; not part of
// the C ABI.
#pragma once

#include "wf_device.h"

namespace wf {

constexpr int kKv8Block = 32;            // tokens per scale block

// 2^(s - 127) of a scale byte (0 and 255 never come from the library).
__device__ __forceinline__ float scale_value(unsigned s) {
    return __uint_as_float(s << 23);
}

// Scale exponent of a block whose largest finite magnitude is amax: the
// smallest integer e with amax <= 1.TOP * 2^(E + e), TOP the mantissa bits of
// the format's largest value and E its exponent (e4m3 448 = 1.75 * 2^8), read
// off amax's own exponent and mantissa bits, so it is exact.  Magnitudes
// below the normal range end at the lower bound anyway.
template <unsigned TOP, int E>
__device__ __forceinline__ int scale_exponent(float amax) {
    const unsigned b = __float_as_uint(amax);
    if (b == 0)
        return 0;
    const int e = (int)(b >> 23) - 127 - E + ((b & 0x7fffffu) > TOP ? 1 : 0);
    return min(max(e, -100), 120);
}
__device__ __forceinline__ int e4m3_exponent(float amax) {
    return scale_exponent<0x600000u, 8>(amax);
}

// |x| where x is finite, else 0 (what a block's largest magnitude counts).
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;
}

// The four e4m3 codes of a dword as fp32.
__device__ __forceinline__ void e4m3x4_to_f32(uint32_t w, float (&f)[4]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = lo[0];
    f[1] = lo[1];
    f[2] = hi[0];
    f[3] = hi[1];
}

// Four values (already divided by their scale, at most 448) as e4m3 codes,
// to nearest even; what is not finite becomes 0x7f.
__device__ __forceinline__ uint32_t f32x4_to_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    const float v[4] = {a, b, c, d};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!(fabsf(v[i]) < INFINITY))
            w = (w & ~(0xff << (8 * i))) | (0x7f << (8 * i));
    return (uint32_t)w;
}

}  // namespace wf
