// The two block formats of values stored in few bits: 32 neighbouring values of a row share a scale 2^(b - 127), b one byte.
//   4 bits  sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6
//   8 bits  sign, 4 exponent bits, 3 mantissa bits: multiples of 2^-9 up to 448; 0x7F and 0xFF are NaN
// The scale of a block is the smallest power of two at which its largest magnitude does not round past the largest code, within
// bounds at which every code's value is a number of the type it came from.  Scaling is exact, a value is rounded once (to
// nearest, ties to the even code): it is off by at most half a step of its code.  The matrix cores' conversion instructions
// take codes and scale as they are stored.
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "lrbi_internal.hpp"

namespace lrbi {

static constexpr int STORE_BLOCK = 32; // values that share a scale
static constexpr int STORE_BIAS = 127;

// smallest and largest scale exponent by source type, and the magnitude beyond which an 8-bit value is cut (240 at the largest
// scale: one more binade of codes would leave the type)
template <typename T> struct StoreBounds {
    static constexpr int lo4 = -125, hi4 = 125, lo8 = -117, hi8 = 120;
    static constexpr float most8 = 0x1.ep127f;
};
template <> struct StoreBounds<__half> {
    static constexpr int lo4 = -23, hi4 = 13, lo8 = -15, hi8 = 8;
    static constexpr float most8 = 0x1.ep15f;
};

__device__ __forceinline__ float store_widen(float v) { return v; }
__device__ __forceinline__ float store_widen(__half v) { return __half2float(v); }
__device__ __forceinline__ float store_widen(__hip_bfloat16 v) { return __bfloat162float(v); }

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }
// a scale byte as the conversion instructions take it: the exponent field of a 32-bit number (0 stands for 2^-127, 255 for NaN)
__device__ __forceinline__ float scale_operand(uint32_t b) { return __builtin_bit_cast(float, b << 23); }

// Exponent of a block's scale from its largest magnitude (finite, not negative).  BITS 4: the codes end at 6 = 1.5 * 2^2 and 7
// is the first to round to 8; BITS 8: they end at 448 = 1.75 * 2^8 and 464 still rounds to it.
template <typename T, int BITS> __device__ __forceinline__ int store_exponent(float most)
{
    using B = StoreBounds<T>;
    const uint32_t u = __builtin_bit_cast(uint32_t, most);
    const int e = (int)(u >> 23) - 127; // zero and what is below the normal numbers end at the lower bound
    const uint32_t frac = u & 0x7FFFFFu;
    const int s = BITS == 4 ? e - 2 + (frac >= 0x600000u ? 1 : 0) : e - 8 + (frac > 0x680000u ? 1 : 0);
    const int lo = BITS == 4 ? B::lo4 : B::lo8, hi = BITS == 4 ? B::hi4 : B::hi8;
    return s < lo ? lo : s > hi ? hi : s;
}

// the 4-bit code of a value in units of its scale: half steps below 2, whole ones below 4, twos up to 6
__device__ __forceinline__ uint32_t code4(float v)
{
    const float a = __builtin_fabsf(v);
    const uint32_t low = (uint32_t)(int)__builtin_rintf(a * 2.f);               // 0 .. 4
    const uint32_t mid = (uint32_t)(int)__builtin_rintf(a) + 2u;                // 4 .. 6
    uint32_t high = (uint32_t)(int)__builtin_rintf(fminf(a, 6.f) * 0.5f) + 4u;  // 6, 7
    const uint32_t c = a < 2.f ? low : a < 4.f ? mid : high;
    return c | ((__builtin_bit_cast(uint32_t, v) >> 28) & 8u);
}

// eight 8-bit codes at their scale, exactly
typedef float store_f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void widen8(uint2 w, float s, float (&o)[8])
{
    const store_f32x2 f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, s, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, s, true),
                              __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, s, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, s, true)};
    __builtin_memcpy(o, f, sizeof(o));
}
__device__ __forceinline__ uint4 widen8_f16(uint2 w, float s)
{
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w.x, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w.x, s, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w.y, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w.y, s, true)));
}
__device__ __forceinline__ uint4 widen8_bf16(uint2 w, float s)
{
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, s, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, s, true)));
}
__device__ __forceinline__ void widen8(uint2 w, float s, __half (&o)[8])
{
    const uint4 v = widen8_f16(w, s);
    __builtin_memcpy(o, &v, sizeof(o));
}
__device__ __forceinline__ void widen8(uint2 w, float s, __hip_bfloat16 (&o)[8])
{
    const uint4 v = widen8_bf16(w, s);
    __builtin_memcpy(o, &v, sizeof(o));
}

} // namespace lrbi
