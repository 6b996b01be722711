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

__device__ __forceinline__ float store_narrow(float, float v) { return v; }
__device__ __forceinline__ __half store_narrow(__half, float v) { return __float2half_rn(v); }
__device__ __forceinline__ __hip_bfloat16 store_narrow(__hip_bfloat16, float v) { return __float2bfloat16(v); }

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

// ---- eight neighbouring values of a row, as they are stored: a lane's share of a block, four lanes a block
template <typename T> struct StorePiece {
    uint4 v[sizeof(T) / 2];
};
// 16 bytes at any element's address: one instruction, as for an aligned one
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) StoreUnaligned {
    uint32_t x, y, z, w;
};
// `left` values of the row from here on, zeros behind them.  STREAM: they are too many for the last-level cache.
template <bool STREAM, typename T> __device__ __forceinline__ StorePiece<T> store_load(const T *src, int64_t left)
{
    StorePiece<T> p;
    if (left >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            if constexpr (STREAM) {
                p.v[i] = stream_load16(src + i * (16 / (int)sizeof(T)));
                continue;
            }
            const StoreUnaligned<T> u = reinterpret_cast<const StoreUnaligned<T> *>(src)[i];
            p.v[i] = make_uint4(u.x, u.y, u.z, u.w);
        }
    } else {
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < left ? src[i] : T{};
        __builtin_memcpy(&p, e, sizeof(p));
    }
    return p;
}
template <bool STREAM, typename T> __device__ __forceinline__ void store_values(T *dst, const StorePiece<T> &p, int64_t left)
{
    if (left >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            if constexpr (STREAM) stream_store16(dst + i * (16 / (int)sizeof(T)), p.v[i]);
            else reinterpret_cast<StoreUnaligned<T> *>(dst)[i] = {p.v[i].x, p.v[i].y, p.v[i].z, p.v[i].w};
        }
    } else {
        T e[8];
        __builtin_memcpy(e, &p, sizeof(e));
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) dst[i] = e[i];
    }
}
// row and place in it of the `at`-th of rows of `per_row`; short: both below 2^32 (a 64-bit division is ten times the work)
__device__ __forceinline__ int64_t store_row(int64_t at, int64_t per_row, bool is_short)
{
    return is_short ? (int64_t)((uint32_t)at / (uint32_t)per_row) : at / per_row;
}
// The largest magnitude of a block as the bits of its number of the type: magnitudes are ordered like their bits, infinities and
// NaN above every number.
typedef unsigned short store_u16x2 __attribute__((ext_vector_type(2)));
template <typename T> __device__ __forceinline__ uint32_t store_most(const StorePiece<T> &p)
{
    uint32_t most;
    if constexpr (sizeof(T) == 2) {
        const uint32_t w[4] = {p.v[0].x & 0x7FFF7FFFu, p.v[0].y & 0x7FFF7FFFu, p.v[0].z & 0x7FFF7FFFu, p.v[0].w & 0x7FFF7FFFu};
        const store_u16x2 a = __builtin_elementwise_max(__builtin_bit_cast(store_u16x2, w[0]), __builtin_bit_cast(store_u16x2, w[1]));
        const store_u16x2 b = __builtin_elementwise_max(__builtin_bit_cast(store_u16x2, w[2]), __builtin_bit_cast(store_u16x2, w[3]));
        const store_u16x2 c = __builtin_elementwise_max(a, b);
        most = c.x > c.y ? c.x : c.y;
    } else {
        uint32_t w[8];
        __builtin_memcpy(w, &p, 32);
        most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = most > (w[i] & 0x7FFFFFFFu) ? most : w[i] & 0x7FFFFFFFu;
    }
    const uint32_t one = (uint32_t)__shfl_xor((int)most, 1, 64);
    most = most > one ? most : one;
    const uint32_t two = (uint32_t)__shfl_xor((int)most, 2, 64);
    return most > two ? most : two;
}
template <typename T> __device__ __forceinline__ float store_magnitude(uint32_t bits); // of a block's largest
template <> __device__ __forceinline__ float store_magnitude<float>(uint32_t b) { return __builtin_bit_cast(float, b); }
template <> __device__ __forceinline__ float store_magnitude<__half>(uint32_t b) { return __half2float(__builtin_bit_cast(__half, (uint16_t)b)); }
template <> __device__ __forceinline__ float store_magnitude<__hip_bfloat16>(uint32_t b) { return __builtin_bit_cast(float, b << 16); }
template <typename T> struct StoreBits { // of infinity, and of the magnitude beyond which an 8-bit value is cut
    static constexpr uint32_t inf = 0x7F800000u, most8 = 0x7F700000u;
};
template <> struct StoreBits<__half> {
    static constexpr uint32_t inf = 0x7C00u, most8 = 0x7B80u;
};
template <> struct StoreBits<__hip_bfloat16> {
    static constexpr uint32_t inf = 0x7F80u, most8 = 0x7F70u;
};

// The codes of eight values at scale 2^e.  The conversion instructions scale and round (to nearest, ties to even) as the formats
// ask (tested for every 16-bit number at every scale, fp32 numbers beside every tie, and back for every code at every scale byte);
// 4 bits: what rounds past 6 is 6; 8 bits: what rounds past 448 and infinities are NaN.
typedef __bf16 store_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 store_f16x2 __attribute__((ext_vector_type(2)));
typedef short store_s16x2 __attribute__((ext_vector_type(2)));
template <int B> __device__ __forceinline__ uint32_t narrow4(__half, uint32_t old, uint32_t w, float s)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(store_f16x2, w), s, B);
}
template <int B> __device__ __forceinline__ uint32_t narrow4(__hip_bfloat16, uint32_t old, uint32_t w, float s)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(store_bf16x2, w), s, B);
}
template <typename T> __device__ __forceinline__ uint32_t codes4(const StorePiece<T> &p, int e)
{
    const float s = power_of_two(e);
    uint32_t c = 0;
    if constexpr (sizeof(T) == 2) {
        c = narrow4<0>(T{}, c, p.v[0].x, s);
        c = narrow4<1>(T{}, c, p.v[0].y, s);
        c = narrow4<2>(T{}, c, p.v[0].z, s);
        c = narrow4<3>(T{}, c, p.v[0].w, s);
    } else {
        float f[8];
        __builtin_memcpy(f, &p, 32);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], s, 3);
    }
    return c;
}
template <bool HI> __device__ __forceinline__ store_s16x2 narrow8(__half, store_s16x2 old, uint32_t w, float s)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(old, __builtin_bit_cast(store_f16x2, w), s, HI);
}
template <bool HI> __device__ __forceinline__ store_s16x2 narrow8(__hip_bfloat16, store_s16x2 old, uint32_t w, float s)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, __builtin_bit_cast(store_bf16x2, w), s, HI);
}
template <typename T> __device__ __forceinline__ uint2 codes8(const StorePiece<T> &p, int e)
{
    const float s = power_of_two(e);
    store_s16x2 lo = {0, 0}, hi = {0, 0};
    if constexpr (sizeof(T) == 2) {
        lo = narrow8<false>(T{}, lo, p.v[0].x, s);
        lo = narrow8<true>(T{}, lo, p.v[0].y, s);
        hi = narrow8<false>(T{}, hi, p.v[0].z, s);
        hi = narrow8<true>(T{}, hi, p.v[0].w, s);
    } else {
        float f[8];
        __builtin_memcpy(f, &p, 32);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, f[0], f[1], s, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, f[2], f[3], s, true);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, f[4], f[5], s, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, f[6], f[7], s, true);
    }
    return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

// eight 8-bit codes at their scale, exactly
typedef float store_f32x2 __attribute__((ext_vector_type(2)));
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
__device__ __forceinline__ StorePiece<__half> values8(__half, uint2 w, float s) { return {{widen8_f16(w, s)}}; }
__device__ __forceinline__ StorePiece<__hip_bfloat16> values8(__hip_bfloat16, uint2 w, float s) { return {{widen8_bf16(w, s)}}; }
__device__ __forceinline__ StorePiece<float> values8(float, uint2 w, float s)
{
    const store_f32x2 f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, s, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, s, true),
                              __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, s, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, s, true)};
    StorePiece<float> p;
    __builtin_memcpy(&p, f, sizeof(p));
    return p;
}
// two 4-bit codes of a 32-bit word, byte B, and all eight of them
template <int B> __device__ __forceinline__ uint32_t widen4(__half, uint32_t w, float s)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, B));
}
template <int B> __device__ __forceinline__ uint32_t widen4(__hip_bfloat16, uint32_t w, float s)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, B));
}
template <typename T> __device__ __forceinline__ StorePiece<T> values4(T, uint32_t w, float s)
{
    return {{make_uint4(widen4<0>(T{}, w, s), widen4<1>(T{}, w, s), widen4<2>(T{}, w, s), widen4<3>(T{}, w, s))}};
}
__device__ __forceinline__ StorePiece<float> values4(float, uint32_t w, float s)
{
    const store_f32x2 f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1),
                              __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3)};
    StorePiece<float> p;
    __builtin_memcpy(&p, f, sizeof(p));
    return p;
}

} // namespace lrbi
