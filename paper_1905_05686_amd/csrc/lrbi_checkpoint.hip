// Activation checkpoints: a layer input X (n x N row-major, row = input, column = batch) in 8-bit codes with a scale per 32
// batch columns, and back.  The weight gradient takes it as it is stored (lrbi_backward.hip, lrbi_grad256.hip, lrbi_f32.hip):
// the batch is what that product sums over, so a block's scale belongs to one step of its reduction.
//
// Both directions move each byte once.  Four lanes share a block, eight values (one or two 16-byte loads, eight bytes of
// codes) each; the block's largest magnitude goes between them in two exchanges.
#include "lrbi_internal.hpp"
#include "lrbi_store.hpp"

namespace lrbi {

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void checkpoint_pack_kernel(const T *__restrict__ X, int64_t ldx, int64_t n, int64_t N,
                                                              unsigned char *__restrict__ codes, int64_t ldc,
                                                              unsigned char *__restrict__ scales, int64_t lds, int64_t pieces)
{
    const int64_t at = wide_block() * 256 + threadIdx.x; // pieces: a multiple of 4, so that a block's lanes stay together
    const int64_t row = at / pieces, p = at - row * pieces;
    const bool inside = row < n;
    const int64_t q0 = p * 8;
    const T *src = X + (inside ? row : 0) * ldx + q0;
    T raw[8];
    if (VEC && inside && q0 + 8 <= N) {
        uint4 v[sizeof(T) / 2];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = reinterpret_cast<const uint4 *>(src)[i];
        __builtin_memcpy(raw, v, sizeof(raw));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[i] = inside && q0 + i < N ? src[i] : T{};
    }
    float v[8], most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = store_widen(raw[i]);
        const float a = __builtin_fabsf(v[i]);
        if (a < __builtin_inff()) most = fmaxf(most, a); // infinities and NaN become NaN codes and leave the scale alone
    }
    most = fmaxf(most, __shfl_xor(most, 1, 64));
    most = fmaxf(most, __shfl_xor(most, 2, 64));
    if (!inside) return;
    most = fminf(most, StoreBounds<T>::most8);
    const int e = store_exponent<T, 8>(most);
    const float inv = power_of_two(-e);
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = fminf(fmaxf(v[i], -most), most) * inv; // at most 464, which the conversion rounds to 448
    uint32_t lo = __builtin_amdgcn_cvt_pk_fp8_f32(u[0], u[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(u[4], u[5], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(u[2], u[3], (int)lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(u[6], u[7], (int)hi, true);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (!(__builtin_fabsf(v[i]) < __builtin_inff())) (i < 4 ? lo : hi) |= 0x7Fu << (8 * (i & 3));
    *reinterpret_cast<uint2 *>(codes + row * ldc + q0) = make_uint2(lo, hi);
    if ((p & 3) == 0) scales[row * lds + (p >> 2)] = (unsigned char)(e + STORE_BIAS);
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void checkpoint_unpack_kernel(const unsigned char *__restrict__ codes, int64_t ldc,
                                                                const unsigned char *__restrict__ scales, int64_t lds, int64_t n, int64_t N,
                                                                T *__restrict__ X, int64_t ldx, int64_t pieces)
{
    const int64_t at = wide_block() * 256 + threadIdx.x;
    const int64_t row = at / pieces, p = at - row * pieces;
    if (row >= n || p * 8 >= N) return;
    const uint2 w = *reinterpret_cast<const uint2 *>(codes + row * ldc + p * 8);
    const float s = scale_operand(scales[row * lds + (p >> 2)]);
    T o[8];
    widen8(w, s, o);
    T *dst = X + row * ldx + p * 8;
    if (VEC && p * 8 + 8 <= N) {
        uint4 v[sizeof(T) / 2];
        __builtin_memcpy(v, o, sizeof(o));
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(dst)[i] = v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (p * 8 + i < N) dst[i] = o[i];
    }
}

template <typename T>
static int launch_pack_t(const T *X, int64_t ldx, int64_t n, int64_t N, unsigned char *codes, int64_t ldc, unsigned char *scales, int64_t lds,
                         hipStream_t stream)
{
    const int64_t pieces = (N + STORE_BLOCK - 1) / STORE_BLOCK * 4, groups = (n * pieces + 255) / 256;
    if (groups > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
    const bool vec = ((uintptr_t)X & 15) == 0 && ldx * (int64_t)sizeof(T) % 16 == 0;
    auto kern = vec ? checkpoint_pack_kernel<T, true> : checkpoint_pack_kernel<T, false>;
    LRBI_LAUNCH(kern, wide_grid(groups, 256), dim3(256), 0, stream, X, ldx, n, N, codes, ldc, scales, lds, pieces);
    return LRBI_OK;
}
int launch_checkpoint_pack(lrbi_dtype dt, const void *dX, int64_t ldx, int64_t n, int64_t N, void *dCodes, int64_t ldc, void *dScales,
                           int64_t lds, hipStream_t stream)
{
    unsigned char *c = (unsigned char *)dCodes, *s = (unsigned char *)dScales;
    switch (dt) {
    case LRBI_F32: return launch_pack_t((const float *)dX, ldx, n, N, c, ldc, s, lds, stream);
    case LRBI_F16: return launch_pack_t((const __half *)dX, ldx, n, N, c, ldc, s, lds, stream);
    default: return launch_pack_t((const __hip_bfloat16 *)dX, ldx, n, N, c, ldc, s, lds, stream);
    }
}

template <typename T>
static int launch_unpack_t(const unsigned char *codes, int64_t ldc, const unsigned char *scales, int64_t lds, int64_t n, int64_t N, T *X,
                           int64_t ldx, hipStream_t stream)
{
    const int64_t pieces = (N + 7) / 8, groups = (n * pieces + 255) / 256;
    if (groups > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
    const bool vec = ((uintptr_t)X & 15) == 0 && ldx * (int64_t)sizeof(T) % 16 == 0;
    auto kern = vec ? checkpoint_unpack_kernel<T, true> : checkpoint_unpack_kernel<T, false>;
    LRBI_LAUNCH(kern, wide_grid(groups, 256), dim3(256), 0, stream, codes, ldc, scales, lds, n, N, X, ldx, pieces);
    return LRBI_OK;
}
int launch_checkpoint_unpack(lrbi_dtype dt, const void *dCodes, int64_t ldc, const void *dScales, int64_t lds, int64_t n, int64_t N,
                             void *dX, int64_t ldx, hipStream_t stream)
{
    const unsigned char *c = (const unsigned char *)dCodes, *s = (const unsigned char *)dScales;
    switch (dt) {
    case LRBI_F32: return launch_unpack_t(c, ldc, s, lds, n, N, (float *)dX, ldx, stream);
    case LRBI_F16: return launch_unpack_t(c, ldc, s, lds, n, N, (__half *)dX, ldx, stream);
    default: return launch_unpack_t(c, ldc, s, lds, n, N, (__hip_bfloat16 *)dX, ldx, stream);
    }
}

} // namespace lrbi
