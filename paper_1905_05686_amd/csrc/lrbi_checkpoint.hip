// Activation checkpoints: a layer input X (n x N row-major, row = input, column = batch) in 8-bit codes with a scale per 32
// batch columns, and back.  The weight gradient takes it as it is stored (lrbi_checkpoint_grad.hip, lrbi_grad256.hip):
// the batch is what that product sums over, so a block's scale belongs to one step of its reduction.
//
// Both directions move each byte once and are bound by that (16384 x 4096 bf16: packing 45 us, taking out 31, 407 MB together at
// 5.4 TB/s, above the 5.0 of a large copy; 800 x 100 f32 3.0 us each).  Four lanes share a block, eight values (one or two
// 16-byte loads, eight bytes of codes) each; the block's largest magnitude goes between them in two exchanges.
#include "lrbi_internal.hpp"
#include "lrbi_store.hpp"

namespace lrbi {

template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void checkpoint_pack_kernel(const T *__restrict__ X, int64_t ldx, int64_t n, int64_t N,
                                                              unsigned char *__restrict__ codes, int64_t ldc,
                                                              unsigned char *__restrict__ scales, int64_t lds, int64_t pieces, bool is_short)
{
    // pieces: a multiple of 4, so that a block's lanes stay together
    const int64_t at = wide_block() * 256 + threadIdx.x, row = store_row(at, pieces, is_short), p = at - row * pieces;
    const int64_t left = row < n ? N - p * 8 : 0;
    StorePiece<T> x = store_load<STREAM>(X + (left > 0 ? row * ldx + p * 8 : 0), left);
    const uint32_t most = store_most<T>(x);
    float largest = store_magnitude<T>(most);
    if (most > StoreBits<T>::most8) { // (rare) what is beyond is cut, infinities and NaN leave the scale alone
        T e[8];
        __builtin_memcpy(e, &x, sizeof(e));
        largest = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = store_widen(e[i]), a = __builtin_fabsf(v);
            if (a < __builtin_inff()) {
                largest = fmaxf(largest, fminf(a, StoreBounds<T>::most8));
                if (a > StoreBounds<T>::most8) e[i] = store_narrow(T{}, __builtin_copysignf(StoreBounds<T>::most8, v));
            }
        }
        __builtin_memcpy(&x, e, sizeof(e));
        largest = fmaxf(largest, __shfl_xor(largest, 1, 64)); // (a block's lanes are all here)
        largest = fmaxf(largest, __shfl_xor(largest, 2, 64));
    }
    if (row >= n) return;
    const int e = store_exponent<T, 8>(largest);
    *reinterpret_cast<uint2 *>(codes + row * ldc + p * 8) = codes8<T>(x, e);
    if ((p & 3) == 0) scales[row * lds + (p >> 2)] = (unsigned char)(e + STORE_BIAS);
}

template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void checkpoint_unpack_kernel(const unsigned char *__restrict__ codes, int64_t ldc,
                                                                const unsigned char *__restrict__ scales, int64_t lds, int64_t n, int64_t N,
                                                                T *__restrict__ X, int64_t ldx, int64_t pieces, bool is_short)
{
    const int64_t at = wide_block() * 256 + threadIdx.x, row = store_row(at, pieces, is_short), p = at - row * pieces;
    if (row >= n) return;
    const uint2 w = *reinterpret_cast<const uint2 *>(codes + row * ldc + p * 8);
    store_values<STREAM>(X + row * ldx + p * 8, values8(T{}, w, scale_operand(scales[row * lds + (p >> 2)])), N - p * 8);
}

template <typename T>
static int launch_pack_t(const T *X, int64_t ldx, int64_t n, int64_t N, unsigned char *codes, int64_t ldc, unsigned char *scales, int64_t lds,
                         hipStream_t stream)
{
    const int64_t pieces = (N + STORE_BLOCK - 1) / STORE_BLOCK * 4, groups = (n * pieces + 255) / 256;
    if (groups > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
    auto kern = n * N * (int64_t)sizeof(T) >= LRBI_STREAM_BYTES ? checkpoint_pack_kernel<T, true> : checkpoint_pack_kernel<T, false>;
    LRBI_LAUNCH(kern, wide_grid(groups, 256), dim3(256), 0, stream, X, ldx, n, N, codes, ldc, scales, lds, pieces,
                groups * 256 < (int64_t)1 << 32);
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
    // (us, 16384 x 8192 bf16: 71 -> 60, read again by the next kernel 163 -> 157; 16384 x 4096, which the cache holds: 31 and 31, 74.5 -> 76.5)
    auto kern = n * N * (int64_t)sizeof(T) >= LRBI_STREAM_BYTES ? checkpoint_unpack_kernel<T, true> : checkpoint_unpack_kernel<T, false>;
    LRBI_LAUNCH(kern, wide_grid(groups, 256), dim3(256), 0, stream, codes, ldc, scales, lds, n, N, X, ldx, pieces,
                groups * 256 < (int64_t)1 << 32);
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
