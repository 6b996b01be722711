// Pruned weights in 4 bits and their product with one or a few columns.
//
//   quant_pack_kernel    W o I_a -> codes (m rows of 16 bytes per 32 columns) and scale bytes.  The mask (Eq. 3) is applied here,
//                        once: a pruned weight is code 0 and does not count for its block's scale.
//   quant_unpack_kernel  codes and scales -> values.
//   quant_matvec_kernel  Y = Wq X on the matrix cores: a byte of codes becomes two 16-bit operands in one instruction that
//                        also applies the scale, exactly; products are exact in fp32 and summed there.
#include <type_traits>

#include "lrbi_internal.hpp"
#include "lrbi_store.hpp"

namespace lrbi {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t q_u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 q_f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 q_bf16x8 __attribute__((ext_vector_type(8)));

// One lane, one block: 32 weights of a row, 16 bytes of codes, one scale byte.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quant_pack_kernel(Geom g, const T *__restrict__ W, int64_t ldw, const uint32_t *__restrict__ Ip,
                                                         const uint32_t *__restrict__ Iz, unsigned char *__restrict__ codes, int64_t ldc,
                                                         unsigned char *__restrict__ scales, int64_t lds, int64_t blocks)
{
    const int64_t at = wide_block() * 256 + threadIdx.x;
    const int64_t row = at / blocks, b = at - row * blocks;
    if (row >= g.m) return;
    const int64_t j0 = b * STORE_BLOCK;
    const int left = g.n - j0 < STORE_BLOCK ? (int)(g.n - j0) : STORE_BLOCK;
    const T *src = W + row * ldw + j0;
    float v[STORE_BLOCK];
    if (VEC && left == STORE_BLOCK) {
        constexpr int PER = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < STORE_BLOCK / PER; ++i) {
            const uint4 p = reinterpret_cast<const uint4 *>(src)[i];
            T e[PER];
            __builtin_memcpy(e, &p, 16);
#pragma unroll
            for (int k = 0; k < PER; ++k) v[i * PER + k] = store_widen(e[k]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < STORE_BLOCK; ++i) v[i] = i < left ? store_widen(src[i]) : 0.f;
    }
    uint32_t kept = left == STORE_BLOCK ? 0xFFFFFFFFu : (1u << left) - 1u;
    if (Ip) {
        const int ti = (int)(row / g.r);
        kept = decode_word<true>(g, Ip, Iz, ti, (int)(row - (int64_t)ti * g.r), (int)b);
    }
    float most = 0.f;
    bool finite = true;
#pragma unroll
    for (int i = 0; i < STORE_BLOCK; ++i) {
        if (!((kept >> i) & 1u)) v[i] = 0.f;
        finite = finite && __builtin_fabsf(v[i]) < __builtin_inff();
        most = fmaxf(most, __builtin_fabsf(v[i]));
    }
    const int e = store_exponent<T, 4>(most);
    const float inv = power_of_two(-e);
    uint32_t words[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t w = 0u;
#pragma unroll
        for (int k = 0; k < 8; ++k) w |= code4(v[8 * q + k] * inv) << (4 * k);
        words[q] = finite ? w : 0u;
    }
    *reinterpret_cast<uint4 *>(codes + row * ldc + b * 16) = make_uint4(words[0], words[1], words[2], words[3]);
    scales[row * lds + b] = finite ? (unsigned char)(e + STORE_BIAS) : 255;
}

// two codes of a 32-bit word, byte B, at their scale
template <int B> __device__ __forceinline__ uint32_t widen4(__half, uint32_t w, float s)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, B));
}
template <int B> __device__ __forceinline__ uint32_t widen4(__hip_bfloat16, uint32_t w, float s)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, B));
}

// One lane, eight columns.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quant_unpack_kernel(const unsigned char *__restrict__ codes, int64_t ldc,
                                                           const unsigned char *__restrict__ scales, int64_t lds, int64_t m, int64_t n,
                                                           T *__restrict__ W, int64_t ldw, int64_t pieces)
{
    const int64_t at = wide_block() * 256 + threadIdx.x;
    const int64_t row = at / pieces, p = at - row * pieces;
    if (row >= m) return;
    const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + row * ldc + p * 4);
    const float s = scale_operand(scales[row * lds + (p >> 2)]);
    T o[8];
    if constexpr (sizeof(T) == 4) {
        f32x2 f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3)};
        __builtin_memcpy(o, f, 32);
    } else {
        uint32_t f[4] = {widen4<0>(T{}, w, s), widen4<1>(T{}, w, s), widen4<2>(T{}, w, s), widen4<3>(T{}, w, s)};
        __builtin_memcpy(o, f, 16);
    }
    T *dst = W + row * ldw + p * 8;
    if (VEC && p * 8 + 8 <= n) {
        constexpr int N16 = sizeof(T) * 8 / 16;
        uint4 q[N16];
        __builtin_memcpy(q, o, sizeof(o));
#pragma unroll
        for (int i = 0; i < N16; ++i) reinterpret_cast<uint4 *>(dst)[i] = q[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (p * 8 + i < n) dst[i] = o[i];
    }
}

// Y = Wq X.  A workgroup owns 16 rows of W; its wavefronts take turns along the columns, 128 at a time: lane (row = lane % 16,
// block = lane / 16) loads the 16 bytes of one block and its scale, and the four products of 16 x 16 x 32 that follow take
// eight codes of every block each (the order of a sum's terms is free as long as both operands have the same one).
// X goes through LDS as [eight rows][column], the eight rows of a column 16 bytes, which is the other operand as it is read.
// fp32 X is split into three bf16 columns, x = x1 + x2 + x3 exactly, whose products are added in the end.
static constexpr int QM_WAVES = 8;
static constexpr int QM_CHUNK = 2048; // columns of W whose X is in LDS at a time

template <typename T> struct QmOperand {
    typedef T type;
    static constexpr int parts = 1;
};
template <> struct QmOperand<float> {
    typedef __hip_bfloat16 type;
    static constexpr int parts = 3;
};
__device__ __forceinline__ f32x4 mfma_16x16x32(__half, q_u32x4 a, q_u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(q_f16x8, a), __builtin_bit_cast(q_f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_16x16x32(__hip_bfloat16, q_u32x4 a, q_u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(q_bf16x8, a), __builtin_bit_cast(q_bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ void qm_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void qm_store(__half *p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void qm_store(__hip_bfloat16 *p, float v) { *p = __float2bfloat16(v); }
// the bits of the `part`-th operand of x
__device__ __forceinline__ uint16_t qm_part(__half x, int) { return __builtin_bit_cast(uint16_t, x); }
__device__ __forceinline__ uint16_t qm_part(__hip_bfloat16 x, int) { return __builtin_bit_cast(uint16_t, x); }
__device__ __forceinline__ uint16_t qm_part(float x, int part)
{
    // cut off, not rounded: 8 of the 24 bits each; an infinity or a NaN is its first part alone
    const bool finite = __builtin_fabsf(x) < __builtin_inff();
    uint32_t u = __builtin_bit_cast(uint32_t, x);
    if (!finite) return part ? (uint16_t)0 : (uint16_t)((u >> 16) | ((u & 0x7FFFFFu) ? 0x40u : 0u));
    for (int i = 0; i < part; ++i) {
        x -= __builtin_bit_cast(float, u & 0xFFFF0000u);
        u = __builtin_bit_cast(uint32_t, x);
    }
    return (uint16_t)(u >> 16);
}

// NT: tiles of 16 operand columns.  cols: columns of X that this launch's workgroups take at a time.
template <typename T, int NT>
__global__ __launch_bounds__(64 * QM_WAVES) void quant_matvec_kernel(const unsigned char *__restrict__ codes, int64_t ldc,
                                                                     const unsigned char *__restrict__ scales, int64_t lds, int64_t m,
                                                                     int64_t n, const T *__restrict__ X, int64_t ldx, int64_t N, int cols,
                                                                     T *__restrict__ Y, int64_t ldy, int64_t row_blocks)
{
    typedef typename QmOperand<T>::type Op;
    constexpr int PARTS = QmOperand<T>::parts;
    extern __shared__ uint4 lrbi_dyn_smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t blk = wide_block();
    const int64_t cb = blk / row_blocks, rb = blk - cb * row_blocks;
    const int64_t q0 = cb * cols, i0 = rb * 16;
    if (q0 >= N) return;
    const int nc = N - q0 < cols ? (int)(N - q0) : cols; // columns of X here
    const int ops = nc * PARTS;                          // operand columns
    uint16_t *Xs = (uint16_t *)lrbi_dyn_smem;            // [QM_CHUNK / 8][ops][8]
    const int r = lane & 15, blkq = lane >> 4;
    const int64_t row = i0 + r < m ? i0 + r : m - 1;
    const int64_t blocks = (n + STORE_BLOCK - 1) / STORE_BLOCK;
    const unsigned char *crow = codes + row * ldc, *srow = scales + row * lds;
    int opc[NT]; // this lane's operand column of each tile (past the last one: any)
#pragma unroll
    for (int t = 0; t < NT; ++t) opc[t] = 16 * t + r < ops ? 16 * t + r : ops - 1;
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int64_t k0 = 0; k0 < n; k0 += QM_CHUNK) {
        const int64_t k1 = (k0 + QM_CHUNK < blocks * STORE_BLOCK ? k0 + QM_CHUNK : blocks * STORE_BLOCK);
        const int kk = (int)(k1 - k0); // a multiple of 32
        if (k0) __syncthreads();
        for (int e = tid; e < kk * nc; e += 64 * QM_WAVES) {
            const int j = e / nc, c = e - j * nc;
            const T x = k0 + j < n ? X[(k0 + j) * ldx + q0 + c] : T{};
#pragma unroll
            for (int p = 0; p < PARTS; ++p) Xs[((j >> 3) * ops + c * PARTS + p) * 8 + (j & 7)] = qm_part(x, p);
        }
        __syncthreads();
        for (int64_t b0 = k0 / STORE_BLOCK + 4 * wave; b0 < k1 / STORE_BLOCK; b0 += 4 * QM_WAVES) {
            const int64_t b = b0 + blkq;
            const bool in = b < k1 / STORE_BLOCK;
            const int64_t bc = in ? b : b0;
            uint4 w = *reinterpret_cast<const uint4 *>(crow + bc * 16);
            const float s = scale_operand(srow[bc]);
            if (!in) w = make_uint4(0u, 0u, 0u, 0u);
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
            const uint16_t *xb = Xs + (int64_t)(bc - k0 / STORE_BLOCK) * 4 * ops * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const q_u32x4 a = {widen4<0>(Op{}, ws[i], s), widen4<1>(Op{}, ws[i], s), widen4<2>(Op{}, ws[i], s),
                                   widen4<3>(Op{}, ws[i], s)};
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    q_u32x4 x = *reinterpret_cast<const q_u32x4 *>(xb + (i * ops + opc[t]) * 8);
                    if (!in) x = q_u32x4{0u, 0u, 0u, 0u}; // (an infinity in it times the zero codes would be NaN)
                    acc[t] = mfma_16x16x32(Op{}, a, x, acc[t]);
                }
            }
        }
    }
    // the wavefronts' sums, in their order
    __syncthreads();
    float *red = (float *)lrbi_dyn_smem; // [wave][tile][16 rows][16 columns + 1]
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) red[((wave * NT + t) * 16 + 4 * blkq + v) * 17 + r] = acc[t][v];
    __syncthreads();
    for (int e = tid; e < 16 * nc; e += 64 * QM_WAVES) {
        const int i = e / nc, c = e - i * nc;
        float y = 0.f;
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p) { // the small parts first
            const int op = c * PARTS + p;
            float part = 0.f;
            for (int w = 0; w < QM_WAVES; ++w) part += red[((w * NT + (op >> 4)) * 16 + i) * 17 + (op & 15)];
            y += part;
        }
        if (i0 + i < m) qm_store(Y + (i0 + i) * ldy + q0 + c, y);
    }
}

template <typename T>
static int launch_pack_t(const Geom &g, const T *W, int64_t ldw, const uint32_t *Ip, const uint32_t *Iz, unsigned char *codes, int64_t ldc,
                         unsigned char *scales, int64_t lds, hipStream_t stream)
{
    const int64_t blocks = (g.n + STORE_BLOCK - 1) / STORE_BLOCK, groups = (g.m * blocks + 255) / 256;
    if (groups > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
    const bool vec = ((uintptr_t)W & 15) == 0 && ldw * (int64_t)sizeof(T) % 16 == 0;
    auto kern = vec ? quant_pack_kernel<T, true> : quant_pack_kernel<T, false>;
    LRBI_LAUNCH(kern, wide_grid(groups, 256), dim3(256), 0, stream, g, W, ldw, Ip, Iz, codes, ldc, scales, lds, blocks);
    return LRBI_OK;
}
int launch_quant_pack(const Geom &g, lrbi_dtype dt, const void *dW, int64_t ldw, const uint32_t *dIp, const uint32_t *dIz, void *dCodes,
                      int64_t ldc, void *dScales, int64_t lds, hipStream_t stream)
{
    unsigned char *c = (unsigned char *)dCodes, *s = (unsigned char *)dScales;
    switch (dt) {
    case LRBI_F32: return launch_pack_t(g, (const float *)dW, ldw, dIp, dIz, c, ldc, s, lds, stream);
    case LRBI_F16: return launch_pack_t(g, (const __half *)dW, ldw, dIp, dIz, c, ldc, s, lds, stream);
    default: return launch_pack_t(g, (const __hip_bfloat16 *)dW, ldw, dIp, dIz, c, ldc, s, lds, stream);
    }
}

template <typename T>
static int launch_unpack_t(const unsigned char *codes, int64_t ldc, const unsigned char *scales, int64_t lds, int64_t m, int64_t n, T *W,
                           int64_t ldw, hipStream_t stream)
{
    const int64_t pieces = (n + 7) / 8, groups = (m * pieces + 255) / 256;
    if (groups > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
    const bool vec = ((uintptr_t)W & 15) == 0 && ldw * (int64_t)sizeof(T) % 16 == 0;
    auto kern = vec ? quant_unpack_kernel<T, true> : quant_unpack_kernel<T, false>;
    LRBI_LAUNCH(kern, wide_grid(groups, 256), dim3(256), 0, stream, codes, ldc, scales, lds, m, n, W, ldw, pieces);
    return LRBI_OK;
}
int launch_quant_unpack(lrbi_dtype dt, const void *dCodes, int64_t ldc, const void *dScales, int64_t lds, int64_t m, int64_t n, void *dW,
                        int64_t ldw, hipStream_t stream)
{
    const unsigned char *c = (const unsigned char *)dCodes, *s = (const unsigned char *)dScales;
    switch (dt) {
    case LRBI_F32: return launch_unpack_t(c, ldc, s, lds, m, n, (float *)dW, ldw, stream);
    case LRBI_F16: return launch_unpack_t(c, ldc, s, lds, m, n, (__half *)dW, ldw, stream);
    default: return launch_unpack_t(c, ldc, s, lds, m, n, (__hip_bfloat16 *)dW, ldw, stream);
    }
}

template <typename T>
static int launch_matvec_t(const unsigned char *codes, int64_t ldc, const unsigned char *scales, int64_t lds, int64_t m, int64_t n,
                           const T *X, int64_t ldx, int64_t N, T *Y, int64_t ldy, hipStream_t stream)
{
    constexpr int PARTS = QmOperand<T>::parts;
    const int nt = N * PARTS <= 16 ? 1 : 2;
    const int most = 16 * nt / PARTS, cols = N < most ? (int)N : most;
    const int64_t row_blocks = (m + 15) / 16, groups = row_blocks * ((N + cols - 1) / cols);
    if (groups > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
    const size_t xs = (size_t)QM_CHUNK * cols * PARTS * 2, red = (size_t)QM_WAVES * nt * 16 * 17 * 4, smem = xs > red ? xs : red;
    auto kern = nt == 1 ? quant_matvec_kernel<T, 1> : quant_matvec_kernel<T, 2>;
    LRBI_SET_MAX_LDS(kern, smem);
    LRBI_LAUNCH(kern, wide_grid(groups, 64 * QM_WAVES), dim3(64 * QM_WAVES), smem, stream, codes, ldc, scales, lds, m, n, X, ldx, N, cols, Y,
                ldy, row_blocks);
    return LRBI_OK;
}
int launch_quant_matvec(lrbi_dtype dt, const void *dCodes, int64_t ldc, const void *dScales, int64_t lds, int64_t m, int64_t n,
                        const void *dX, int64_t ldx, int64_t N, void *dY, int64_t ldy, hipStream_t stream)
{
    const unsigned char *c = (const unsigned char *)dCodes, *s = (const unsigned char *)dScales;
    switch (dt) {
    case LRBI_F32: return launch_matvec_t(c, ldc, s, lds, m, n, (const float *)dX, ldx, N, (float *)dY, ldy, stream);
    case LRBI_F16: return launch_matvec_t(c, ldc, s, lds, m, n, (const __half *)dX, ldx, N, (__half *)dY, ldy, stream);
    default: return launch_matvec_t(c, ldc, s, lds, m, n, (const __hip_bfloat16 *)dX, ldx, N, (__hip_bfloat16 *)dY, ldy, stream);
    }
}

} // namespace lrbi
