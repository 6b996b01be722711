// Pruned weights in 4 bits and their product with one or a few columns.
//
//   quant_pack_kernel    W o I_a -> codes (m rows of 16 bytes per 32 columns) and scale bytes.  The mask (Eq. 3) is applied here,
//                        once: a pruned weight is code 0 and does not count for its block's scale.
//   quant_unpack_kernel  codes and scales -> values.
//   quant_matvec_kernel  Y = Wq X on the matrix cores: a byte of codes becomes two 16-bit operands in one instruction that
//                        also applies the scale, exactly; products are exact in fp32 and summed there.
#include <type_traits>

#include "lrbi_internal.hpp"
#include "lrbi_mfma_common.hpp"
#include "lrbi_store.hpp"

namespace lrbi {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t q_u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 q_f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 q_bf16x8 __attribute__((ext_vector_type(8)));

// A wavefront takes 2048 columns of a row: each lane forms one of their 64 mask words while the weights are on their way, then the
// lanes go along them eight columns at a time, four lanes a block.  Bound by the weights read and, where tiles are small or line up
// with nothing, by the mask words' chain of loads (16000 x 9224 bf16 in 512 x 512 tiles 78 us = 4.8 TB/s; 6000 x 3000 f16 in 300 x 300
// tiles 17, without a mask 11).  Loads return in order, so the mask's wait behind the weights'; asking for its first ones before the weights
// cost more registers than it saved (1 us less on the small one, 1 more on the large).
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void quant_pack_kernel(Geom g, const T *__restrict__ W, int64_t ldw, const uint32_t *__restrict__ Ip,
                                                         const uint32_t *__restrict__ Iz, unsigned char *__restrict__ codes, int64_t ldc,
                                                         unsigned char *__restrict__ scales, int64_t lds, int64_t segments)
{
    constexpr int COLS = 2048, PIECES = COLS / 512;
    const int lane = threadIdx.x & 63;
    const int64_t at = wide_block(), seg = at % segments, row = at / segments * 4 + (threadIdx.x >> 6);
    if (row >= g.m) return;
    const int64_t j0 = seg * COLS + lane * 8;
    const T *src = W + row * ldw + j0;
    StorePiece<T> p[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) p[i] = store_load<STREAM>(src + 512 * i, g.n - j0 - 512 * i);
    uint32_t word = 0xFFFFFFFFu;
    if (Ip) {
        const int ti = (int)(row / g.r);
        word = decode_word<true>(g, Ip, Iz, ti, (int)(row - (int64_t)ti * g.r), (int)(seg * (COLS / 32)) + lane);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const uint32_t kept = (uint32_t)__shfl((int)word, 16 * i + (lane >> 2), 64) >> (8 * (lane & 3));
        if constexpr (sizeof(T) == 2) {
            p[i].v[0] = apply_mask8(p[i].v[0], kept & 255u);
        } else {
            uint32_t w[8];
            __builtin_memcpy(w, &p[i], 32);
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = ((kept >> k) & 1u) ? w[k] : 0u;
            __builtin_memcpy(&p[i], w, 32);
        }
        const uint32_t most = store_most<T>(p[i]);
        const bool finite = most < StoreBits<T>::inf;
        const int e = store_exponent<T, 4>(store_magnitude<T>(most));
        const int64_t j = j0 + 512 * i;
        if (j - (lane & 3) * 8 >= g.n) continue; // no block here
        *reinterpret_cast<uint32_t *>(codes + row * ldc + j / 2) = finite ? codes4<T>(p[i], e) : 0u;
        if ((lane & 3) == 0) scales[row * lds + j / STORE_BLOCK] = finite ? (unsigned char)(e + STORE_BIAS) : 255;
    }
}

// A lane takes eight columns.  Bound by the values written (16000 x 9224 bf16 51 us = 7.3 TB/s, 6000 x 3000 f16 8.2).
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void quant_unpack_kernel(const unsigned char *__restrict__ codes, int64_t ldc,
                                                           const unsigned char *__restrict__ scales, int64_t lds, int64_t m, int64_t n,
                                                           T *__restrict__ W, int64_t ldw, int64_t pieces, bool is_short)
{
    const int64_t at = wide_block() * 256 + threadIdx.x, row = store_row(at, pieces, is_short), p = at - row * pieces;
    if (row >= m) return;
    const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + row * ldc + p * 4);
    store_values<STREAM>(W + row * ldw + p * 8, values4(T{}, w, scale_operand(scales[row * lds + (p >> 2)])), n - p * 8);
}

// Y = Wq X.  The codes are read once, straight into registers, and that is what takes the time: 16384 x 16384 bf16, one column,
// 142 MB in 28.4 us = 5.0 TB/s (8192 x 8192 11.2 us; 500 x 800 f32, latency alone, 5.3).  More columns take longer: from 64 KB on X
// comes in chunks, fetched and turned between two barriers by every workgroup (16384 x 16384 f16, 8 columns 39 us, 32 76; one f32 column, three
// parts, 32).  A wavefront owns 16 rows of W and takes 512 of their columns at a time, the next 512 under way while it multiplies:
// lane (row = lane % 16, block = lane / 16) loads the 16 bytes of one block of each 128 columns, and one piece of 16 scale
// bytes for all of them.  The four products of 16 x 16 x 32 for 128 columns take eight codes of every block each (the order of
// a sum's terms is free as long as both operands have the same one).  X goes through LDS as [eight rows][column], the eight
// rows of a column 16 bytes, which is the other operand as it is read.  fp32 X is split into three bf16 columns, x = x1 + x2 +
// x3 exactly, whose products are added in the end.
// Of a workgroup's eight wavefronts WR own different rows (they share X: for many columns, whose X is what a workgroup reads
// most of), the others every 8 / WR-th piece of 512 columns, their sums are added in LDS.
static constexpr int QM_WAVES = 8;
static constexpr int QM_QUAD = 512; // columns of W a wavefront takes at a time: four times four blocks
static constexpr int QM_LDS = 64 * 1024; // for X

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

struct QmQuad { // a lane's share of 512 columns
    uint4 codes[4];
    uint32_t scales[4];
};
struct alignas(4) QmScales {
    uint32_t v[4];
};
// columns from 512 quad on; what lies behind the last block is read from it (X is zero there) at a scale of 1
__device__ __forceinline__ void qm_load(QmQuad &w, const unsigned char *crow, const unsigned char *srow, int64_t quad, int64_t blocks, int blkq)
{
    const int64_t b0 = quad * 16;
    if (b0 + 16 <= blocks) {
#pragma unroll
        for (int g = 0; g < 4; ++g) w.codes[g] = *reinterpret_cast<const uint4 *>(crow + (b0 + 4 * g + blkq) * 16);
        const QmScales s = *reinterpret_cast<const QmScales *>(srow + b0);
#pragma unroll
        for (int g = 0; g < 4; ++g) w.scales[g] = s.v[g] >> (8 * blkq);
    } else {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int64_t b = b0 + 4 * g + blkq, in = b < blocks ? b : blocks - 1;
            w.codes[g] = *reinterpret_cast<const uint4 *>(crow + in * 16);
            w.scales[g] = b < blocks ? srow[b] : (uint32_t)STORE_BIAS;
        }
    }
}

// NT: tiles of 16 operand columns.  cols: columns of X that a workgroup takes at a time; chunk: columns of W whose X is in LDS at a
// time, a multiple of 512 (8 / WR).  VX: columns of X that are loaded together (at any element's address; cols is at least VX); 0: a
// single column, contiguous and 16-byte aligned.
template <typename T, int NT, int WR, int VX>
__global__ __launch_bounds__(64 * QM_WAVES) void quant_matvec_kernel(const unsigned char *__restrict__ codes, int64_t ldc,
                                                                     const unsigned char *__restrict__ scales, int64_t lds, int64_t m,
                                                                     int64_t n, const T *__restrict__ X, int64_t ldx, int64_t N, int cols,
                                                                     int chunk, T *__restrict__ Y, int64_t ldy, int64_t row_blocks, int64_t workgroups)
{
    typedef typename QmOperand<T>::type Op;
    constexpr int PARTS = QmOperand<T>::parts, WK = QM_WAVES / WR;
    extern __shared__ uint4 lrbi_dyn_smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wk = wave % WK, wr = wave / WK;
    const int64_t blk = wide_block();
    const int64_t cb = blk / workgroups;
    int64_t rb = blk - cb * workgroups;
    if (cb * cols >= N) return;
    const int64_t q0 = cb * cols < N - cols ? cb * cols : N - cols; // (the last ones may be the neighbour's too: the same sums)
    const int ops = cols * PARTS;                        // operand columns
    uint4 *Xs = lrbi_dyn_smem;                           // [chunk / 8][ops]
    float *red = (float *)(Xs + chunk / 8 * ops);        // [two in turn][wave][tile][16 rows][16 columns + 1]
    const int r = lane & 15, blkq = lane >> 4;
    const int64_t blocks = (n + STORE_BLOCK - 1) / STORE_BLOCK, quads = (n + QM_QUAD - 1) / QM_QUAD;
    const unsigned char *crow = nullptr, *srow = nullptr;
    int opc[NT]; // this lane's operand column of each tile (past the last one: any)
#pragma unroll
    for (int t = 0; t < NT; ++t) opc[t] = 16 * t + r < ops ? 16 * t + r : ops - 1;

    QmQuad w, next;
    const bool once = chunk >= n; // all of X stays in LDS
    const int64_t rounds = (quads + WK - 1) / WK;
    int64_t turn = 0;
    auto begin = [&](int64_t block) __attribute__((always_inline)) { // asks for the first columns of a block of rows
        const int64_t i = block * (16 * WR) + 16 * wr + r, row = i < m ? i : m - 1;
        crow = codes + row * ldc;
        srow = scales + row * lds;
        // Rows a power of two apart have the same columns in the same memory channels: where all of X is there, each block of rows
        // begins at another of its rounds.
        turn = once ? block % rounds : 0;
        if (turn * WK + wk < quads) qm_load(next, crow, srow, turn * WK + wk, blocks, blkq);
    };
    begin(rb);
    int half = 0;
    for (; rb < row_blocks; rb += workgroups, half ^= 1) {
    const int64_t i0 = rb * (16 * WR);
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    int64_t done = 0; // rounds
    for (int64_t k0 = 0; k0 < n; k0 += chunk) {
        const int kk = (int)(k0 + chunk < quads * QM_QUAD ? chunk : quads * QM_QUAD - k0); // a multiple of 512
        constexpr int V = VX ? VX : 1; // eight rows of V columns a lane
        const int per_row = (cols + V - 1) / V;
        const bool fill = !once || rb == blk - cb * workgroups;
        if (!once) __syncthreads(); // the last chunk has been read
        for (int e = fill ? tid : kk; e < kk / 8 * per_row; e += 64 * QM_WAVES) {
            const int j8 = e / per_row, c4 = (e - j8 * per_row) * V, c = c4 < cols - V ? c4 : cols - V; // (the last V)
            const int64_t j = k0 + 8 * j8;
            struct __attribute__((packed, aligned(sizeof(T)))) Row {
                T v[V];
            } x[8];
            if (VX == 0 && j + 8 <= n) {
                uint4 v[sizeof(T) / 2];
#pragma unroll
                for (int k = 0; k < (int)sizeof(T) / 2; ++k) v[k] = reinterpret_cast<const uint4 *>(X + j)[k];
                __builtin_memcpy(x, v, sizeof(v));
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (j + k < n) x[k] = *reinterpret_cast<const Row *>(X + (j + k) * ldx + q0 + c);
                    else x[k] = Row{};
                }
            }
#pragma unroll
            for (int l = 0; l < V; ++l)
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    uint16_t h[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) h[k] = qm_part(x[k].v[l], p);
                    uint4 v;
                    __builtin_memcpy(&v, h, 16);
                    Xs[j8 * ops + (c + l) * PARTS + p] = v;
                }
        }
        if (fill) __syncthreads();
        for (const int64_t end = once ? rounds : (k0 + kk + WK * QM_QUAD - 1) / (WK * QM_QUAD); done < end; ++done) {
            const int64_t quad = turn * WK + wk;
            if (++turn == rounds) turn = 0;
            w = next;
            if (done + 1 < rounds && turn * WK + wk < quads) qm_load(next, crow, srow, turn * WK + wk, blocks, blkq);
            if (quad >= quads) continue;
            const uint4 *xb = Xs + (quad * 64 - k0 / 8 + 4 * blkq) * ops;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float s = scale_operand(w.scales[g] & 255u);
                const uint32_t ws[4] = {w.codes[g].x, w.codes[g].y, w.codes[g].z, w.codes[g].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const q_u32x4 a = {widen4<0>(Op{}, ws[k], s), widen4<1>(Op{}, ws[k], s), widen4<2>(Op{}, ws[k], s),
                                       widen4<3>(Op{}, ws[k], s)};
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        acc[t] = mfma_16x16x32(Op{}, a, *reinterpret_cast<const q_u32x4 *>(xb + (16 * g + k) * ops + opc[t]), acc[t]);
                }
            }
        }
    }
    if (rb + workgroups < row_blocks) begin(rb + workgroups);
    // the wavefronts' sums, in their order (the other half is written next: what is read here is not overwritten before the
    // barrier after that)
    float *part = red + half * (QM_WAVES * NT * 16 * 17);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) part[((wave * NT + t) * 16 + 4 * blkq + v) * 17 + r] = acc[t][v];
    __syncthreads();
    for (int e = tid; e < 16 * WR * cols; e += 64 * QM_WAVES) {
        const int il = e / cols, c = e - il * cols;
        float y = 0.f;
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p) { // the small parts first
            const int op = c * PARTS + p;
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < WK; ++v) sum += part[((((il >> 4) * WK + v) * NT + (op >> 4)) * 16 + (il & 15)) * 17 + (op & 15)];
            y += sum;
        }
        if (i0 + il < m) qm_store(Y + (i0 + il) * ldy + q0 + c, y);
    }
    }
}

template <typename T>
static int launch_pack_t(const Geom &g, const T *W, int64_t ldw, const uint32_t *Ip, const uint32_t *Iz, unsigned char *codes, int64_t ldc,
                         unsigned char *scales, int64_t lds, hipStream_t stream)
{
    const int64_t segments = (g.n + 2047) / 2048, groups = (g.m + 3) / 4 * segments;
    if (groups > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
    // (with the other direction, 16000 x 9224 bf16: 162 -> 128 us)
    auto kern = g.m * g.n * (int64_t)sizeof(T) >= LRBI_STREAM_BYTES ? quant_pack_kernel<T, true> : quant_pack_kernel<T, false>;
    LRBI_LAUNCH(kern, wide_grid(groups, 256), dim3(256), 0, stream, g, W, ldw, Ip, Iz, codes, ldc, scales, lds, segments);
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
    auto kern = m * n * (int64_t)sizeof(T) >= LRBI_STREAM_BYTES ? quant_unpack_kernel<T, true> : quant_unpack_kernel<T, false>;
    LRBI_LAUNCH(kern, wide_grid(groups, 256), dim3(256), 0, stream, codes, ldc, scales, lds, m, n, W, ldw, pieces,
                groups * 256 < (int64_t)1 << 32);
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
    const int most = 16 * nt / PARTS;
    const int64_t col_blocks = (N + most - 1) / most;
    const int cols = (int)((N + col_blocks - 1) / col_blocks);
    const bool column = N == 1 && ldx == 1 && ((uintptr_t)X & 15) == 0;
    const bool fours = cols >= 4;
    // Wavefronts on different rows share X in LDS and add up fewer sums; there are fewer workgroups.  As many as leave one for
    // every compute unit (us a call, with 1, 2, 4: 8192 x 8192, 7 columns f16 20.8 / 15.9 / 18.5, one column f32 13.3 / 14.6 / 14.5;
    // 16384 x 4096, 8 columns f16 17.8 / 14.3 / 11.6; 16384 x 16384, one column f32 39.9 / 39.1 / 36.1; 2000 x 4000, 7 columns f16 6.5 / 7.5 /
    // 9.2; 6000 x 3000, 7 columns f16 7.8 / 7.1 / 8.2, 2 columns f32 10.4 / 8.5 / 9.6), two for more than 8 operand columns, whose X fills LDS
    // (with 2, 4: 6000 x 3000, 17 columns f16 12.4 / 15.1; 8192 x 8192, 16 columns 19.4 / 23.4; 16384 x 4096, 17 columns 29.3 / 21.3); one
    // 16-bit column is little to share (300 x 16384 9.1 / 16.2 / 24.5, 16384 x 16384 30.2 / 40.8 / 32.7).
    int wr = m >= 64 * 256 ? 4 : m >= 32 * 256 || cols * PARTS > 8 ? 2 : 1;
    if (column && sizeof(T) == 2) wr = 1;
    const int64_t row_blocks = (m + 16 * wr - 1) / (16 * wr);
    // X of a chunk in LDS: all of it where it fits, otherwise whole rounds of the wavefronts
    const int64_t round = (int64_t)QM_QUAD * (QM_WAVES / wr), per_row = (int64_t)cols * PARTS * 2, all = (n + QM_QUAD - 1) / QM_QUAD * QM_QUAD;
    int64_t chunk = QM_LDS / per_row / round * round;
    if (chunk < round) chunk = round;
    if (chunk > all) chunk = all;
    // workgroups that keep X take several blocks of rows, with two sets of sums: two on a compute unit
    const int64_t x_bytes = chunk * per_row, sums = (int64_t)QM_WAVES * nt * 16 * 17 * 4;
    const bool several = chunk == all && row_blocks > 512 && x_bytes + 2 * sums <= 160 * 1024;
    const int64_t workgroups = several ? 512 : row_blocks, groups = workgroups * col_blocks;
    if (groups > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
    const size_t smem = (size_t)(x_bytes + (several ? 2 : 1) * sums); // at most 145 KB
#define LRBI_QM(NT, WR) (fours ? quant_matvec_kernel<T, NT, WR, 4> : quant_matvec_kernel<T, NT, WR, 1>)
    auto kern = nt == 2   ? (wr == 4 ? LRBI_QM(2, 4) : LRBI_QM(2, 2))
                : !column ? (wr == 4 ? LRBI_QM(1, 4) : wr == 2 ? LRBI_QM(1, 2) : LRBI_QM(1, 1))
                          : quant_matvec_kernel<T, 1, 1, 0>;
#undef LRBI_QM
    if constexpr (sizeof(T) == 4)
        if (column && wr > 1) kern = wr == 4 ? quant_matvec_kernel<T, 1, 4, 0> : quant_matvec_kernel<T, 1, 2, 0>;
    LRBI_SET_MAX_LDS(kern, smem);
    LRBI_LAUNCH(kern, wide_grid(groups, 64 * QM_WAVES), dim3(64 * QM_WAVES), smem, stream, codes, ldc, scales, lds, m, n, X, ldx, N, cols,
                (int)chunk, Y, ldy, row_blocks, workgroups);
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
