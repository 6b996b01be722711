// Weight gradient dW = (dY Xq^T) o I_a from an activation checkpoint, on the matrix cores: any shape, alignment and type (long
// batches of lined-up shapes go to the 256 x 256 form, lrbi_grad256.hip).
//
// A short batch makes the output most of the work (4096 x 9216, batch 128: 75 MB of dW, 2 MB read), so the kernel is built to keep
// stores flowing: a workgroup takes 128 x 128 blocks of dW one after the other, and while a block is multiplied, masked and
// written the first operands of the next one are on their way; its four wavefronts own 64 x 64 each, mask and write them on their own,
// and wait for each other only when a slab of 64 batch columns changes hands.
//   * dY: 16 bytes a load at any element's address, staged in LDS as [row][batch].
//   * X: staged as codes, widened when they are read by the conversion instruction that also applies the scale: exactly, but for values of
//     a wider type's checkpoint that are no f16 numbers (rounded; infinities beyond the type).
//   * fp32 dY is split into three bf16 parts, y = y1 + y2 + y3 exactly (down to 2^-133); a checkpoint's values are bf16 numbers, so three 16-bit
//     products, exact in fp32, do the work of sixteen times slower fp32 ones.
//   * output: f16 / bf16 through LDS, eight rows of 128 bytes a store; fp32 with the roles of the two operands exchanged, so that a
//     store is two rows of 128 bytes (2324 x 4839, batch 211: 63 -> 40 us).
//   * mask: tile sizes that are multiples of 64 and ranks up to 64: each wavefront fetches its block's slices of the factors before
//     the products and forms its words behind them (Eq. 3); other shapes word by word.
// 4100 x 9224, batch 131 f16 35 to 39 us (its 75 MB written alone 14), batch 40 23, batch 192 37: 16 and 7 more for each slab; 4096 x 4096,
// batch 100 f32 29; 2000 x 8000 in 300 x 320 tiles, batch 777 f16 55.  With stores, loads or products left out (4096 x 9216, batch 128, 27 us)
// 21, 23, 23: three workgroups a compute unit in turns of loading, multiplying and storing, no one of which is full.
#include <type_traits>

#include "lrbi_internal.hpp"
#include "lrbi_mfma_common.hpp"
#include "lrbi_store.hpp"

namespace lrbi {

static constexpr int CG_THREADS = 256;
static constexpr int CG_B = 128;            // rows and columns of a block of dW
static constexpr int CG_K = 64;             // batch columns per slab: two blocks of codes
static constexpr int CG_A_ROW = CG_K + 8;   // halfs of a staged row of dY
static constexpr int CG_X_ROW = CG_K + 16;  // bytes of a staged row of X
static constexpr int CG_C_ROW = 64 + 4;     // halfs of a row of a wavefront's strip of output

struct F32Tag {};
template <typename Tag> struct CgTypes {
    typedef uint16_t elem;
    typedef Tag op;
    static constexpr int parts = 1, waves = 3; // wavefronts a SIMD: workgroups that share a compute unit
};
template <> struct CgTypes<F32Tag> {
    typedef float elem;
    typedef BF16Tag op;
    static constexpr int parts = 3, waves = 2;
};
template <typename Tag> struct SmemCg {
    static constexpr int a_bytes = CG_B * CG_A_ROW * 2; // of one part
    static constexpr int x_off = CgTypes<Tag>::parts * a_bytes;
    static constexpr int s_off = x_off + CG_B * CG_X_ROW;  // [128 rows][2 blocks] scales as conversion operands
    static constexpr int w_off = s_off + CG_B * 2 * 4;     // per wavefront: factor slice [64][2], mask words [64][2]
    static constexpr int c_off = w_off + 4 * 2 * 64 * 8;   // per wavefront: 32 rows of output (16-bit types)
    static constexpr int bytes = c_off + (CgTypes<Tag>::parts == 1 ? 4 * 32 * CG_C_ROW * 2 : 0);
};

__device__ __forceinline__ uint4 cg_widen(F16Tag, uint2 w, float s) { return widen8_f16(w, s); }
__device__ __forceinline__ uint4 cg_widen(BF16Tag, uint2 w, float s) { return widen8_bf16(w, s); }

// to nearest even, as the conversion instruction has it
__device__ __forceinline__ uint16_t cg_narrow(F16Tag, float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ uint16_t cg_narrow(BF16Tag, float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

// 16 bytes of a row at any element's address, columns q on.  What lies behind column N is zero once cg_trim has seen it: a piece that the
// row's end cuts off is read as the row's last 16 bytes and moved down, when it is staged (at the load it would be waited for).
template <typename E> __device__ __forceinline__ uint4 cg_load(const E *row, int q, int N)
{
    constexpr int U = 16 / sizeof(E);
    struct __attribute__((packed, aligned(sizeof(E)))) Piece {
        uint32_t x, y, z, w;
    };
    if (N >= U) {
        const Piece p = *reinterpret_cast<const Piece *>(row + (q < N - U ? q : N - U));
        return make_uint4(p.x, p.y, p.z, p.w);
    }
    uint64_t lo = 0, hi = 0; // a row of less than 16 bytes
#pragma unroll 1
    for (int e = 0; e < U && q + e < N; ++e) {
        uint64_t v = 0;
        __builtin_memcpy(&v, row + q + e, sizeof(E));
        const int s = e * (int)sizeof(E) * 8;
        if (s < 64) lo |= v << s;
        else hi |= v << (s - 64);
    }
    return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}
template <typename E> __device__ __forceinline__ uint4 cg_trim(uint4 v, int q, int N)
{
    constexpr int U = 16 / sizeof(E);
    const int over = q - (N - U);
    if (N < U || over <= 0) return v;
    const int s = (over < U ? over : U) * (int)sizeof(E) * 8; // bits
    uint64_t lo = v.x | (uint64_t)v.y << 32, hi = v.z | (uint64_t)v.w << 32;
    lo = s >= 128 ? 0 : s >= 64 ? hi >> (s & 63) : lo >> s | hi << (64 - s);
    hi = s >= 64 ? 0 : hi >> s;
    return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

// 16 codes from column p on, zeros behind column N: p of a piece behind the last one that exists is read as that one
__device__ __forceinline__ int cg_piece(int p, int N) { return p < N ? p : (N - 1) & ~15; }
__device__ __forceinline__ uint4 cg_trim_codes(uint4 v, int p, int N)
{
    const int left = N - p; // codes that count
    if (left >= 16) return v;
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = left >= 4 * k + 4 ? w[k] : left <= 4 * k ? 0u : w[k] & ((1u << (8 * (left - 4 * k))) - 1u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Eight fp32 numbers as three bf16 parts each: cut off, not rounded, 8 of the 24 bits each; an infinity or a NaN is its first part
// alone.
__device__ __forceinline__ void cg_split(const uint4 (&y)[2], uint4 (&parts)[3])
{
    uint32_t y8[8], h[3][4];
    __builtin_memcpy(y8, y, 32);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t e3[3][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t u = y8[2 * k + e];
            const bool finite = __builtin_isfinite(__builtin_bit_cast(float, u));
            const float v = finite ? __builtin_bit_cast(float, u) - __builtin_bit_cast(float, u & 0xFFFF0000u) : 0.f;
            e3[0][e] = u;
            if (__builtin_isnan(__builtin_bit_cast(float, u))) e3[0][e] = 0x7FFF0000u; // (its bits may lie below the cut)
            e3[1][e] = __builtin_bit_cast(uint32_t, v);
            e3[2][e] = __builtin_bit_cast(uint32_t, v - __builtin_bit_cast(float, e3[1][e] & 0xFFFF0000u));
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) h[q][k] = __builtin_amdgcn_perm(e3[q][1], e3[q][0], 0x07060302u); // the upper halves
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) parts[q] = make_uint4(h[q][0], h[q][1], h[q][2], h[q][3]);
}

// What a wavefront needs for the mask words of 64 x 64 entries from (i0, j0) on, one row a lane: slices of the factors, asked for before
// the products, or the words themselves.  lined_up: tile sizes are multiples of 64, ranks up to 64 (a tile that the matrix cuts off
// has whole factors; what lies outside is not stored).
struct CgMask {
    uint32_t z[2], p[2], words[2];
};
__device__ __forceinline__ CgMask cg_mask_begin(const Geom &g, const uint32_t *__restrict__ Ip, const uint32_t *__restrict__ Iz, int64_t i0,
                                                int64_t j0, bool lined_up, int lane)
{
    CgMask q = {{0u, 0u}, {0u, 0u}, {0u, 0u}};
    if (i0 >= g.m || j0 >= g.n) return q;
    if (lined_up) {
        const int ti = (int)(i0 / g.r), tj = (int)(j0 / g.c);
        const int64_t t = (int64_t)ti * g.tile_cols + tj;
        const int il = (int)(i0 - (int64_t)ti * g.r) + lane, zw = (int)((j0 - (int64_t)tj * g.c) >> 5);
        if (lane < g.k) {
            const u32x2 v = *reinterpret_cast<const u32x2 *>(Iz + (t * g.k + lane) * g.izw + zw);
            q.z[0] = v.x;
            q.z[1] = v.y;
        }
        q.p[0] = Ip[(t * g.r + il) * g.ipw];
        if (g.ipw > 1) q.p[1] = Ip[(t * g.r + il) * g.ipw + 1];
    } else if (i0 + lane < g.m) {
        const int ti = (int)((i0 + lane) / g.r), il = (int)(i0 + lane - (int64_t)ti * g.r);
#pragma unroll
        for (int w = 0; w < 2; ++w) q.words[w] = decode_word<true>(g, Ip, Iz, ti, il, (int)(j0 >> 5) + w);
    }
    return q;
}
// fz: 64 pairs of words of the wavefront's own
__device__ __forceinline__ void cg_mask_end(CgMask &q, uint32_t *fz, bool lined_up, int lane)
{
    if (!lined_up) return;
    wave_fence();
    *reinterpret_cast<u32x2 *>(fz + lane * 2) = u32x2{q.z[0], q.z[1]};
    wave_fence();
#pragma unroll
    for (int h = 0; h < 2; ++h)
        for (uint32_t sel = q.p[h]; sel; sel &= sel - 1u) {
            const u32x2 v = *reinterpret_cast<const u32x2 *>(fz + (__builtin_ctz(sel) + 32 * h) * 2);
            q.words[0] |= v.x;
            q.words[1] |= v.y;
        }
}

template <typename Tag, bool STREAM>
__global__ __launch_bounds__(CG_THREADS, CgTypes<Tag>::waves) void checkpoint_grad_kernel(
    Geom g, const typename CgTypes<Tag>::elem *__restrict__ DY, int64_t lddy, const unsigned char *__restrict__ X, int64_t ldx,
    const unsigned char *__restrict__ XS, int64_t ldxs, int N, const uint32_t *__restrict__ Ip, const uint32_t *__restrict__ Iz,
    typename CgTypes<Tag>::elem *__restrict__ DW, int64_t lddw, uint32_t jblocks, uint32_t blocks)
{
    typedef typename CgTypes<Tag>::elem E;
    typedef typename CgTypes<Tag>::op Op;
    constexpr int PARTS = CgTypes<Tag>::parts;
    using S = SmemCg<Tag>;
    extern __shared__ uint4 lrbi_dyn_smem[];
    unsigned char *smem = (unsigned char *)lrbi_dyn_smem;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wi = wave >> 1, wj = wave & 1;
    const int l32 = lane & 31, lg = lane >> 5;
    uint32_t *fz = (uint32_t *)(smem + S::w_off + wave * 1024), *mask = fz + 128;
    const int nslabs = (N + CG_K - 1) / CG_K;
    const bool lined_up = g.c % 64 == 0 && g.r % 64 == 0 && g.k <= FAST_MAX_K;

    // a slab on its way: lane = (row tid / 8 + 32 c, eight columns tid % 8) of dY, (row tid / 4 + 64 c, 16 columns tid % 4) of X
    constexpr int AV = sizeof(E) / 2; // 16-byte pieces of eight elements
    uint4 areg[4][AV];
    uint4 xreg[2];
    uint32_t sreg[2];
    auto load = [&](uint32_t block, int slab) __attribute__((always_inline)) {
        const uint32_t ib = block / jblocks;
        const int64_t i0 = (int64_t)ib * CG_B, j0 = (int64_t)(block - ib * jblocks) * CG_B;
        const int q = slab * CG_K + (tid & 7) * 8;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t i = i0 + (tid >> 3) + 32 * c, row = i < g.m ? i : g.m - 1; // (rows past the matrix are not stored)
#pragma unroll
            for (int k = 0; k < AV; ++k) areg[c][k] = cg_load(DY + row * lddy, q + k * (16 / (int)sizeof(E)), N);
        }
        const int p = cg_piece(slab * CG_K + (tid & 3) * 16, N);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int64_t j = j0 + (tid >> 2) + 64 * c, row = j < g.n ? j : g.n - 1;
            xreg[c] = *reinterpret_cast<const uint4 *>(X + row * ldx + p);
            sreg[c] = XS[row * ldxs + (p >> 5)];
        }
    };
    auto stage = [&](int slab) __attribute__((always_inline)) {
        if ((slab + 1) * CG_K > N) { // the last slab: columns behind N are zero
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int k = 0; k < AV; ++k)
                    areg[c][k] = cg_trim<E>(areg[c][k], slab * CG_K + (tid & 7) * 8 + k * (16 / (int)sizeof(E)), N);
#pragma unroll
            for (int c = 0; c < 2; ++c) xreg[c] = cg_trim_codes(xreg[c], slab * CG_K + (tid & 3) * 16, N);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            unsigned char *dst = smem + ((tid >> 3) + 32 * c) * (CG_A_ROW * 2) + (tid & 7) * 16;
            if constexpr (PARTS == 1) {
                *reinterpret_cast<uint4 *>(dst) = areg[c][0];
            } else {
                uint4 parts[3];
                cg_split(areg[c], parts);
#pragma unroll
                for (int q = 0; q < 3; ++q)
                    *reinterpret_cast<uint4 *>(dst + q * S::a_bytes) = parts[q];
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int row = (tid >> 2) + 64 * c;
            *reinterpret_cast<uint4 *>(smem + S::x_off + row * CG_X_ROW + (tid & 3) * 16) = xreg[c];
            if ((tid & 1) == 0) *reinterpret_cast<uint32_t *>(smem + S::s_off + row * 8 + ((tid >> 1) & 1) * 4) = sreg[c] << 23;
        }
    };

    // Workgroups go to the eight XCDs in turn: each XCD takes an eighth of the blocks, neighbouring ones, whose columns of dW share lines
    // where rows are not made of whole ones, and whose workgroups share X.
    uint32_t block = blockIdx.x, step = gridDim.x, end = blocks;
    if (gridDim.x % 8 == 0) {
        const uint32_t per = (blocks + 7) / 8;
        step = gridDim.x / 8;
        block = (blockIdx.x % 8) * per + blockIdx.x / 8;
        end = (blockIdx.x % 8 + 1) * per < blocks ? (blockIdx.x % 8 + 1) * per : blocks;
    }
    if (block >= end) return; // the whole workgroup
    load(block, 0);
#pragma unroll 1
    for (; block < end; block += step) {
        const uint32_t next = block + step;
        const uint32_t ib = block / jblocks;
        // this wavefront's 64 x 64
        const int64_t i0 = (int64_t)ib * CG_B + wi * 64, j0 = (int64_t)(block - ib * jblocks) * CG_B + wj * 64;
        CgMask q = cg_mask_begin(g, Ip, Iz, i0, j0, lined_up, lane);
        // ---- products
        f32x16 acc[2][2];
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.f;
#pragma unroll 1
        for (int s = 0; s < nslabs; ++s) {
            __syncthreads(); // the slab before has been read
            stage(s);
            const bool more = s + 1 < nslabs;
            if (more || next < end) load(more ? block : next, more ? s + 1 : 0);
            __syncthreads();
            const unsigned char *as = smem + (wi * 64 + l32) * (CG_A_ROW * 2) + 16 * lg;
            const unsigned char *xs = smem + S::x_off + (wj * 64 + l32) * CG_X_ROW + 8 * lg;
            const unsigned char *ss = smem + S::s_off + (wj * 64 + l32) * 8;
            float sc[2];
#pragma unroll
            for (int kk = 0; kk < CG_K / 16; ++kk) {
                uint4 xf[2], yf[2];
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    if (kk % 2 == 0) sc[a] = *reinterpret_cast<const float *>(ss + a * 32 * 8 + kk * 2);
                    xf[a] = cg_widen(Op{}, *reinterpret_cast<const uint2 *>(xs + a * 32 * CG_X_ROW + kk * 16), sc[a]);
                }
#pragma unroll
                for (int part = PARTS - 1; part >= 0; --part) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        yf[b] = *reinterpret_cast<const uint4 *>(as + part * S::a_bytes + b * 32 * (CG_A_ROW * 2) + kk * 32);
#pragma unroll
                    for (int a = 0; a < 2; ++a)
#pragma unroll
                        for (int b = 0; b < 2; ++b)
                            acc[a][b] = PARTS == 1 ? mfma_32x32x16(Op{}, xf[a], yf[b], acc[a][b]) : mfma_32x32x16(Op{}, yf[b], xf[a], acc[a][b]);
                }
            }
        }
        cg_mask_end(q, fz, lined_up, lane);
        const uint32_t (&words)[2] = q.words;
        // ---- masked output
        if constexpr (PARTS == 1) { // per 32 x 32 block the lane holds row l32 (of dW) and columns 8 * (v / 4) + 4 * lg + (v % 4)
            wave_fence();
            *reinterpret_cast<u32x2 *>(mask + lane * 2) = u32x2{words[0], words[1]};
            int ln = lane; // what is derived from it here is not to occupy registers during the products
            asm volatile("" : "+v"(ln));
            uint16_t *strip = (uint16_t *)(smem + S::c_off) + wave * (32 * CG_C_ROW);
            const unsigned char *mb = (const unsigned char *)mask;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                wave_fence();
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int v4 = 0; v4 < 4; ++v4) {
                        uint16_t o[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = cg_narrow(Op{}, acc[a][b][4 * v4 + e]);
                        uint2 w;
                        __builtin_memcpy(&w, o, 8);
                        *reinterpret_cast<uint2 *>(strip + l32 * CG_C_ROW + a * 32 + 8 * v4 + 4 * lg) = w;
                    }
                wave_fence();
#pragma unroll
                for (int v8 = 0; v8 < 4; ++v8) { // eight rows an instruction, 128 bytes each
                    const int rr = 8 * v8 + (ln >> 3), pc = ln & 7;
                    const uint2 lo = *reinterpret_cast<const uint2 *>(strip + rr * CG_C_ROW + pc * 8);
                    const uint2 hi = *reinterpret_cast<const uint2 *>(strip + rr * CG_C_ROW + pc * 8 + 4);
                    const uint4 v = apply_mask8(make_uint4(lo.x, lo.y, hi.x, hi.y), (uint32_t)mb[(b * 32 + rr) * 8 + pc]);
                    const int64_t i = i0 + b * 32 + rr, j = j0 + pc * 8;
                    if (i >= g.m || j >= g.n) continue;
                    E *dst = DW + i * lddw + j;
                    if (j + 8 <= g.n) {
                        struct __attribute__((packed, aligned(2))) Piece { // at any element's address
                            uint32_t x, y, z, w;
                        };
                        if constexpr (STREAM) stream_store16(dst, v);
                        else *reinterpret_cast<Piece *>(dst) = {v.x, v.y, v.z, v.w};
                    } else {
                        const uint32_t w4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (j + e < g.n) dst[e] = (uint16_t)(w4[e >> 1] >> (16 * (e & 1)));
                    }
                }
            }
        } else { // the lane holds column l32 and rows 8 * (v / 4) + 4 * lg + (v % 4): a store is two rows of 128 bytes
            // Stores count with the loads, in order: a block that lies inside has no branches here, so that the wait for the next slab
            // can leave its stores on their way (4096 x 4096, batch 131: 41 -> 36.5 us; f16 / bf16, with an eighth of the stores: nothing).
            auto output = [&](auto inside_c) __attribute__((always_inline)) {
                constexpr bool inside = decltype(inside_c)::value;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int rr = b * 32 + 8 * (v >> 2) + (v & 3);
                        const int64_t i = i0 + rr + 4 * lg;
                        if (!inside && i >= g.m) continue;
                        E *dst = DW + i * lddw + j0 + l32;
#pragma unroll
                        for (int a = 0; a < 2; ++a) {
                            const uint32_t lo = __builtin_amdgcn_readlane(words[a], rr), hi = __builtin_amdgcn_readlane(words[a], rr + 4);
                            const float value = ((lg ? hi : lo) >> l32 & 1u) ? acc[a][b][v] : 0.f;
                            if constexpr (inside && STREAM) __builtin_nontemporal_store(value, dst + a * 32);
                            else if (inside || j0 + a * 32 + l32 < g.n) dst[a * 32] = value;
                        }
                    }
            };
            if (i0 + 64 <= g.m && j0 + 64 <= g.n) {
                output(std::true_type{});
            } else {
                output(std::false_type{});
                __builtin_amdgcn_s_waitcnt(0x0F70); // every load and store, so that the other path's count holds behind both
            }
        }
    }
}

// The same for few blocks: 64 x 64 of dW a workgroup, slabs of 128 batch columns, a quarter of which each wavefront multiplies; the
// four sums are added in LDS.  Bound by a slab's chain of loads, two barriers and products, so two slabs are on their way: four times the
// workgroups, half the slabs (us against the kernel above: 6793 x 203, batch 896 f16 27.6 -> 14.6; 362 x 1088, batch 557 f16 17 -> 9.4;
// 192 x 1088, batch 150 f32 18 -> 9.4; with 256 blocks of 128 x 128 it would take 12.5 instead of 9.5.  One slab under way: 256 x 256,
// batch 16384 bf16 124 instead of 96.  Operands straight from memory into the lanes, no LDS: 22 instead of 15 on the first).
static constexpr int CS_B = 64, CS_K = 128;
static constexpr int CS_A_ROW = CS_K + 8;  // halfs
static constexpr int CS_X_ROW = CS_K + 16; // bytes
static constexpr int CS_P_ROW = CS_B + 4;  // floats of a row of partial sums
template <typename Tag> struct SmemCs {
    static constexpr int a_bytes = CS_B * CS_A_ROW * 2;
    static constexpr int x_off = CgTypes<Tag>::parts * a_bytes;
    static constexpr int s_off = x_off + CS_B * CS_X_ROW; // [64 rows][4 blocks]
    static constexpr int staged = s_off + CS_B * 4 * 4;
    static constexpr int sums = 4 * CS_B * CS_P_ROW * 4; // in their place, behind the last slab
    static constexpr int w_off = staged > sums ? staged : sums; // factor slice [64][2], mask words [64][2]
    static constexpr int bytes = w_off + 2 * 64 * 8;
};

template <typename Tag>
__global__ __launch_bounds__(CG_THREADS, 2) void checkpoint_grad_small_kernel(Geom g, const typename CgTypes<Tag>::elem *__restrict__ DY,
                                                                              int64_t lddy, const unsigned char *__restrict__ X, int64_t ldx,
                                                                              const unsigned char *__restrict__ XS, int64_t ldxs, int N,
                                                                              const uint32_t *__restrict__ Ip, const uint32_t *__restrict__ Iz,
                                                                              typename CgTypes<Tag>::elem *__restrict__ DW, int64_t lddw,
                                                                              int64_t jblocks)
{
    typedef typename CgTypes<Tag>::elem E;
    typedef typename CgTypes<Tag>::op Op;
    constexpr int PARTS = CgTypes<Tag>::parts;
    using S = SmemCs<Tag>;
    extern __shared__ uint4 lrbi_dyn_smem[];
    unsigned char *smem = (unsigned char *)lrbi_dyn_smem;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, lg = lane >> 5;
    const int64_t ib = blockIdx.x / jblocks, i0 = ib * CS_B, j0 = (blockIdx.x - ib * jblocks) * CS_B;
    const int nslabs = (N + CS_K - 1) / CS_K;
    const bool lined_up = g.c % 64 == 0 && g.r % 64 == 0 && g.k <= FAST_MAX_K;

    // lane = (row tid / 16 + 16 c, eight columns tid % 16) of dY, (row tid / 8 + 32 c, 16 columns tid % 8) of X
    constexpr int AV = sizeof(E) / 2;
    struct Slab {
        uint4 a[4][AV], x[2];
        uint32_t s[2];
    } w0, w1; // two on their way
    auto load = [&](Slab &w, int slab) __attribute__((always_inline)) {
        const int q = slab * CS_K + (tid & 15) * 8;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t i = i0 + (tid >> 4) + 16 * c, row = i < g.m ? i : g.m - 1; // (rows past the matrix are not stored)
#pragma unroll
            for (int k = 0; k < AV; ++k) w.a[c][k] = cg_load(DY + row * lddy, q + k * (16 / (int)sizeof(E)), N);
        }
        const int p = cg_piece(slab * CS_K + (tid & 7) * 16, N);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int64_t j = j0 + (tid >> 3) + 32 * c, row = j < g.n ? j : g.n - 1;
            w.x[c] = *reinterpret_cast<const uint4 *>(X + row * ldx + p);
            w.s[c] = XS[row * ldxs + (p >> 5)];
        }
    };
    load(w0, 0);
    if (nslabs > 1) load(w1, 1);
    CgMask q = {};
    if (wave == 0) q = cg_mask_begin(g, Ip, Iz, i0, j0, lined_up, lane);
    f32x16 acc[2][2];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.f;
    auto slab = [&](Slab &w, int s) __attribute__((always_inline)) {
        if (s) __syncthreads(); // the slab before has been read
        if ((s + 1) * CS_K > N) { // the last slab: columns behind N are zero
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int k = 0; k < AV; ++k)
                    w.a[c][k] = cg_trim<E>(w.a[c][k], s * CS_K + (tid & 15) * 8 + k * (16 / (int)sizeof(E)), N);
#pragma unroll
            for (int c = 0; c < 2; ++c) w.x[c] = cg_trim_codes(w.x[c], s * CS_K + (tid & 7) * 16, N);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            unsigned char *dst = smem + ((tid >> 4) + 16 * c) * (CS_A_ROW * 2) + (tid & 15) * 16;
            if constexpr (PARTS == 1) {
                *reinterpret_cast<uint4 *>(dst) = w.a[c][0];
            } else {
                uint4 parts[3];
                cg_split(w.a[c], parts);
#pragma unroll
                for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4 *>(dst + k * S::a_bytes) = parts[k];
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int row = (tid >> 3) + 32 * c;
            *reinterpret_cast<uint4 *>(smem + S::x_off + row * CS_X_ROW + (tid & 7) * 16) = w.x[c];
            if ((tid & 1) == 0) *reinterpret_cast<uint32_t *>(smem + S::s_off + row * 16 + ((tid >> 1) & 3) * 4) = w.s[c] << 23;
        }
        if (s + 2 < nslabs) load(w, s + 2);
        __syncthreads();
        if (s * CS_K + wave * 32 >= N) return; // nothing in this quarter
        const unsigned char *as = smem + l32 * (CS_A_ROW * 2) + wave * 64 + 16 * lg;
        const unsigned char *xs = smem + S::x_off + l32 * CS_X_ROW + wave * 32 + 8 * lg;
        float sc[2];
#pragma unroll
        for (int a = 0; a < 2; ++a) sc[a] = *reinterpret_cast<const float *>(smem + S::s_off + (l32 + 32 * a) * 16 + wave * 4);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            uint4 xf[2], yf[2];
#pragma unroll
            for (int a = 0; a < 2; ++a) xf[a] = cg_widen(Op{}, *reinterpret_cast<const uint2 *>(xs + a * 32 * CS_X_ROW + kk * 16), sc[a]);
#pragma unroll
            for (int part = PARTS - 1; part >= 0; --part) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    yf[b] = *reinterpret_cast<const uint4 *>(as + part * S::a_bytes + b * 32 * (CS_A_ROW * 2) + kk * 32);
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int b = 0; b < 2; ++b) acc[a][b] = mfma_32x32x16(Op{}, xf[a], yf[b], acc[a][b]);
            }
        }
    };
#pragma unroll 1
    for (int s = 0; s < nslabs; s += 2) {
        slab(w0, s);
        if (s + 1 < nslabs) slab(w1, s + 1);
    }
    __syncthreads(); // the last slab has been read: the sums take its place
    float *sums = (float *)smem + wave * (CS_B * CS_P_ROW);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4)
                *reinterpret_cast<float4 *>(sums + (b * 32 + l32) * CS_P_ROW + a * 32 + 8 * v4 + 4 * lg) =
                    make_float4(acc[a][b][4 * v4], acc[a][b][4 * v4 + 1], acc[a][b][4 * v4 + 2], acc[a][b][4 * v4 + 3]);
    uint32_t *mask = (uint32_t *)(smem + S::w_off) + 128;
    if (wave == 0) {
        cg_mask_end(q, (uint32_t *)(smem + S::w_off), lined_up, lane);
        *reinterpret_cast<u32x2 *>(mask + lane * 2) = u32x2{q.words[0], q.words[1]};
    }
    __syncthreads();
    // a lane's share: 16 columns of row tid / 4
    const int row = tid >> 2, col = (tid & 3) * 16;
    const uint32_t bits = mask[row * 2 + (col >> 5)] >> (col & 31);
    const int64_t i = i0 + row, left = g.n - j0 - col;
    if (i >= g.m || left <= 0) return;
    E o[16];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float4 y = *reinterpret_cast<const float4 *>((const float *)smem + row * CS_P_ROW + col + 4 * k);
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            const float4 z = *reinterpret_cast<const float4 *>((const float *)smem + (w * CS_B + row) * CS_P_ROW + col + 4 * k);
            y.x += z.x;
            y.y += z.y;
            y.z += z.z;
            y.w += z.w;
        }
        const float e4[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v = ((bits >> (4 * k + e)) & 1u) ? e4[e] : 0.f; // pruned: exactly zero
            if constexpr (PARTS == 1) o[4 * k + e] = cg_narrow(Op{}, v);
            else o[4 * k + e] = v;
        }
    }
    E *dst = DW + i * lddw + j0 + col;
    if (left >= 16) {
        struct __attribute__((packed, aligned(sizeof(E)))) Piece { // at any element's address
            uint32_t x, y, z, w;
        };
        uint4 v[sizeof(o) / 16];
        __builtin_memcpy(v, o, sizeof(o));
#pragma unroll
        for (int k = 0; k < (int)(sizeof(o) / 16); ++k) reinterpret_cast<Piece *>(dst)[k] = {v[k].x, v[k].y, v[k].z, v[k].w};
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (e < left) dst[e] = o[e];
    }
}

template <typename Tag>
static int launch_t(const Geom &g, const void *dDY, int64_t lddy, const void *dCodes, int64_t ldc, const void *dScales, int64_t lds, int64_t N,
                    const uint32_t *dIp, const uint32_t *dIz, void *dDW, int64_t lddw, hipStream_t stream)
{
    typedef typename CgTypes<Tag>::elem E;
    const int64_t iblocks = (g.m + CG_B - 1) / CG_B, jblocks = (g.n + CG_B - 1) / CG_B, blocks = iblocks * jblocks;
    const int64_t cus = compute_units_of(stream), at_once = CgTypes<Tag>::waves * cus;
    if (2 * blocks <= cus) { // then all of the small ones run at once, two a compute unit
        const int64_t ji = (g.n + CS_B - 1) / CS_B, small = (g.m + CS_B - 1) / CS_B * ji;
        auto kern = checkpoint_grad_small_kernel<Tag>;
        LRBI_SET_MAX_LDS(kern, SmemCs<Tag>::bytes);
        LRBI_LAUNCH(kern, dim3((unsigned)small), dim3(CG_THREADS), SmemCs<Tag>::bytes, stream, g, (const E *)dDY, lddy, (const unsigned char *)dCodes,
                    ldc, (const unsigned char *)dScales, lds, (int)N, dIp, dIz, (E *)dDW, lddw, ji);
        return LRBI_OK;
    }
    if (blocks > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
    const int64_t groups = blocks < at_once ? blocks : at_once;
    // dW past the last-level cache where it does not fit it and its rows are whole lines (16384 x 16384, batch 64 bf16 137 -> 111 us; rows
    // that begin inside a line, 4100 x 9224: 23 -> 42)
    const bool stream_dw = g.m * g.n * (int64_t)sizeof(E) >= LRBI_STREAM_BYTES && (((uintptr_t)dDW | (uint64_t)(lddw * (int64_t)sizeof(E))) & 127) == 0;
    auto kern = stream_dw ? checkpoint_grad_kernel<Tag, true> : checkpoint_grad_kernel<Tag, false>;
    LRBI_SET_MAX_LDS(kern, SmemCg<Tag>::bytes);
    LRBI_LAUNCH(kern, dim3((unsigned)groups), dim3(CG_THREADS), SmemCg<Tag>::bytes, stream, g, (const E *)dDY, lddy, (const unsigned char *)dCodes,
                ldc, (const unsigned char *)dScales, lds, (int)N, dIp, dIz, (E *)dDW, lddw, (uint32_t)jblocks, (uint32_t)blocks);
    return LRBI_OK;
}

int launch_checkpoint_grad(const Geom &g, lrbi_dtype dt, const void *dDY, int64_t lddy, const void *dCodes, int64_t ldc, const void *dScales,
                           int64_t lds, int64_t N, const uint32_t *dIp, const uint32_t *dIz, void *dDW, int64_t lddw, hipStream_t stream)
{
    // The 256 x 256 form by the rule of the gradient from 16-bit X (for 256 compute units).  Us here, 256 against 128, 256 x 256 tiles of
    // rank 16:
    //   * One round: 4096 x 4096 f16, batch 64 12.2 / 12.4, 128 13.8 / 14.3, 512 23.7 / 32.8, bf16, 256 21.0 / 19.8, 1024 40.2 / 54.9; 144
    //     tiles, 2304 x 4096, bf16, 512 23.8 / 23.3, f16, 1024 28.9 / 38.7; 128 tiles, 2048 x 4096, bf16, 1024 32.6 / 31.4.
    //   * Two: 8192 x 4096, f16, 512 44.5 / 59.3, bf16, 1024 77 / 105.  More: 8192 x 8192 in 512 x 512, rank 32, bf16, 256 79 / 71, 768 131 / 156,
    //     f16, 512 90 / 118, 1024 142 / 206; 9216 x 9216, f16, 1024 196 / 267.
    // Where that rule is off here: f16 gains earlier than it says (8192 x 4096, batch 256 31 / 35; 9216 x 9216, 512 130 / 149), so do long
    // batches of half-full rounds (4096 x 9216, f16, 768 77 / 94, bf16, 1024 102 / 118; 2048 x 4096, f16, 2048 46 / 55), and tile widths of 64
    // (2 j + 1) with more than 32 ranks lose in bf16 on short ones (8192 x 8192, rank 64, 128 69 / 54; 12288 x 4096, rank 40, 128 51 / 41; f16, 256
    // 71 / 75).
    // (it addresses a block's rows of scales with 32-bit offsets too)
    if (dt != LRBI_F32 && grad256_wins(g, N) && grad256_ok(g, dDY, lddy, dCodes, ldc, N) && lds < (int64_t)1 << 22)
        return launch_grad256(g, dt, dDY, lddy, dCodes, ldc, dScales, lds, N, dIp, dIz, dDW, lddw, stream);
#define LRBI_ARGS g, dDY, lddy, dCodes, ldc, dScales, lds, N, dIp, dIz, dDW, lddw, stream
    switch (dt) {
    case LRBI_F32: return launch_t<F32Tag>(LRBI_ARGS);
    case LRBI_F16: return launch_t<F16Tag>(LRBI_ARGS);
    default: return launch_t<BF16Tag>(LRBI_ARGS);
    }
#undef LRBI_ARGS
}

} // namespace lrbi
