// Token log probabilities of a language model's logits and their gradient.  The logits are what a masked product leaves:
// x is V x N row-major, row = word, column = token.  Per column q, with m = max_v x and d_v = x_v - m,
//   s = sum_v e^d_v,  t = sum_v d_v e^d_v:   log p_v = d_v - log s,   entropy = log s - t / s,
// and the `top` largest log p_v with their words (equal ones: the lower word first).
//
// One pass over the logits.  A lane owns P neighbouring columns (one load of up to 8 bytes a row) and runs down its own
// rows, sixteen at a time: their maximum first, then one rescaling of the running (m, s, t), then sixteen exponentials.  The
// lanes of a workgroup that share a column join through LDS, the workgroups of different row slices through a partial
// (m, s, t) each in the workspace, which the finishing kernel adds up in slice order.
// Exponents are kept in base 2, e^d = 2^(x c - r) with c = log2 e and r = fl(m c): the rounding of r moves a column's sums
// and its log p by the same factor and cancels.  Beyond |m| = 2^30 that factor, and x c itself, could overflow (masks of the
// type's lowest value and nothing else): there c = 1.  Neighbouring numbers are at least 64 apart, so that e^d and 2^d are both
// 1 at the maximum and nothing elsewhere.
//
// Top words.  The rows are cut into runs of 32; the first kernel leaves the largest logit of every run and column, its row, and
// the second largest.  A word that belongs to the top K lies in a run whose maximum is not below the K-th largest of any K or
// more such maxima: the finishing wavefront takes the maxima of its 64 lanes' runs and, to 16 bits, their K-th largest as a bound.  The few
// runs that reach it give their largest word; only those whose second largest reaches it too are read again.  The words
// found are ranked by counting.  (Reading every run that reaches the bound instead: 65536 words, 256 tokens, 20 top words 32 us
// against 22 when the second largest was brought in.)
//
// Bounds.  65536 words, 4096 tokens bf16 (537 MB): the pass 96 us, reads at 5.6 TB/s; the finish 6; the gradient 198 to 205, read and
// written at 5.3 TB/s.  With top words the pass has 17.4 vector instructions a logit (counted; 8.0 without): 256 tokens, 33.5 MB, 13 to 14 us, of
// which they are 7.4 at four clocks each, with the two halves of a run loaded one after the other; the finish is one wavefront's chain of
// loads a column (9).
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <type_traits>

#include "lrbi_internal.hpp"

namespace lrbi {

static constexpr int LP_THREADS = 256;
static constexpr int LP_BATCH = 16; // rows whose maximum is taken before their exponentials
static constexpr int LP_RUN = 32;   // rows per run of the top words
static constexpr int LP_GRAD = 8;   // rows of a batch of the gradient
static constexpr float LP_LOG2E = 1.44269504088896f, LP_LN2 = 0.693147180559945f;
static constexpr float LP_HUGE = 0x1p30f;

template <typename T> struct Logit;
template <> struct Logit<float> {
    static constexpr bool can_be_huge = true;
    static constexpr float lowest = -0x1.fffffep127f; // every finite number of the type is at least this
    __device__ static float widen(float v) { return v; }
    __device__ static float narrow(float v) { return v; }
};
template <> struct Logit<__half> {
    static constexpr bool can_be_huge = false;
    static constexpr float lowest = -65504.f;
    __device__ static float widen(__half v) { return __half2float(v); }
    __device__ static __half narrow(float v) { return __float2half_rn(v); }
};
template <> struct Logit<__hip_bfloat16> {
    static constexpr bool can_be_huge = true;
    static constexpr float lowest = -0x1.fffffep127f; // every finite number of the type is at least this
    __device__ static float widen(__hip_bfloat16 v) { return __bfloat162float(v); }
    __device__ static __hip_bfloat16 narrow(float v) { return __builtin_bit_cast(__hip_bfloat16, (__bf16)v); } // nearest-even
};

// P values of a row as one load or store, at any element's address
template <typename T, int P> struct __attribute__((packed, aligned(sizeof(T)))) Piece {
    T v[P];
};
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Piece16 {
    uint32_t v[4];
};
// first column of a lane's piece: the last piece of a row that P does not divide (WHOLE: it does) begins earlier, at columns that it
// shares with its neighbour
template <int P, bool WHOLE> __device__ __forceinline__ int64_t lp_first(int64_t piece, int64_t N)
{
    const int64_t q = piece * P;
    return WHOLE || q + P <= N ? q : N - P;
}

__device__ __forceinline__ float lp_exp2(float v) { return __builtin_amdgcn_exp2f(v); }
// d as a factor of 2^d, which is 0 from -150 on: no infinity is multiplied with that 0.  (A NaN goes through 2^d.)
__device__ __forceinline__ float lp_finite(float d) { return fmaxf(d, -200.f); }

// the factor of a column's exponents, from its largest logit (see above)
template <typename T> __device__ __forceinline__ float lp_factor(float m)
{
    if constexpr (!Logit<T>::can_be_huge) return LP_LOG2E;
    return __builtin_fabsf(m) > LP_HUGE ? 1.f : LP_LOG2E;
}

// running sums of a column; m starts at the type's lowest finite number, so that nothing is subtracted from an infinity
struct LpSums {
    float m, s, t; // t in base 2
};
template <typename T> __device__ __forceinline__ LpSums lp_empty() { return {Logit<T>::lowest, 0.f, 0.f}; }

// the sums seen from a larger maximum: from the reference that they were taken at, which is the rounded product, so that
// nothing changes where the maximum stays
__device__ __forceinline__ void lp_raise(LpSums &a, float m, float c, float r)
{
#pragma clang fp contract(off)
    const float old = a.m * c, d = old - r, e = lp_exp2(d);
    a.s *= e;
    a.t = __builtin_fmaf(a.t, e, lp_finite(d) * a.s);
    a.m = m;
}
template <typename T> __device__ __forceinline__ LpSums lp_join(LpSums a, LpSums b)
{
    const float m = fmaxf(a.m, b.m), c = lp_factor<T>(m), r = m * c;
    lp_raise(a, m, c, r);
    lp_raise(b, m, c, r);
    a.s += b.s;
    a.t += b.t;
    return a;
}

template <int BYTES> struct StreamWord;
template <> struct StreamWord<2> {
    typedef uint16_t type;
};
template <> struct StreamWord<4> {
    typedef uint32_t type __attribute__((aligned(2)));
};
template <> struct StreamWord<8> {
    typedef uint32_t type __attribute__((ext_vector_type(2), aligned(2)));
};

// Rows of P columns from `src` on, rows ldl apart; COLUMN: the logits are one column without gaps (P = 1), read as
// 16-byte pieces.  STREAM: they are too many for the last-level cache.
template <typename T, int P, bool COLUMN, bool STREAM, int ROWS>
__device__ __forceinline__ void lp_load(Piece<T, P> (&x)[ROWS], const T *src, int64_t ldl, int left)
{
    if (left < ROWS) { // past the last row: words of probability 0
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (i < left) {
                x[i] = *reinterpret_cast<const Piece<T, P> *>(src + i * ldl);
            } else {
#pragma unroll
                for (int p = 0; p < P; ++p) x[i].v[p] = Logit<T>::narrow(-__builtin_inff());
            }
        }
    } else if constexpr (COLUMN) {
        constexpr int N16 = ROWS * sizeof(T) / 16;
        Piece16<T> v[N16];
#pragma unroll
        for (int i = 0; i < N16; ++i) v[i] = reinterpret_cast<const Piece16<T> *>(src)[i];
        __builtin_memcpy(x, v, sizeof(x));
    } else if constexpr (STREAM) {
        typedef typename StreamWord<P * sizeof(T)>::type Word;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const Word w = __builtin_nontemporal_load(reinterpret_cast<const Word *>(src + i * ldl));
            __builtin_memcpy(&x[i], &w, sizeof(w));
        }
    } else {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) x[i] = *reinterpret_cast<const Piece<T, P> *>(src + i * ldl);
    }
}

// The second largest logit of a run, rounded up to 27 bits, and the row of the largest in the other five.
__device__ __forceinline__ uint32_t lp_more(float second, int row)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, second);
    // a positive number with its last five bits set is not smaller, a negative one with them cleared not larger
    return (((u >> 31) ? u : u + 31u) & ~31u) | (uint32_t)row;
}
// (a second largest that is +infinity stays one; what is rounded up past the largest number is read again for nothing)
__device__ __forceinline__ float lp_second(uint32_t more) { return __builtin_bit_cast(float, more & ~31u); }

// One pass: lane (tx, ty) of a workgroup takes columns (block * tx_count + tx) P .. + P - 1 and the `runs` runs of 32 rows
// from ((slice * ty_count) + ty) * runs on.  part: [column][slice]; TOP: run_max, run_more: [column][run_pitch].
template <typename T, int P, bool WHOLE, bool COLUMN, bool TOP, bool STREAM>
__global__ __launch_bounds__(LP_THREADS) void logprobs_pass_kernel(const T *__restrict__ L, int64_t ldl, int64_t V, int64_t N,
                                                                   int tx_count, int ty_count, int64_t col_blocks, int64_t runs, int64_t slices,
                                                                   float4 *__restrict__ part, float *__restrict__ run_max,
                                                                   uint32_t *__restrict__ run_more, int64_t run_pitch)
{
    __shared__ float join[3 * P][LP_THREADS];
    const int tid = threadIdx.x;
    const int ty = tid / tx_count, tx = tid - ty * tx_count;
    const int64_t blk = wide_block();
    const int64_t slice = blk / col_blocks, cb = blk - slice * col_blocks; // neighbours read the same rows
    if (slice >= slices) return; // a workgroup past the last one
    const int64_t mine = cb * tx_count + tx, q0 = lp_first<P, WHOLE>(mine, N);
    const bool has = mine * P < N;
    LpSums a[P];
    float top[P]; // of the current run, and more of it
    uint32_t more[P];
#pragma unroll
    for (int p = 0; p < P; ++p) a[p] = lp_empty<T>();
    if (ty < ty_count && has) {
        const int64_t run0 = (slice * ty_count + ty) * runs;
        for (int64_t run = run0; run < run0 + runs && run * LP_RUN < V; ++run) {
            float second[P];
            int at[P];
            if constexpr (TOP)
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    top[p] = second[p] = -__builtin_inff();
                    at[p] = 0;
                }
#pragma unroll 1
            for (int h = 0; h < LP_RUN; h += LP_BATCH) {
                const int64_t v0 = run * LP_RUN + h;
                if (v0 >= V) break;
                const int left = V - v0 < LP_BATCH ? (int)(V - v0) : LP_BATCH;
                Piece<T, P> x[LP_BATCH];
                lp_load<T, P, COLUMN, STREAM, LP_BATCH>(x, L + v0 * ldl + q0, ldl, left);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    float b = Logit<T>::widen(x[0].v[p]);
                    if constexpr (TOP) {
                        float b2 = -__builtin_inff(); // the middle one of (x, largest, second) is the new second
#pragma unroll
                        for (int i = 1; i < LP_BATCH; ++i) {
                            const float v = Logit<T>::widen(x[i].v[p]);
                            b2 = __builtin_amdgcn_fmed3f(v, b, b2);
                            b = fmaxf(b, v);
                        }
                        int row = 0;
#pragma unroll
                        for (int i = LP_BATCH - 1; i >= 0; --i) row = Logit<T>::widen(x[i].v[p]) == b ? i : row;
                        second[p] = fmaxf(fmaxf(second[p], b2), fminf(top[p], b));
                        at[p] = b > top[p] ? h + row : at[p];
                        top[p] = fmaxf(top[p], b);
                    } else {
#pragma unroll
                        for (int i = 1; i < LP_BATCH; ++i) b = fmaxf(b, Logit<T>::widen(x[i].v[p]));
                    }
                    const float m = fmaxf(a[p].m, b), c = lp_factor<T>(m), r = m * c;
                    lp_raise(a[p], m, c, r);
#pragma unroll
                    for (int i = 0; i < LP_BATCH; ++i) {
                        const float d = __builtin_fmaf(Logit<T>::widen(x[i].v[p]), c, -r);
                        const float e = lp_exp2(d);
                        a[p].s += e;
                        a[p].t = __builtin_fmaf(lp_finite(d), e, a[p].t);
                    }
                }
            }
            if constexpr (TOP)
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    more[p] = lp_more(second[p], at[p]);
                    if (runs > 1) { // a lane's own runs lie side by side
                        run_max[(q0 + p) * run_pitch + run] = top[p];
                        run_more[(q0 + p) * run_pitch + run] = more[p];
                    }
                }
        }
    }
    if (TOP && runs == 1) { // one run a lane: those of a column together, so that its neighbours share a store
#pragma unroll
        for (int p = 0; p < P; ++p) {
            join[p][tid] = top[p];
            join[P + p][tid] = __builtin_bit_cast(float, more[p]);
        }
        __syncthreads();
        for (int e = tid; e < tx_count * P * ty_count; e += blockDim.x) {
            const int col = e / ty_count, y = e - col * ty_count, from = y * tx_count + col / P;
            const int64_t its = cb * tx_count + col / P, q = lp_first<P, WHOLE>(its, N) + col % P, run = slice * ty_count + y;
            if (its * P < N && run * LP_RUN < V) {
                run_max[q * run_pitch + run] = join[col % P][from];
                run_more[q * run_pitch + run] = __builtin_bit_cast(uint32_t, join[P + col % P][from]);
            }
        }
        __syncthreads();
    }
    // the lanes that share a column: pairs ever closer together
#pragma unroll
    for (int p = 0; p < P; ++p) {
        join[3 * p][tid] = a[p].m;
        join[3 * p + 1][tid] = a[p].s;
        join[3 * p + 2][tid] = a[p].t;
    }
    int step = 1;
    while (step < ty_count) step *= 2;
    for (step /= 2; step > 0; step /= 2) {
        __syncthreads();
        if (ty < step && ty + step < ty_count) {
            const int other = tid + step * tx_count;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                a[p] = lp_join<T>(a[p], LpSums{join[3 * p][other], join[3 * p + 1][other], join[3 * p + 2][other]});
                join[3 * p][tid] = a[p].m;
                join[3 * p + 1][tid] = a[p].s;
                join[3 * p + 2][tid] = a[p].t;
            }
        }
    }
    if (ty == 0 && has)
#pragma unroll
        for (int p = 0; p < P; ++p) part[(q0 + p) * slices + slice] = make_float4(a[p].m, a[p].s, a[p].t, 0.f);
}

static constexpr int LP_LIST = 256;  // words a wavefront holds at a time
// It looks at 256 AHEAD runs in a round: AHEAD loads of four a lane, in flight together.
template <int AHEAD> struct alignas(16) LpList {
    uint64_t key[LP_LIST + 8]; // larger: the likelier word; all different
    int run[256 * AHEAD], again[64];
};
// a logit's place among the numbers (both zeros the same), then the lower word first
__device__ __forceinline__ uint64_t lp_key(float x, int word)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
    return ((uint64_t)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32) | (uint32_t)~word;
}
__device__ __forceinline__ float lp_key_logit(uint64_t key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __builtin_bit_cast(float, o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ int lp_key_word(uint64_t key) { return (int)~(uint32_t)key; }

// The K largest keys of the list, sorted, at its start; the rest is dropped.  Returns how many there are.  A key's place is the
// number of keys above it; PER keys a lane.
template <int PER, int AHEAD> __device__ __forceinline__ int lp_rank_of(LpList<AHEAD> &l, int count, int K, int lane)
{
    wave_fence();
    if (lane < 8) l.key[count + lane] = 0; // below every key
    wave_fence();
    uint64_t k[PER];
    int rank[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        k[i] = lane + 64 * i < count ? l.key[lane + 64 * i] : 0;
        rank[i] = 0;
    }
    for (int j = 0; j < count; j += 8) {
        ulonglong2 o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = *reinterpret_cast<const ulonglong2 *>(&l.key[j + 2 * e]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < PER; ++i) rank[i] += (o[e].x > k[i] ? 1 : 0) + (o[e].y > k[i] ? 1 : 0);
    }
    wave_fence();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (k[i] && rank[i] < K) l.key[rank[i]] = k[i];
    wave_fence();
    return count < K ? count : K;
}
template <int AHEAD> __device__ __forceinline__ int lp_rank(LpList<AHEAD> &l, int count, int K, int lane)
{
    return count <= 64 ? lp_rank_of<1>(l, count, K, lane) : lp_rank_of<LP_LIST / 64>(l, count, K, lane);
}

// Four runs' maxima: -infinity past the last run
__device__ __forceinline__ void lp_runs(float (&p)[4], const float *run_max, int i, int runs)
{
    const float none = -__builtin_inff();
    const float4 v = i < runs ? *reinterpret_cast<const float4 *>(run_max + i) : make_float4(none, none, none, none);
    p[0] = v.x;
    p[1] = i + 1 < runs ? v.y : none;
    p[2] = i + 2 < runs ? v.z : none;
    p[3] = i + 3 < runs ? v.w : none;
}

// The K most likely words of column q, by one wavefront: sorted in `l`; returns how many there are (words at -infinity are
// none, nor are NaN).  run_max: the column's runs, 16-byte aligned, room for a multiple of 4; piece: the first round of them,
// run 256 k + 4 lane + e as piece[k][e].
template <typename T, int AHEAD>
__device__ __forceinline__ int lp_top(LpList<AHEAD> &l, const T *__restrict__ L, int64_t ldl, int V, int64_t q, const float *__restrict__ run_max,
                                      const uint32_t *__restrict__ run_more, int runs, float (&piece)[AHEAD][4], int K, int lane)
{
    constexpr int ROUND = 256 * AHEAD;
    typedef std::conditional_t<(AHEAD > 8), uint64_t, uint32_t> Hits; // a bit a run of the lane's
    const float none = -__builtin_inff();
    float mine = none;
    for (int i0 = 0;;) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) mine = fmaxf(mine, fmaxf(fmaxf(piece[k][0], piece[k][1]), fmaxf(piece[k][2], piece[k][3])));
        i0 += ROUND;
        if (i0 >= runs) break;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) lp_runs(piece[k], run_max, i0 + 256 * k + 4 * lane, runs);
    }
    // a bound that K lanes' maxima reach: the largest number of 16 leading bits for which that holds
    const uint32_t place = (uint32_t)(lp_key(mine, -1) >> 32);
    uint32_t leading = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit)
        if (__builtin_popcountll(__ballot(place >= (leading | 1u << bit))) >= K) leading |= 1u << bit;
    const uint64_t least_key = lp_key(none, -1) > (uint64_t)leading << 32 ? lp_key(none, -1) : (uint64_t)leading << 32;
    const float least = lp_key_logit(least_key);
    // keys that are not above `bound` are behind K others, or of no word
    const uint64_t lowest = lp_key(none, -1) | 0xFFFFFFFFu;
    uint64_t bound = least_key > lowest ? least_key : lowest;
    int count = 0;
    const uint64_t below = (1ull << lane) - 1;
    auto push = [&](uint64_t key, bool in) __attribute__((always_inline)) {
        const uint64_t all = __ballot(in && key > bound);
        if (!all) return;
        if ((all >> lane) & 1) l.key[count + __builtin_popcountll(all & below)] = key;
        count += __builtin_popcountll(all);
        if (count > LP_LIST - 64) {
            count = lp_rank_of<LP_LIST / 64>(l, count, K, lane);
            if (count == K) bound = l.key[K - 1];
        }
    };
    for (int i0 = 0; i0 < runs; i0 += ROUND) {
        // the runs that reach the bound: each lane's behind those of the lanes before it
        Hits hit = 0;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (runs > ROUND) lp_runs(piece[k], run_max, i0 + 256 * k + 4 * lane, runs); // otherwise they are there
#pragma unroll
            for (int e = 0; e < 4; ++e) hit |= piece[k][e] >= least && piece[k][e] > none ? (Hits)1 << (4 * k + e) : 0;
        }
        int end = __builtin_popcountll(hit);
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const int before = __shfl_up(end, step, 64);
            end += lane >= step ? before : 0;
        }
        const int found = __builtin_amdgcn_readlane(end, 63);
        wave_fence();
        for (int at = end - __builtin_popcountll(hit); hit; hit &= hit - 1) {
            const int bit = __builtin_ctzll(hit);
            l.run[at++] = i0 + 256 * (bit >> 2) + 4 * lane + (bit & 3);
        }
        wave_fence();
        for (int from = 0; from < found; from += 64) {
            const bool in = from + lane < found;
            const int run = l.run[in ? from + lane : from];
            const uint32_t more = run_more[run];
            const int word = run * LP_RUN + (int)(more & 31u);
            push(lp_key(run_max[run], word), in);
            // second largest: at best the run's first word
            const bool again = in && lp_second(more) > none && lp_key(lp_second(more), run * LP_RUN) > bound;
            const uint64_t all = __ballot(again);
            const int left = __builtin_popcountll(all);
            if (!left) continue;
            wave_fence();
            if (again) l.again[__builtin_popcountll(all & below)] = word;
            wave_fence();
            constexpr int LOADS = 8; // of two runs each, in flight together
            for (int a0 = 0; a0 < left; a0 += 2 * LOADS) {
                float v[LOADS];
                int w[LOADS];
                bool is[LOADS];
#pragma unroll
                for (int u = 0; u < LOADS; ++u) {
                    const int at = a0 + 2 * u + (lane >> 5), best = l.again[at < left ? at : 0];
                    w[u] = best / LP_RUN * LP_RUN + (lane & 31);
                    is[u] = at < left && w[u] < V && w[u] != best;
                    v[u] = is[u] ? Logit<T>::widen(L[w[u] * ldl + q]) : none;
                }
#pragma unroll
                for (int u = 0; u < LOADS; ++u) push(lp_key(v[u], w[u]), is[u] && v[u] > none);
            }
        }
    }
    return lp_rank(l, count, K, lane);
}

// A column's joined sums: its largest logit and the natural logarithm of its sum, written with what follows from them by lane 0.
template <typename T>
__device__ __forceinline__ float lp_write(const LpSums &a, int64_t q, int64_t V, int64_t N, int64_t word, float x, bool has_word,
                                          float *__restrict__ logp, float *__restrict__ entropy, float *__restrict__ stats, int lane)
{
    // the sum was taken at the rounded reference r: brought to the maximum itself
    const float c = lp_factor<T>(a.m), r = a.m * c, log_s = __log2f(a.s), log_m = log_s - __builtin_fmaf(a.m, c, -r);
    const float ln_s = LP_LN2 * log_m;
    if (lane == 0) {
        const bool empty = a.s == 0.f; // every logit is -infinity
        stats[q] = empty ? -__builtin_inff() : a.m;
        stats[N + q] = log_m;
        if (entropy) entropy[q] = empty ? 0.f : LP_LN2 * (log_s - a.t / a.s);
        if (has_word) logp[q] = word < 0 ? 0.f : word >= V ? __builtin_nanf("") : empty ? -__builtin_inff() : x - a.m - ln_s;
    }
    return ln_s;
}
template <typename T> __device__ __forceinline__ LpSums lp_join_lanes(LpSums a, int lanes)
{
    for (int step = 1; step < lanes; step *= 2)
        a = lp_join<T>(a, LpSums{__shfl_xor(a.m, step, 64), __shfl_xor(a.s, step, 64), __shfl_xor(a.t, step, 64)});
    return a;
}
template <int AHEAD>
__device__ __forceinline__ void lp_write_top(const LpList<AHEAD> &l, int count, const LpSums &a, float ln_s, int64_t q, int64_t N, int K,
                                             int64_t *__restrict__ top_ids, float *__restrict__ top_logp, int lane)
{
    if (lane < K) {
        top_ids[lane * N + q] = lane < count ? lp_key_word(l.key[lane]) : -1;
        top_logp[lane * N + q] = lane < count ? lp_key_logit(l.key[lane]) - a.m - ln_s : -__builtin_inff();
    }
}

// Joins a column's slices and writes its results, one wavefront a column and workgroup: few columns go to as many compute units (four
// wavefronts a workgroup, 8 ahead: 94272 words, 66 tokens, 17 top words 21.9 us against 20.8, both kernels).
// AHEAD: 0 without top words, otherwise as many as its runs fill in one round, up to 16 (us a call with 8 and 16, both kernels: 94272
// words, 66 tokens, 17 top words 21.2 / 18.9; 131072 words, 64 tokens, 20 top words 23.1 / 19.5, one token 14.6 / 12.2).
template <typename T, int AHEAD>
__global__ __launch_bounds__(64) void logprobs_finish_kernel(
    const T *__restrict__ L, int64_t ldl, int64_t V, int64_t N, const int64_t *__restrict__ tok, const float4 *__restrict__ part,
    int64_t slices, const float *__restrict__ run_max, const uint32_t *__restrict__ run_more, int64_t run_pitch, float *__restrict__ logp,
    float *__restrict__ entropy, float *__restrict__ stats, int K, int64_t *__restrict__ top_ids, float *__restrict__ top_logp)
{
    constexpr bool TOP = AHEAD > 0;
    const int lane = threadIdx.x;
    const int64_t q = wide_block();
    if (q >= N) return;
    // what the column needs is asked for at once: its word, the first round of its runs, its slices
    const int64_t word = logp ? tok[q] : -1;
    const int runs = (int)((V + LP_RUN - 1) / LP_RUN);
    const float *column_runs = TOP ? run_max + q * run_pitch : nullptr;
    float piece[TOP ? AHEAD : 1][4];
    if constexpr (TOP)
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) lp_runs(piece[k], column_runs, 256 * k + 4 * lane, runs);
    LpSums a = lp_empty<T>();
    for (int64_t i0 = 0; i0 < slices; i0 += 64 * 4) {
        float4 p[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t i = i0 + 64 * k + lane;
            p[k] = i < slices ? part[q * slices + i] : make_float4(Logit<T>::lowest, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i0 + 64 * k < slices) a = lp_join<T>(a, LpSums{p[k].x, p[k].y, p[k].z});
    }
    const float x = word >= 0 && word < V ? Logit<T>::widen(L[word * ldl + q]) : 0.f;
    a = lp_join_lanes<T>(a, 64);
    const float ln_s = lp_write<T>(a, q, V, N, word, x, logp != nullptr, logp, entropy, stats, lane);
    if constexpr (TOP) {
        __shared__ LpList<AHEAD> l;
        const int count = lp_top(l, L, ldl, (int)V, q, column_runs, run_more + q * run_pitch, runs, piece, K, lane);
        lp_write_top(l, count, a, ln_s, q, N, K, top_ids, top_logp, lane);
    }
}

// A single column without gaps, up to 32768 words, in one launch: a word of a served sequence.  1024 lanes take eight words at a
// time, four lanes a run; the runs stay in LDS.  (Us a call against two launches: 10000 words f16, 8 top words 8.7 / 11.7, the kernel 7.0;
// 32768 words bf16, 20 top words 9.5 / 11.5, none 7.9 / 10.7.)
static constexpr int LP_COLUMN_LANES = 1024;
static constexpr int LP_COLUMN_SWEEPS = 4;
static constexpr int LP_COLUMN_MOST = LP_COLUMN_LANES * 8 * LP_COLUMN_SWEEPS;
template <typename T, bool TOP>
__global__ __launch_bounds__(LP_COLUMN_LANES) void logprobs_column_kernel(const T *__restrict__ L, int V, const int64_t *__restrict__ tok,
                                                                          float *__restrict__ logp, float *__restrict__ entropy,
                                                                          float *__restrict__ stats, int K, int64_t *__restrict__ top_ids,
                                                                          float *__restrict__ top_logp)
{
    __shared__ float4 run_max4[TOP ? LP_COLUMN_MOST / LP_RUN / 4 : 1];
    __shared__ uint32_t run_more[TOP ? LP_COLUMN_MOST / LP_RUN : 1];
    __shared__ LpSums join[LP_COLUMN_LANES / 64];
    float *run_max = (float *)run_max4;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float none = -__builtin_inff();
    const int64_t word = logp ? tok[0] : -1;
    float x[LP_COLUMN_SWEEPS][8];
#pragma unroll
    for (int s = 0; s < LP_COLUMN_SWEEPS; ++s) {
        const int v0 = (s * LP_COLUMN_LANES + tid) * 8;
        if (v0 + 8 <= V) {
            Piece16<T> p[sizeof(T) / 2];
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) p[i] = reinterpret_cast<const Piece16<T> *>(L + v0)[i];
            T e[8];
            __builtin_memcpy(e, p, sizeof(e));
#pragma unroll
            for (int i = 0; i < 8; ++i) x[s][i] = Logit<T>::widen(e[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[s][i] = v0 + i < V ? Logit<T>::widen(L[v0 + i]) : none;
        }
    }
    const float own = word >= 0 && word < V ? Logit<T>::widen(L[word]) : 0.f;
    LpSums a = lp_empty<T>();
#pragma unroll
    for (int s = 0; s < LP_COLUMN_SWEEPS; ++s) {
        if (s * LP_COLUMN_LANES * 8 >= V) break;
        float b = x[s][0], b2 = none; // largest and second largest
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            b2 = __builtin_amdgcn_fmed3f(x[s][i], b, b2);
            b = fmaxf(b, x[s][i]);
        }
        a.m = fmaxf(a.m, b);
        if constexpr (TOP) {
            int row = 0;
#pragma unroll
            for (int i = 7; i >= 0; --i) row = x[s][i] == b ? i : row;
            row += (lane & 3) * 8;
            b = fmaxf(b, none); // (NaN alone: none)
#pragma unroll
            for (int step = 1; step < 4; step *= 2) {
                const float o = __shfl_xor(b, step, 64), o2 = __shfl_xor(b2, step, 64);
                const int other = __shfl_xor(row, step, 64);
                b2 = fmaxf(fmaxf(b2, o2), fminf(b, o));
                row = o > b || (o == b && other < row) ? other : row;
                b = fmaxf(b, o);
            }
            if ((lane & 3) == 0) {
                const int run = (s * LP_COLUMN_LANES + tid) / 4;
                run_max[run] = b;
                run_more[run] = lp_more(b2, row);
            }
        }
    }
    const float c = lp_factor<T>(a.m), r = a.m * c;
#pragma unroll
    for (int s = 0; s < LP_COLUMN_SWEEPS; ++s) {
        if (s * LP_COLUMN_LANES * 8 >= V) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = __builtin_fmaf(x[s][i], c, -r), e = lp_exp2(d);
            a.s += e;
            a.t = __builtin_fmaf(lp_finite(d), e, a.t);
        }
    }
    a = lp_join_lanes<T>(a, 64);
    if (lane == 0) join[wave] = a;
    __syncthreads();
    if (wave > 0) return;
    a = lp_join_lanes<T>(join[lane & 15], 16);
    const float ln_s = lp_write<T>(a, 0, V, 1, word, own, logp != nullptr, logp, entropy, stats, lane);
    if constexpr (TOP) {
        constexpr int AHEAD = LP_COLUMN_MOST / LP_RUN / 256; // one round
        __shared__ LpList<AHEAD> l;
        const int runs = (V + LP_RUN - 1) / LP_RUN;
        float piece[AHEAD][4];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) lp_runs(piece[k], run_max, 256 * k + 4 * lane, runs);
        const int count = lp_top(l, L, 1, V, 0, run_max, run_more, runs, piece, K, lane);
        lp_write_top(l, count, a, ln_s, 0, 1, K, top_ids, top_logp, lane);
    }
}
static_assert(LP_COLUMN_LANES == 16 * 64 && LP_COLUMN_MOST % (256 * LP_RUN) == 0, "one partial a lane of 16, one round of runs");

// dx_v = gl (1[v = word] - p_v) - gh p_v (log p_v + entropy); a lane owns P columns and the `batches` batches of 8 rows from
// ((block * ty_count) + ty) * batches on.  DL may be L: a batch is read whole before any of it is
// written, and what a lane reads of a neighbour's columns it does not use.
template <typename T, int P, bool WHOLE>
__global__ __launch_bounds__(LP_THREADS) void logprobs_grad_kernel(const T *L, int64_t ldl, int64_t V, int64_t N,
                                                                   const int64_t *__restrict__ tok, const float *__restrict__ stats,
                                                                   const float *__restrict__ entropy, const float *__restrict__ g_logp,
                                                                   const float *__restrict__ g_entropy, T *DL, int64_t lddl,
                                                                   int tx_count, int ty_count, int64_t col_blocks, int64_t batches)
{
    __shared__ float column[7][64 * P]; // factor, reference, log2 of the sum, the two gradients, entropy, word of every column
    const int tid = threadIdx.x;
    const int ty = tid / tx_count, tx = tid - ty * tx_count;
    const int64_t blk = wide_block();
    const int64_t rb = blk / col_blocks, cb = blk - rb * col_blocks; // neighbours read the same rows
    const int64_t mine = cb * tx_count + tx, q0 = lp_first<P, WHOLE>(mine, N), first = (rb * ty_count + ty) * batches * LP_GRAD;
    const int shared = (int)(mine * P - q0); // columns that are the neighbour's to write
    for (int e = tid; e < tx_count * P; e += blockDim.x) {
        const int64_t its = cb * tx_count + e / P, q = lp_first<P, WHOLE>(its, N) + e % P;
        if (its * P >= N) break;
        const float m = fmaxf(stats[q], Logit<T>::lowest), c = lp_factor<T>(m), r = m * c;
        float log_s = stats[N + q] + __builtin_fmaf(m, c, -r);
        const int64_t w = g_logp ? tok[q] : -1;
        float gl = w < 0 ? 0.f : g_logp[q];
        const float gh = g_entropy ? g_entropy[q] * LP_LN2 : 0.f; // log p below is in base 2
        float h = g_entropy ? entropy[q] * LP_LOG2E : 0.f;
        // Columns that hold a NaN or +infinity, and words that are none: NaN, through gl, since log p is cut below.
        // No gradient comes in: none goes out, whatever the logits.  A column of -infinity alone: every p is 0.
        const bool none = gl == 0.f && gh == 0.f;
        if (!none && (w >= V || log_s != log_s)) gl = __builtin_nanf("");
        if (none) h = 0.f;
        if (none || log_s == -__builtin_inff()) log_s = 0.f;
        column[0][e] = c;
        column[1][e] = r;
        column[2][e] = log_s;
        column[3][e] = gl;
        column[4][e] = gh;
        column[5][e] = h;
        column[6][e] = __builtin_bit_cast(float, w >= 0 && w < V ? (int)w : -1);
    }
    __syncthreads();
    if (ty >= ty_count || mine * P >= N || first >= V) return;
    float c[P], r[P], log_s[P], gl[P], gh[P], h[P];
    int word[P]; // from the lane's first row on
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int e = tx * P + p;
        c[p] = column[0][e];
        r[p] = column[1][e];
        log_s[p] = column[2][e];
        gl[p] = column[3][e];
        gh[p] = column[4][e];
        h[p] = column[5][e];
        const int64_t w = __builtin_bit_cast(int, column[6][e]);
        word[p] = w >= first && w < first + batches * LP_GRAD ? (int)(w - first) : -1;
    }
    const auto batch = [&](int64_t v0, auto words) {
        const int left = V - v0 < LP_GRAD ? (int)(V - v0) : LP_GRAD;
        Piece<T, P> x[LP_GRAD];
        lp_load<T, P, false, false, LP_GRAD>(x, L + v0 * ldl + q0, ldl, left);
        T *dst = DL + v0 * lddl + q0;
#pragma unroll
        for (int i = 0; i < LP_GRAD; ++i) {
            Piece<T, P> o;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                // (a NaN becomes -200)
                const float l = __builtin_amdgcn_fmed3f(__builtin_fmaf(Logit<T>::widen(x[i].v[p]), c[p], -r[p]) - log_s[p], -200.f, 1.f);
                float g = -lp_exp2(l) * __builtin_fmaf(gh[p], l + h[p], gl[p]);
                if constexpr (decltype(words)::value) g += word[p] == (int)(v0 - first) + i ? gl[p] : 0.f;
                o.v[p] = Logit<T>::narrow(g);
            }
            if (i >= left) continue;
            if (WHOLE || shared == 0) {
                *reinterpret_cast<Piece<T, P> *>(dst + i * lddl) = o;
            } else {
#pragma unroll
                for (int p = 1; p < P; ++p)
                    if (p >= shared) dst[i * lddl + p] = o.v[p];
            }
        }
    };
#pragma unroll 1
    for (int64_t v0 = first; v0 < first + batches * LP_GRAD && v0 < V; v0 += LP_GRAD) {
        bool here = false; // few batches hold one of the wavefront's words
#pragma unroll
        for (int p = 0; p < P; ++p) here = here || (word[p] >= 0 && word[p] / LP_GRAD == (int)(v0 - first) / LP_GRAD);
        if (__any(here)) batch(v0, std::true_type{});
        else batch(v0, std::false_type{});
    }
}

// Columns per lane and lanes per row.  Wider pieces of P columns, one load each, need fewer instructions a column, and fewer lanes:
// they are taken while `lanes` of them with `rows` rows each are left (131072: two wavefronts on every SIMD).  P divides N and
// the row pitch and the base is aligned to it, if 8 bytes or more can be had that way; otherwise the widest at any address, the last
// piece of a row shared with its neighbour (us, loss and gradient: 71485 words, 1877 columns f32 461 -> 403 against one column a
// lane; 41089 words, 2561 columns f16 224 -> 187; 50000 words, 300 columns f16 40 in 16 bytes at any address, 35 in aligned 8).
struct LpShape {
    int p, tx, ty;
    int64_t col_blocks;
};
static LpShape lp_shape(int es, int64_t V, int64_t N, int64_t bits, int rows, int most_bytes, int least, int64_t lanes)
{
    LpShape s;
    s.p = 1;
    const int64_t pieces_of_rows = (V + rows - 1) / rows;
    for (int pass = 0; pass < 2 && s.p == 1; ++pass)
        for (int p = most_bytes / es; p > 1; p /= 2) {
            if (pass == 0 && (p * es < 8 || N % p != 0 || (bits & (p * es - 1)) != 0)) continue;
            if (p > N || (p > least && pieces_of_rows * ((N + p - 1) / p) < lanes)) continue;
            s.p = p;
            break;
        }
    const int64_t pieces = (N + s.p - 1) / s.p;
    // few lanes in all: workgroups of one wavefront, so that more compute units take part
    const int threads = pieces_of_rows * pieces <= 16384 ? 64 : LP_THREADS;
    s.col_blocks = (pieces + 63) / 64;
    s.tx = (int)((pieces + s.col_blocks - 1) / s.col_blocks); // (300 columns in 75 pieces: 38 and 37 lanes, not 64 and 11)
    s.ty = threads / s.tx;
    return s;
}

// Workgroups of the pass kernel; the workspace holds four numbers per column and slice, then two per column and run of the top words.
struct LpPlan {
    LpShape shape;
    int64_t runs, slices, run_pitch;
    uint64_t part_bytes, bytes;
};
static LpPlan lp_plan(int es, int64_t V, int64_t N, int32_t top)
{
    LpPlan p;
    // The top words' comparisons are hidden by more wavefronts (us a call, 8-byte pieces and 2-byte ones, bf16: 65536 words, 256 tokens
    // 23.6 / 21.7, 11 tokens 13.4 / 13.0; 10000 words, 200 tokens 13.5 / 12.7; 131072 words, 64 tokens 19.0 / 19.5).
    p.shape = top > 0 ? lp_shape(es, V, N, 0, LP_RUN, 8, 1, 524288) : lp_shape(es, V, N, 0, LP_RUN, 8, 2, 131072);
    const int64_t all = (V + LP_RUN - 1) / LP_RUN;
    // runs a lane: as many as leave 2048 workgroups, eight for each compute unit
    const int64_t groups = (all + p.shape.ty - 1) / p.shape.ty * p.shape.col_blocks;
    p.runs = groups / 2048 > 1 ? groups / 2048 : 1;
    p.slices = (all + p.runs * p.shape.ty - 1) / (p.runs * p.shape.ty);
    p.run_pitch = (all + 3) / 4 * 4;
    p.part_bytes = (uint64_t)p.slices * 16 * (uint64_t)N;
    p.bytes = p.part_bytes + (top > 0 ? (uint64_t)p.run_pitch * (uint64_t)N * 8 : 0);
    return p;
}
uint64_t logprobs_workspace_bytes(int es, int64_t V, int64_t N, int32_t top) { return lp_plan(es, V, N, top).bytes; }

template <typename T>
static int launch_logprobs_t(const T *L, int64_t ldl, int64_t V, int64_t N, const int64_t *tok, float *logp, float *entropy,
                             float *stats, int32_t top, int64_t *top_ids, float *top_logp, void *ws, hipStream_t stream)
{
    const bool column = N == 1 && ldl == 1;
    if (column && V <= LP_COLUMN_MOST) {
        auto kern = top > 0 ? logprobs_column_kernel<T, true> : logprobs_column_kernel<T, false>;
        LRBI_LAUNCH(kern, dim3(1), dim3(LP_COLUMN_LANES), 0, stream, L, (int)V, tok, logp, entropy, stats, top, top_ids, top_logp);
        return LRBI_OK;
    }
    const LpPlan p = lp_plan((int)sizeof(T), V, N, top);
    float4 *part = (float4 *)ws;
    float *run_max = (float *)((char *)ws + p.part_bytes);
    uint32_t *run_more = (uint32_t *)run_max + p.run_pitch * N;
    const int threads = p.shape.tx * p.shape.ty <= 64 ? 64 : LP_THREADS;
    const int64_t blocks = p.shape.col_blocks * p.slices;
    if (blocks > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
#define LRBI_PASS_TOP(P, WHOLE, COLUMN, TOP, STREAM)                                                                       \
    LRBI_LAUNCH((logprobs_pass_kernel<T, P, WHOLE, COLUMN, TOP, STREAM>), wide_grid(blocks, threads), dim3(threads), 0, stream, L, ldl, V, \
                N, p.shape.tx, p.shape.ty, p.shape.col_blocks, p.runs, p.slices, part, run_max, run_more, p.run_pitch)
#define LRBI_PASS(P, WHOLE, COLUMN)                                                                                        \
    do {                                                                                                                   \
        if (top > 0) LRBI_PASS_TOP(P, WHOLE, COLUMN, true, false);                                                         \
        else if (!COLUMN && past_cache) LRBI_PASS_TOP(P, WHOLE, COLUMN, false, !COLUMN);                                   \
        else LRBI_PASS_TOP(P, WHOLE, COLUMN, false, false);                                                                \
    } while (0)
    const bool whole = N % p.shape.p == 0;
    // Logits that do not fit the last-level cache, rows of whole lines (us, 65536 words, 4096 tokens bf16 107 -> 96; 71485 words, 1877 columns
    // f32, whose rows share lines, with the gradient 403 -> 413; the gradient's loads that way: 300 -> 303)
    const bool past_cache = V * N * (int64_t)sizeof(T) >= LRBI_STREAM_BYTES && (((uintptr_t)L | (uint64_t)(ldl * (int64_t)sizeof(T))) & 127) == 0;
    switch (p.shape.p) {
    case 1:
        if (column) LRBI_PASS(1, true, true);
        else LRBI_PASS(1, true, false);
        break;
    case 2:
        if (whole) LRBI_PASS(2, true, false);
        else LRBI_PASS(2, false, false);
        break;
    default:
        if constexpr (sizeof(T) == 2) {
            if (whole) LRBI_PASS(4, true, false);
            else LRBI_PASS(4, false, false);
        }
        break;
    }
#undef LRBI_PASS
#undef LRBI_PASS_TOP
#define LRBI_FINISH(AHEAD)                                                                                                   \
    LRBI_LAUNCH((logprobs_finish_kernel<T, AHEAD>), wide_grid(N, 64), dim3(64), 0, stream, L, ldl, V, N, tok, part,  \
                p.slices, run_max, run_more, p.run_pitch, logp, entropy, stats, top, top_ids, top_logp)
    if (top == 0) LRBI_FINISH(0);
    else if (V <= 256 * 4 * LP_RUN) LRBI_FINISH(4);
    else if (V <= 256 * 8 * LP_RUN) LRBI_FINISH(8);
    else LRBI_FINISH(16);
#undef LRBI_FINISH
    return LRBI_OK;
}
int launch_logprobs(lrbi_dtype dt, const void *dL, int64_t ldl, int64_t V, int64_t N, const int64_t *dTok, float *dLogp, float *dEntropy,
                    float *dStats, int32_t top, int64_t *dTopIds, float *dTopLogp, void *ws, hipStream_t stream)
{
#define LRBI_ARGS(T) (const T *)dL, ldl, V, N, dTok, dLogp, dEntropy, dStats, top, dTopIds, dTopLogp, ws, stream
    switch (dt) {
    case LRBI_F32: return launch_logprobs_t<float>(LRBI_ARGS(float));
    case LRBI_F16: return launch_logprobs_t<__half>(LRBI_ARGS(__half));
    default: return launch_logprobs_t<__hip_bfloat16>(LRBI_ARGS(__hip_bfloat16));
    }
#undef LRBI_ARGS
}

template <typename T>
static int launch_logprobs_grad_t(const T *L, int64_t ldl, int64_t V, int64_t N, const int64_t *tok, const float *stats,
                                  const float *entropy, const float *g_logp, const float *g_entropy, T *DL, int64_t lddl,
                                  hipStream_t stream)
{
    const int64_t bits = (int64_t)((uintptr_t)L | (uintptr_t)DL) | (ldl | lddl) * (int64_t)sizeof(T);
    const LpShape s = lp_shape((int)sizeof(T), V, N, bits, LP_GRAD, 16, 2, 131072);
    const int threads = s.tx * s.ty <= 64 ? 64 : LP_THREADS;
    // batches a lane, for whose columns it reads 28 bytes each: up to eight while 2048 workgroups are left
    int64_t batches = (V + LP_GRAD - 1) / LP_GRAD / s.ty * s.col_blocks / 2048;
    batches = batches < 1 ? 1 : batches > 8 ? 8 : batches;
    const int64_t rows = s.ty * batches * LP_GRAD, row_blocks = (V + rows - 1) / rows, blocks = s.col_blocks * row_blocks;
    if (blocks > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
#define LRBI_GRAD(P, WHOLE)                                                                                                \
    LRBI_LAUNCH((logprobs_grad_kernel<T, P, WHOLE>), wide_grid(blocks, threads), dim3(threads), 0, stream, L, ldl, V, N, tok, stats,  \
                entropy, g_logp, g_entropy, DL, lddl, s.tx, s.ty, s.col_blocks, batches)
    const bool whole = N % s.p == 0;
    switch (s.p) {
    case 1: LRBI_GRAD(1, true); break;
    case 2:
        if (whole) LRBI_GRAD(2, true);
        else LRBI_GRAD(2, false);
        break;
    case 4:
        if (whole) LRBI_GRAD(4, true);
        else LRBI_GRAD(4, false);
        break;
    default:
        if constexpr (sizeof(T) == 2) {
            if (whole) LRBI_GRAD(8, true);
            else LRBI_GRAD(8, false);
        }
        break;
    }
#undef LRBI_GRAD
    return LRBI_OK;
}
int launch_logprobs_grad(lrbi_dtype dt, const void *dL, int64_t ldl, int64_t V, int64_t N, const int64_t *dTok, const float *dStats,
                         const float *dEntropy, const float *dGLogp, const float *dGEntropy, void *dDL, int64_t lddl,
                         hipStream_t stream)
{
#define LRBI_ARGS(T) (const T *)dL, ldl, V, N, dTok, dStats, dEntropy, dGLogp, dGEntropy, (T *)dDL, lddl, stream
    switch (dt) {
    case LRBI_F32: return launch_logprobs_grad_t<float>(LRBI_ARGS(float));
    case LRBI_F16: return launch_logprobs_grad_t<__half>(LRBI_ARGS(__half));
    default: return launch_logprobs_grad_t<__hip_bfloat16>(LRBI_ARGS(__hip_bfloat16));
    }
#undef LRBI_ARGS
}

} // namespace lrbi
