// Token log probabilities of a language model's logits and their gradient.  The logits are what a masked product leaves:
// x is V x N row-major, row = word, column = token.  Per column q, with m = max_v x and d_v = x_v - m,
//   s = sum_v e^d_v,  t = sum_v d_v e^d_v:   log p_v = d_v - log s,   entropy = log s - t / s,
// and the `top` largest log p_v with their words (equal ones: the lower word first).
//
// One pass over the logits.  A lane owns P neighbouring columns (one load of up to 16 bytes a row) and runs down its own
// rows, sixteen at a time: their maximum first, then one rescaling of the running (m, s, t), then sixteen exponentials.  The
// lanes of a workgroup that share a column join through LDS, the workgroups of different row slices through a partial
// (m, s, t) each in the workspace, which the finishing kernel adds up in slice order.
// Exponents are kept in base 2, e^d = 2^(x c - r) with c = log2 e and r = fl(m c): the rounding of r moves a column's sums
// and its log p by the same factor and cancels.  Beyond |m| = 2^30 that factor, and x c itself, could overflow (masks of the
// type's lowest value and nothing else): there c = 1.  Neighbouring numbers are at least 64 apart, so that e^d and 2^d are both
// 1 at the maximum and nothing elsewhere.
//
// Top words.  The rows are cut into runs of 32; the first kernel leaves the maximum of every run and column.  A word that
// belongs to the top K lies in a run whose maximum is not below the K-th largest of any K or more such maxima: the
// finishing wavefront takes the 64 maxima of its lanes' runs, their K-th largest as a bound, reads the few runs that reach it
// and ranks the words that reach it by counting.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "lrbi_internal.hpp"

namespace lrbi {

static constexpr int LP_THREADS = 256;
static constexpr int LP_BATCH = 16; // rows whose maximum is taken before their exponentials
static constexpr int LP_RUN = 32;   // rows per run of the top words
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
    __device__ static __hip_bfloat16 narrow(float v) { return __float2bfloat16(v); }
};

// P values of a row as one load or store
template <typename T, int P> struct alignas(sizeof(T) * P) Piece {
    T v[P];
};

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

// One pass: lane (tx, ty) of a workgroup takes columns (block * tx_count + tx) P .. + P - 1 and the `runs` runs of 32 rows
// from ((slice * ty_count) + ty) * runs on.  part: [slice][3][N].  run_max: [run][N], or NULL.
template <typename T, int P>
__global__ __launch_bounds__(LP_THREADS) void logprobs_pass_kernel(const T *__restrict__ L, int64_t ldl, int64_t V, int64_t N,
                                                                   int tx_count, int ty_count, int64_t runs, int64_t slices,
                                                                   float *__restrict__ part, float *__restrict__ run_max)
{
    __shared__ float join[3 * P][LP_THREADS];
    const int tid = threadIdx.x;
    const int ty = tid / tx_count, tx = tid - ty * tx_count;
    const int64_t blk = wide_block();
    const int64_t cb = blk / slices, slice = blk - cb * slices;
    const int64_t q0 = (cb * tx_count + tx) * P;
    if (cb * tx_count * P >= N) return; // a workgroup past the last one
    LpSums a[P];
#pragma unroll
    for (int p = 0; p < P; ++p) a[p] = lp_empty<T>();
    if (ty < ty_count && q0 < N) {
        const int64_t run0 = (slice * ty_count + ty) * runs;
        for (int64_t run = run0; run < run0 + runs && run * LP_RUN < V; ++run) {
            float top[P];
#pragma unroll
            for (int p = 0; p < P; ++p) top[p] = -__builtin_inff();
#pragma unroll 1
            for (int h = 0; h < LP_RUN; h += LP_BATCH) {
                const int64_t v0 = run * LP_RUN + h;
                if (v0 >= V) break;
                const T *src = L + v0 * ldl + q0;
                Piece<T, P> x[LP_BATCH];
                const int left = V - v0 < LP_BATCH ? (int)(V - v0) : LP_BATCH;
                if (left == LP_BATCH) {
#pragma unroll
                    for (int i = 0; i < LP_BATCH; ++i) x[i] = *reinterpret_cast<const Piece<T, P> *>(src + i * ldl);
                } else { // past the last row: the last one again, and not counted
#pragma unroll
                    for (int i = 0; i < LP_BATCH; ++i)
                        x[i] = *reinterpret_cast<const Piece<T, P> *>(src + (i < left ? i : left - 1) * ldl);
                }
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    float b = Logit<T>::widen(x[0].v[p]);
#pragma unroll
                    for (int i = 1; i < LP_BATCH; ++i) b = fmaxf(b, Logit<T>::widen(x[i].v[p]));
                    top[p] = fmaxf(top[p], b);
                    const float m = fmaxf(a[p].m, b), c = lp_factor<T>(m), r = m * c;
                    lp_raise(a[p], m, c, r);
#pragma unroll
                    for (int i = 0; i < LP_BATCH; ++i) {
                        const float d = __builtin_fmaf(Logit<T>::widen(x[i].v[p]), c, -r);
                        float e = lp_exp2(d);
                        if (left != LP_BATCH && i >= left) e = 0.f;
                        a[p].s += e;
                        a[p].t = __builtin_fmaf(lp_finite(d), e, a[p].t);
                    }
                }
            }
            if (run_max)
#pragma unroll
                for (int p = 0; p < P; ++p)
                    if (q0 + p < N) run_max[run * N + q0 + p] = top[p];
        }
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
    if (ty == 0)
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (q0 + p < N) {
                float *o = part + slice * 3 * N + q0 + p;
                o[0] = a[p].m;
                o[N] = a[p].s;
                o[2 * N] = a[p].t;
            }
}

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

static constexpr int LP_LIST = 256; // words a wavefront holds at a time
struct LpList {
    float value[LP_LIST];
    int64_t word[LP_LIST];
    int64_t run[LP_THREADS]; // runs to read
};

// The K best words of the list, sorted, at its start; the rest is dropped.  Returns how many there are.
__device__ __forceinline__ int lp_rank(LpList &l, int count, int K, int lane)
{
    float v[LP_LIST / 64];
    int64_t w[LP_LIST / 64];
    int rank[LP_LIST / 64];
    wave_sync();
#pragma unroll
    for (int i = 0; i < LP_LIST / 64; ++i) {
        const int at = lane + 64 * i;
        v[i] = at < count ? l.value[at] : 0.f;
        w[i] = at < count ? l.word[at] : 0;
        rank[i] = at < count ? 0 : LP_LIST;
    }
    for (int j = 0; j < count; ++j) {
        const float vj = l.value[j];
        const int64_t wj = l.word[j];
#pragma unroll
        for (int i = 0; i < LP_LIST / 64; ++i) rank[i] += (vj > v[i] || (vj == v[i] && wj < w[i])) ? 1 : 0;
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < LP_LIST / 64; ++i)
        if (rank[i] < K) {
            l.value[rank[i]] = v[i];
            l.word[rank[i]] = w[i];
        }
    wave_sync();
    return count < K ? count : K;
}

// The K most likely words of column q, by one wavefront: sorted in `l`; returns how many there are (words at -infinity are
// none, nor are NaN).
template <typename T>
__device__ int lp_top(LpList &l, const T *__restrict__ L, int64_t ldl, int64_t V, int64_t N, int64_t q, const float *__restrict__ run_max,
                      int K, int lane)
{
    const int64_t runs = (V + LP_RUN - 1) / LP_RUN;
    const float none = -__builtin_inff();
    float mine = none;
    for (int64_t i = lane; i < runs; i += 64) mine = fmaxf(mine, run_max[i * N + q]);
    int rank = 0;
    for (int j = 0; j < 64; ++j) {
        const float v = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, mine), j));
        rank += (v > mine || (v == mine && j < lane)) ? 1 : 0;
    }
    // a word below `bound` is behind K others; once K words are held, so is an equal one that comes later
    float bound = __shfl(mine, __builtin_ctzll(__ballot(rank == K - 1)), 64);
    bool full = false;
    int count = 0, waiting = 0;
    constexpr int LOADS = 8; // of two runs each, in flight together
    auto read = [&]() {
        wave_sync();
        float v[LOADS];
        int64_t w[LOADS];
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int at = 2 * u + (lane >> 5);
            w[u] = at < waiting ? l.run[at] * LP_RUN + (lane & 31) : V;
            v[u] = w[u] < V ? Logit<T>::widen(L[w[u] * ldl + q]) : none;
        }
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const uint64_t in = __ballot(v[u] > none && (full ? v[u] > bound : v[u] >= bound));
            if (!in) continue;
            if (count > LP_LIST - 64) {
                count = lp_rank(l, count, K, lane);
                if (count == K) {
                    bound = l.value[K - 1];
                    full = true;
                }
            }
            if ((in >> lane) & 1) {
                const int at = count + __builtin_popcountll(in & ((1ull << lane) - 1));
                l.value[at] = v[u];
                l.word[at] = w[u];
            }
            count += __builtin_popcountll(in);
        }
        // the runs that were not read move to the front
        wave_sync();
        const int64_t next = lane + 2 * LOADS < waiting ? l.run[lane + 2 * LOADS] : 0;
        wave_sync();
        l.run[lane] = next;
        waiting = waiting > 2 * LOADS ? waiting - 2 * LOADS : 0;
    };
    for (int64_t i0 = 0; i0 < runs; i0 += 64) {
        const float v = i0 + lane < runs ? run_max[(i0 + lane) * N + q] : none;
        const bool in = v > none && (full ? v > bound : v >= bound);
        const uint64_t all = __ballot(in);
        if (in) l.run[waiting + __builtin_popcountll(all & ((1ull << lane) - 1))] = i0 + lane;
        waiting += __builtin_popcountll(all);
        while (waiting >= 2 * LOADS) read();
    }
    if (waiting) read();
    return lp_rank(l, count, K, lane);
}

// Joins the slices of 16 columns and writes their results; with TOP, wavefront w finds the top words of column w.
template <typename T, bool TOP>
__global__ __launch_bounds__(TOP ? 1024 : 256) void logprobs_finish_kernel(
    const T *__restrict__ L, int64_t ldl, int64_t V, int64_t N, const int64_t *__restrict__ tok, const float *__restrict__ part,
    int64_t slices, const float *__restrict__ run_max, float *__restrict__ logp, float *__restrict__ entropy,
    float *__restrict__ stats, int K, int64_t *__restrict__ top_ids, float *__restrict__ top_logp)
{
    constexpr int THREADS = TOP ? 1024 : 256, WAVES = THREADS / 64;
    __shared__ LpSums join[WAVES][16];
    __shared__ float column[2][16]; // largest logit, ln of the sum
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t q0 = (int64_t)blockIdx.x * 16, q = q0 + (tid & 15);
    LpSums a = lp_empty<T>();
    if (q < N)
        for (int64_t i = tid >> 4; i < slices; i += THREADS / 16) {
            const float *p = part + i * 3 * N + q;
            a = lp_join<T>(a, LpSums{p[0], p[N], p[2 * N]});
        }
#pragma unroll
    for (int step = 16; step < 64; step *= 2)
        a = lp_join<T>(a, LpSums{__shfl_xor(a.m, step, 64), __shfl_xor(a.s, step, 64), __shfl_xor(a.t, step, 64)});
    if (lane < 16) join[wave][lane] = a;
    __syncthreads();
    if (tid < 16) {
        a = join[0][tid];
        for (int w = 1; w < WAVES; ++w) a = lp_join<T>(a, join[w][tid]);
        // the sum was taken at the rounded reference r: brought to the maximum itself
        const float c = lp_factor<T>(a.m), r = a.m * c, log_s = __log2f(a.s), log_m = log_s - __builtin_fmaf(a.m, c, -r);
        const float ln_s = LP_LN2 * log_m;
        column[0][tid] = a.m;
        column[1][tid] = ln_s;
        if (q < N) {
            const bool empty = a.s == 0.f; // every logit is -infinity
            stats[q] = empty ? -__builtin_inff() : a.m;
            stats[N + q] = log_m;
            if (entropy) entropy[q] = empty ? 0.f : LP_LN2 * (log_s - a.t / a.s);
            if (logp) {
                const int64_t w = tok[q];
                float v = 0.f;
                if (w >= V) v = __builtin_nanf("");
                else if (w >= 0) v = empty ? -__builtin_inff() : Logit<T>::widen(L[w * ldl + q]) - a.m - ln_s;
                logp[q] = v;
            }
        }
    }
    if constexpr (TOP) {
        __shared__ LpList lists[WAVES];
        __syncthreads();
        const int64_t qw = q0 + wave;
        if (qw >= N) return;
        const int count = lp_top(lists[wave], L, ldl, V, N, qw, run_max, K, lane);
        if (lane < K) {
            top_ids[lane * N + qw] = lane < count ? lists[wave].word[lane] : -1;
            top_logp[lane * N + qw] =
                lane < count ? lists[wave].value[lane] - column[0][wave] - column[1][wave] : -__builtin_inff();
        }
    }
}

// dx_v = gl (1[v = word] - p_v) - gh p_v (log p_v + entropy); a lane owns P columns and 16 rows.
template <typename T, int P>
__global__ __launch_bounds__(LP_THREADS) void logprobs_grad_kernel(const T *__restrict__ L, int64_t ldl, int64_t V, int64_t N,
                                                                   const int64_t *__restrict__ tok, const float *__restrict__ stats,
                                                                   const float *__restrict__ entropy, const float *__restrict__ g_logp,
                                                                   const float *__restrict__ g_entropy, T *__restrict__ DL, int64_t lddl,
                                                                   int tx_count, int ty_count, int64_t row_blocks)
{
    const int tid = threadIdx.x;
    const int ty = tid / tx_count, tx = tid - ty * tx_count;
    const int64_t blk = wide_block();
    const int64_t cb = blk / row_blocks, rb = blk - cb * row_blocks;
    const int64_t q0 = (cb * tx_count + tx) * P, v0 = (rb * ty_count + ty) * LP_BATCH;
    if (ty >= ty_count || q0 >= N || v0 >= V) return;
    float c[P], r[P], log_s[P], gl[P], gh[P], h[P];
    int64_t word[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int64_t q = q0 + p < N ? q0 + p : N - 1;
        const float m = fmaxf(stats[q], Logit<T>::lowest);
        c[p] = lp_factor<T>(m);
        r[p] = m * c[p];
        log_s[p] = stats[N + q] + __builtin_fmaf(m, c[p], -r[p]);
        if (log_s[p] == -__builtin_inff()) log_s[p] = 0.f; // an empty column: every probability is 0
        const int64_t w = g_logp ? tok[q] : -1;
        gl[p] = w < 0 ? 0.f : w >= V ? __builtin_nanf("") : g_logp[q];
        word[p] = w - v0;
        gh[p] = g_entropy ? g_entropy[q] * LP_LN2 : 0.f; // log p below is in base 2
        h[p] = g_entropy ? entropy[q] * LP_LOG2E : 0.f;
    }
    const int left = V - v0 < LP_BATCH ? (int)(V - v0) : LP_BATCH;
    const T *src = L + v0 * ldl + q0;
    T *dst = DL + v0 * lddl + q0;
    Piece<T, P> x[LP_BATCH];
#pragma unroll
    for (int i = 0; i < LP_BATCH; ++i) x[i] = *reinterpret_cast<const Piece<T, P> *>(src + (i < left ? i : left - 1) * ldl);
#pragma unroll
    for (int i = 0; i < LP_BATCH; ++i) {
        Piece<T, P> o;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const float l = __builtin_fmaf(Logit<T>::widen(x[i].v[p]), c[p], -r[p]) - log_s[p], e = lp_exp2(l);
            const float g = e * __builtin_fmaf(gh[p], lp_finite(l) + h[p], gl[p]);
            const float v = (word[p] == i ? gl[p] : 0.f) - g;
            o.v[p] = Logit<T>::narrow(gl[p] == 0.f && gh[p] == 0.f ? 0.f : v); // no gradient comes in: none goes out, whatever the logits
        }
        if (i < left) *reinterpret_cast<Piece<T, P> *>(dst + i * lddl) = o;
    }
}

// Columns per lane and lanes per row.  A piece of P columns is one load: P divides N and the row pitch, the base is aligned to
// it.  Wider pieces need fewer instructions a column, and fewer lanes: they are taken while every SIMD still gets two
// wavefronts of lanes with one run of rows each.
struct LpShape {
    int p, tx, ty;
    int64_t col_blocks;
};
static LpShape lp_shape(int es, int64_t V, int64_t N, int64_t bits, int rows)
{
    LpShape s;
    s.p = 1;
    const int64_t pieces_of_rows = (V + rows - 1) / rows;
    for (int p = 16 / es; p > 1; p /= 2) {
        if (N % p != 0 || (bits & (p * es - 1)) != 0) continue;
        if (p > 2 && pieces_of_rows * (N / p) < 131072) continue;
        s.p = p;
        break;
    }
    const int64_t pieces = N / s.p;
    s.tx = pieces < 64 ? (int)pieces : 64;
    s.ty = LP_THREADS / s.tx;
    s.col_blocks = (pieces + s.tx - 1) / s.tx;
    return s;
}

// rows of the pass kernel's grid; the workspace holds three numbers per slice and column, then the run maxima
struct LpPlan {
    LpShape shape;
    int64_t runs, slices;
    uint64_t part_bytes, bytes;
};
static LpPlan lp_plan(int es, int64_t V, int64_t N, int32_t top, int64_t bits)
{
    LpPlan p;
    p.shape = lp_shape(es, V, N, bits, LP_RUN);
    const int64_t all = (V + LP_RUN - 1) / LP_RUN;
    // runs a lane: as many as leave 2048 workgroups, eight for each compute unit
    int64_t groups = (all + p.shape.ty - 1) / p.shape.ty * p.shape.col_blocks;
    p.runs = groups / 2048 > 1 ? groups / 2048 : 1;
    p.slices = (all + p.runs * p.shape.ty - 1) / (p.runs * p.shape.ty);
    p.part_bytes = (uint64_t)p.slices * 3 * (uint64_t)N * 4;
    p.bytes = p.part_bytes + (top > 0 ? (uint64_t)all * (uint64_t)N * 4 : 0);
    return p;
}
uint64_t logprobs_workspace_bytes(int es, int64_t V, int64_t N, int32_t top)
{
    // whatever the alignment of the call: the pieces decide how many slices there are
    uint64_t most = 0;
    for (int64_t bits = es; bits <= 16; bits *= 2) {
        const uint64_t b = lp_plan(es, V, N, top, bits).bytes;
        most = b > most ? b : most;
    }
    return most;
}

template <typename T>
static int launch_logprobs_t(const T *L, int64_t ldl, int64_t V, int64_t N, const int64_t *tok, float *logp, float *entropy,
                             float *stats, int32_t top, int64_t *top_ids, float *top_logp, void *ws, hipStream_t stream)
{
    const LpPlan p = lp_plan((int)sizeof(T), V, N, top, (int64_t)(uintptr_t)L | ldl * (int64_t)sizeof(T));
    float *part = (float *)ws, *run_max = top > 0 ? (float *)((char *)ws + p.part_bytes) : nullptr;
    const int64_t blocks = p.shape.col_blocks * p.slices, finish = (N + 15) / 16;
    if (blocks > 0x7FFFFFFF || finish > 0x7FFFFFFF / 1024) return LRBI_ERR_SHAPE;
#define LRBI_PASS(P)                                                                                                     \
    LRBI_LAUNCH((logprobs_pass_kernel<T, P>), wide_grid(blocks, LP_THREADS), dim3(LP_THREADS), 0, stream, L, ldl, V, N, p.shape.tx, \
                p.shape.ty, p.runs, p.slices, part, run_max)
    switch (p.shape.p) {
    case 1: LRBI_PASS(1); break;
    case 2: LRBI_PASS(2); break;
    case 4: LRBI_PASS(4); break;
    default:
        if constexpr (sizeof(T) == 2) LRBI_PASS(8);
        break;
    }
#undef LRBI_PASS
    if (top > 0)
        LRBI_LAUNCH((logprobs_finish_kernel<T, true>), dim3((unsigned)finish), dim3(1024), 0, stream, L, ldl, V, N, tok, part, p.slices,
                    run_max, logp, entropy, stats, top, top_ids, top_logp);
    else
        LRBI_LAUNCH((logprobs_finish_kernel<T, false>), dim3((unsigned)finish), dim3(256), 0, stream, L, ldl, V, N, tok, part, p.slices,
                    run_max, logp, entropy, stats, top, top_ids, top_logp);
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
    const LpShape s = lp_shape((int)sizeof(T), V, N, bits, LP_BATCH);
    const int64_t row_blocks = (V + (int64_t)s.ty * LP_BATCH - 1) / ((int64_t)s.ty * LP_BATCH), blocks = s.col_blocks * row_blocks;
    if (blocks > 0x7FFFFFFF) return LRBI_ERR_SHAPE;
#define LRBI_GRAD(P)                                                                                                       \
    LRBI_LAUNCH((logprobs_grad_kernel<T, P>), wide_grid(blocks, LP_THREADS), dim3(LP_THREADS), 0, stream, L, ldl, V, N, tok, stats,  \
                entropy, g_logp, g_entropy, DL, lddl, s.tx, s.ty, row_blocks)
    switch (s.p) {
    case 1: LRBI_GRAD(1); break;
    case 2: LRBI_GRAD(2); break;
    case 4: LRBI_GRAD(4); break;
    default:
        if constexpr (sizeof(T) == 2) LRBI_GRAD(8);
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
