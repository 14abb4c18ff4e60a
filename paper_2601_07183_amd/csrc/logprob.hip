// Log probabilities of a table's rows under a softmax over inner products, and their gradients.
//
// One pass over the logits l = scale <q, t_v>, which are never written: a wave that has a tile's products
// in registers folds them into a running maximum m, s = sum 2^t and e = sum 2^t t with t = (<q, t_v> - m) scale log2(e),
// and leaves one {m, s, e} per query and run of table rows ("part").  From them
//     lse = scale m + ln 2 log2 s,     entropy = ln 2 (log2 s - e / s).
// m is the largest product itself: rounded to a multiple of log2(e) first, which would save an operation a value, it would
// not be given back by lse, and logits past 2^31 would overflow against it.
// For the most probable rows it also leaves the largest products of every 16 (or 64) rows ("group"): a row
// among the K best lies in a group whose maximum is at least the K-th best maximum less what the sums can
// be off by.  Groups of 16 also say which row the maximum is, in the value's last four bits, and what the
// second largest product is, so that little more than K rows are scored again in float64, which orders
// rows whose fp32 products are too close to tell apart.
#include <algorithm>

#include "fewrows.h"
#include "query_ops.h"

#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f
#define NEG_INF (-__builtin_huge_valf())
// The product of a row that the mask hides: the lowest value whose last four bits are zero, so that a row written into them
// makes it smaller.  Live products are above -3.4e38 (the caller's), 2.8e34 away: times a scale of 1e-30 still a logit that is out of reach.
#define HIDDEN (-0x1.ffffep+127f)

// ---- statistics of a tile ----------------------------------------------------------------------------

struct StatsArgs {
    int n, V;
    float c;                        // scale log2(e)
    const uint32_t *live;
    int64_t ld_live;
    const int64_t *targets;
    float4 *parts;                  // [n][nparts] {m, s, e, 0}; m: the largest product itself, not times c
    int nparts;
    // Groups of block b (rows 64 b .. 64 b + 63): [b][n][4] the largest of rows 64 b + 16 i + 4 h + r for h = 0..3 (a wave's
    // store is one run of memory) and, apart, the second largest; or, wide, [n][b] the largest of all (a sixteenth of that;
    // a query's are read in one run)
    float *gmax, *gsecond;
    int nblocks;
    int wide, wstride;              // (a query's run is filled up to a multiple of four values)
    float *zt;                      // [n] the target's product
};

// 2^x for x <= 0 (a result below 2^-126 may be flushed)
static __device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The larger value, a NaN if there is one.  (The instruction for it takes values as they come out of the
// matrix cores; fmaxf's has each quieted by an instruction of its own first.)
static __device__ __forceinline__ float max_of(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// The largest of the four lanes that hold the same query (lane & 15), in each of them: registers' halves are swapped
// between copies of a value, so that each step is one maximum (written as instructions, with the idle slots
// that the compiler puts around its own; four trips through the LDS crossbar per query took a fifth of the
// epilogue's time).
static __device__ __forceinline__ float max_of_four(float x)
{
    float y = x;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(x), "+v"(y));
    x = max_of(x, y);
    y = x;
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(x), "+v"(y));
    return max_of(x, y);
}

// sums relative to a maximum m0, brought to m1 >= m0
static __device__ __forceinline__ void rebase(float &s, float &e, float m0, float m1, float c)
{
    if (m0 == m1) return;
    if (m0 == HIDDEN) { s = 0.0f; e = 0.0f; return; }
    const float d = (m0 - m1) * c, f = exp2_fast(d);
    e = f * fmaf(s, fmaxf(d, -1e4f), e);
    s *= f;
}

// ENT: e is wanted too.  TOP: the groups' maxima are, 1 wide, 2 with their rows (0: none).
template <int QT, bool ENT, int TOP>
struct StatsState {
    float m[QT], s[QT], e[QT];
    int32_t target[QT];             // the query's target, -1: none (V is below 2^31)
    __device__ __forceinline__ void begin(const StatsArgs &a, int q0, int lane)
    {
#pragma unroll
        for (int j = 0; j < QT; j++) {
            m[j] = HIDDEN; s[j] = 0.0f; e[j] = 0.0f;
            const int q = q0 + 16 * j + (lane & 15);
            const int64_t t = q < a.n ? a.targets[q] : -1;
            target[j] = t >= 0 && t < a.V ? (int32_t)t : -1;
        }
    }
    // a tile's products: rows p0 + 16 i + 4 (lane >> 4) + r, queries q0 + 16 j + (lane & 15); acc is
    // overwritten (HIDDEN where the mask hides a row)
    template <int PT>
    __device__ __forceinline__ void tile(const StatsArgs &a, v4f (&acc)[PT][QT], int p0, int q0, int lane)
    {
        const int h = lane >> 4;
        const bool ragged = p0 + 16 * PT > a.V;                       // uniform
#pragma unroll
        for (int j = 0; j < QT; j++) {
            const int q = q0 + 16 * j + (lane & 15);
            const bool in = q < a.n;
            // the target's product, by the lane that has it
            const uint32_t dp = (uint32_t)(target[j] - p0);           // (no target: far out)
            if (__any(dp < 16 * PT && target[j] >= 0)) {              // (seldom)
                uint32_t at = dp - 4 * h;                             // 16 i + r in that lane
                asm volatile("" : "+v"(at));                          // (the comparisons stay in here)
                if (target[j] >= 0 && dp < 16 * PT && ((dp >> 2) & 3) == (uint32_t)h) {
#pragma unroll
                    for (int i = 0; i < PT; i++)
#pragma unroll
                        for (int r = 0; r < 4; r++)
                            if (at == (uint32_t)(16 * i + r)) a.zt[q] = acc[i][j][r];
                }
            }
            if (a.live || ragged) {
                const uint32_t *live = a.live ? a.live + (in ? q : 0) * a.ld_live : nullptr;
#pragma unroll
                for (int i = 0; i < PT; i++) {
                    const int p = p0 + 16 * i;                        // (a multiple of 16: within one word of the mask)
                    uint32_t bits = 0;
                    if (p < a.V) {
                        bits = live ? live[p >> 5] >> ((p & 31) + 4 * h) : 0xFu;
                        const int left = a.V - p - 4 * h;
                        bits &= left >= 4 ? 0xFu : left <= 0 ? 0u : (1u << left) - 1u;
                    }
#pragma unroll
                    for (int r = 0; r < 4; r++)
                        if (!((bits >> r) & 1u)) acc[i][j][r] = HIDDEN;
                }
            }
            float top = HIDDEN;
#pragma unroll
            for (int b = 0; b < PT; b += 4) {
                const int blk = p0 / 64 + b / 4;                      // uniform
                float g = HIDDEN, g2 = HIDDEN;
                if constexpr (TOP == 2) {
#pragma unroll
                    for (int i = b; i < b + 4; i++)
#pragma unroll
                        for (int r = 0; r < 4; r++) {
                            const float x = __uint_as_float((__float_as_uint(acc[i][j][r]) & ~15u) | (uint32_t)(4 * (i - b) + r));
                            g2 = __builtin_amdgcn_fmed3f(g, g2, x);
                            g = max_of(g, x);
                        }
                    if (blk < a.nblocks) {
                        const int64_t at = ((int64_t)blk * a.n + q0 + 16 * j) * 4;    // uniform
                        if (in) {
                            (a.gmax + at)[4 * (lane & 15) + h] = g;
                            (a.gsecond + at)[4 * (lane & 15) + h] = g2;
                        }
                    }
                } else {
#pragma unroll
                    for (int i = b; i < b + 4; i++)
                        g = max_of(max_of(max_of(g, acc[i][j][0]), acc[i][j][1]), max_of(acc[i][j][2], acc[i][j][3]));
                    if constexpr (TOP == 1) {
                        const float w = max_of_four(g);
                        if (in && h == 0 && blk < a.nblocks) a.gmax[(int64_t)q * a.wstride + blk] = w;
                    }
                }
                top = max_of(top, g);
            }
            // (the row in a maximum's last bits makes it up to 2^-19 of itself smaller or larger)
            if (__any(!((TOP == 2 ? fmaf(fabsf(top), 0x1p-19f, top) : top) <= m[j]))) {      // (ever more seldom)
                if constexpr (TOP == 2) {
                    top = HIDDEN;
#pragma unroll
                    for (int i = 0; i < PT; i++) top = max_of(max_of(max_of(top, acc[i][j][0]), acc[i][j][1]), max_of(acc[i][j][2], acc[i][j][3]));
                }
                const float m1 = max_of(m[j], top);
                rebase(s[j], e[j], m[j], m1, a.c);
                m[j] = m1;
            }
            const float from = m[j] == HIDDEN ? 0.0f : m[j];
            float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
            for (int i = 0; i < PT; i++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const float t = (acc[i][j][r] - from) * a.c, x = exp2_fast(t);
                    if (r & 1) s1 += x;
                    else s0 += x;
                    if constexpr (ENT) e[j] = fmaf(x, fmaxf(t, -1e4f), e[j]);
                }
            s[j] += s0 + s1;
            __builtin_amdgcn_sched_barrier(0);                        // (one query's values at a time in registers)
        }
    }
    __device__ __forceinline__ void end(const StatsArgs &a, int part, int q0, int lane)
    {
#pragma unroll
        for (int j = 0; j < QT; j++) {
            float top = fmaxf(m[j], __shfl_xor(m[j], 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            rebase(s[j], e[j], m[j], top, a.c);
            float ss = s[j] + __shfl_xor(s[j], 16), ee = e[j] + __shfl_xor(e[j], 16);
            ss += __shfl_xor(ss, 32);
            ee += __shfl_xor(ee, 32);
            const int q = q0 + 16 * j + (lane & 15);
            if (q < a.n && lane < 16) a.parts[(int64_t)q * a.nparts + part] = make_float4(top, ss, ee, 0.0f);
        }
    }
};

// NORM: the largest squared norm of the rows is wanted as well (a wave has all of the queries then)
template <bool ENT, int TOP, bool NORM = false>
struct StatsEpi {
    StatsArgs a;
    const uint32_t *any_live;
    float *xmax;                    // [parts]
    template <class T>
    struct State {
        StatsState<T::QT, ENT, TOP> s;
        float most;
    };
    template <class T>
    __device__ __forceinline__ void begin(State<T> &st, int64_t q0, int lane) const
    {
        st.s.begin(a, (int)q0, lane);
        st.most = 0.0f;
    }
    template <class T>
    __device__ __forceinline__ void tile(State<T> &st, RowAcc<T> &acc, int64_t p0, int64_t q0, int lane, int) const
    {
        st.s.tile(a, acc.v, (int)p0, (int)q0, lane);
        if constexpr (NORM) {
#pragma unroll
            for (int i = 0; i < T::PT; i++) {
                float x = acc.nrm[i] + __shfl_xor(acc.nrm[i], 16);
                x += __shfl_xor(x, 32);
                const int p = (int)p0 + 16 * i + (lane & 15);
                if (p < a.V && (!any_live || ((any_live[p >> 5] >> (p & 31)) & 1u))) st.most = fmaxf(st.most, x);
            }
        }
    }
    template <class T>
    __device__ __forceinline__ void end(State<T> &st, int run, int wp, int64_t q0, int lane) const
    {
        st.s.end(a, run * T::WP + wp, (int)q0, lane);
        if constexpr (NORM) {
            float x = fmaxf(st.most, lane_xor8(st.most));
            x = fmaxf(x, lane_xor4(x));
            x = fmaxf(x, lane_xor2(x));
            x = fmaxf(x, lane_xor1(x));
            if (lane == 0) xmax[run * T::WP + wp] = x;
        }
    }
};

// Largest squared norm of the live rows, one value per workgroup (what the margin of the selection needs).
template <class S>
__global__ __launch_bounds__(WG) void table_norm_kernel(const S *__restrict__ t, int64_t ld, int64_t V, int d, const uint32_t *__restrict__ live,
                                                        int vec, float *__restrict__ out)
{
    __shared__ float best[WG / 64];
    constexpr int CH = FewLoad<S>::CH;
    const int lane = threadIdx.x & 63, sub = lane & 15;
    float most = 0.0f;
    // four rows per wave, 16 lanes each
    for (int64_t v0 = ((int64_t)blockIdx.x * (WG / 64) + (threadIdx.x >> 6)) * 4; v0 < V; v0 += (int64_t)gridDim.x * WG / 16) {
        const int64_t v = v0 + (lane >> 4);
        float x = 0.0f;
        if (v < V && (!live || ((live[v >> 5] >> (v & 31)) & 1u)))
            for (int k = sub * CH; k < d; k += 16 * CH) {
                const FewFrag<S, CH> f = vec ? few_load<S, CH, true>(t + v * ld, k, d) : few_load<S, CH, false>(t + v * ld, k, d);
#pragma unroll
                for (int e = 0; e < CH; e++) x = fmaf((float)f.e[e], (float)f.e[e], x);
            }
        x += lane_xor8(x);
        x += lane_xor4(x);
        x += lane_xor2(x);
        x += lane_xor1(x);
        most = fmaxf(most, x);
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    if (lane == 0) best[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x == 0) out[blockIdx.x] = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
}

// words of the masks of all queries, or-ed: rows that any query sees
__global__ __launch_bounds__(WG) void any_live_kernel(const uint32_t *__restrict__ live, int64_t ld, int64_t n, int64_t words,
                                                      uint32_t *__restrict__ out)
{
    const int64_t w = (int64_t)blockIdx.x * WG + threadIdx.x;
    if (w >= words) return;
    uint32_t x = 0;
    for (int64_t i = 0; i < n; i++) x |= live[i * ld + w];
    out[w] = x;
}

// ---- a few queries: the table's rows straight from memory -------------------------------------------

struct FewStatsArgs {
    StatsArgs st;
    const void *table, *q;
    int64_t ldt, ldq;
    int d, rounds;                  // rounds of 64 rows per wave: a part
    const uint32_t *any_live;
    float *xmax;                    // [nparts] largest squared norm of a part's rows, or null
};

template <class S, class Q, int QT, bool VEC, bool NORM>
__global__ __launch_bounds__(WG, QT == 1 ? 4 : QT == 2 ? 3 : 2) void few_stats_kernel(FewStatsArgs a)
{
    const int lane = threadIdx.x & 63;
    const int part = blockIdx.x * (WG / 64) + (threadIdx.x >> 6);
    if (part >= a.st.nparts) return;
    const Q *qrow[QT];
#pragma unroll
    for (int j = 0; j < QT; j++) {
        const int q = min(16 * j + (lane & 15), a.st.n - 1);
        qrow[j] = (const Q *)a.q + q * a.ldq;
    }
    const int steps = (a.d + 4 * FewLoad<S>::CH - 1) / (4 * FewLoad<S>::CH);
    StatsState<QT, true, NORM ? 2 : 0> st;
    st.begin(a.st, 0, lane);
    float most = 0.0f;
    for (int r = 0; r < a.rounds; r++) {
        const int p0 = (part * a.rounds + r) * 64;
        if (p0 >= a.st.V) break;
        // 32 rows at a time: twice the waves on a SIMD, so that some load while others multiply
        v4f acc[4][QT];
#pragma unroll
        for (int half = 0; half < 2; half++) {
            const S *prow[2];
            v4f part[2][QT];
            float nrm[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                prow[i] = (const S *)a.table + (int64_t)min(p0 + 32 * half + 16 * i + (lane & 15), a.st.V - 1) * a.ldt;
                nrm[i] = 0.0f;
#pragma unroll
                for (int j = 0; j < QT; j++) part[i][j] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
            }
            few_dot<S, Q, 2, QT, VEC, NORM>(prow, qrow, 0, steps, a.d, lane, part, nrm);
#pragma unroll
            for (int i = 0; i < 2; i++) {
#pragma unroll
                for (int j = 0; j < QT; j++) acc[2 * half + i][j] = part[i][j];
                if constexpr (NORM) {
                    float x = nrm[i] + __shfl_xor(nrm[i], 16);
                    x += __shfl_xor(x, 32);
                    const int p = p0 + 32 * half + 16 * i + (lane & 15);
                    if (p < a.st.V && (!a.any_live || ((a.any_live[p >> 5] >> (p & 31)) & 1u))) most = fmaxf(most, x);
                }
            }
        }
        st.tile(a.st, acc, p0, 0, lane);
    }
    st.end(a.st, part, 0, lane);
    if constexpr (NORM) {
        most = fmaxf(most, lane_xor8(most));
        most = fmaxf(most, lane_xor4(most));
        most = fmaxf(most, lane_xor2(most));
        most = fmaxf(most, lane_xor1(most));
        if (lane == 0) a.xmax[part] = most;
    }
}

// ---- joining the parts, and the most probable rows --------------------------------------------------

struct FinishArgs {
    StatsArgs st;
    const void *table, *q;
    int64_t ldt, ldq;
    int d, vec;
    int dot_lanes;                  // lanes that share a row's float64 product
    float scale;
    float slack;                    // relative error of a product against |q||t|
    const float *xmax;
    int nxmax;
    float *logp, *lse, *entropy;
    int top;
    int64_t *top_ids;
    float *top_logp;
};

// A query is finished by a team of threads: a wave of its own in a large batch, a workgroup of 16 waves if
// there are few queries and one has to be done soon.  Lists in LDS are per team.  (One query, 1M rows, top 10: 21 us, a
// chain of some ten steps that wait for one another; 4,096 queries, 128,000 x 1024 bf16, top 20: 160 us, of them 20 the
// groups' 131 MB and about as much the rows scored again.)
template <int NT>
struct FinishShared {
    static constexpr int LIST = NT == 64 ? 384 : 1024;    // rows (wide: groups) that reach the bound
    static constexpr int ITEMS = NT == 64 ? 256 : 1024;   // rows to score at a time
    double val[ITEMS + RAIRS_MAX_TOP];
    double best[RAIRS_MAX_TOP];
    double lse;
    uint32_t id[ITEMS + RAIRS_MAX_TOP];
    uint32_t best_id[RAIRS_MAX_TOP];
    uint32_t take[ITEMS];
    float lval[LIST];
    uint32_t lid[LIST];
    float kth_in[256];
    float red[16], red5[NT > 64 ? 16 : 1][5];
    float kth_out;
    int count, nbest, wcnt[16];
};

template <int NT>
static __device__ __forceinline__ void team_sync()
{
    if constexpr (NT == 64) wave_lds_sync();
    else __syncthreads();
}

// f over the team's values, in every thread
template <int NT, class F>
static __device__ __forceinline__ float team_fold(FinishShared<NT> &sh, float x, const F &f)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) x = f(x, __shfl_xor(x, o));
    if constexpr (NT > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sh.red[threadIdx.x >> 6] = x;
        __syncthreads();
        x = sh.red[0];
        for (int w = 1; w < NT / 64; w++) x = f(x, sh.red[w]);
    }
    return x;
}

// sums of s, e and q2, the largest x2, the least zero
template <int NT>
static __device__ __forceinline__ void team_fold5(FinishShared<NT> &sh, float &s, float &e, float &q2, float &x2, float &zero)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        s += __shfl_xor(s, o);
        e += __shfl_xor(e, o);
        q2 += __shfl_xor(q2, o);
        x2 = fmaxf(x2, __shfl_xor(x2, o));
        zero = fminf(zero, __shfl_xor(zero, o));
    }
    if constexpr (NT > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            float *to = sh.red5[threadIdx.x >> 6];
            to[0] = s; to[1] = e; to[2] = q2; to[3] = x2; to[4] = zero;
        }
        __syncthreads();
        s = sh.red5[0][0]; e = sh.red5[0][1]; q2 = sh.red5[0][2]; x2 = sh.red5[0][3]; zero = sh.red5[0][4];
        for (int w = 1; w < NT / 64; w++) {
            s += sh.red5[w][0];
            e += sh.red5[w][1];
            q2 += sh.red5[w][2];
            x2 = fmaxf(x2, sh.red5[w][3]);
            zero = fminf(zero, sh.red5[w][4]);
        }
    }
}

// rows of an entry of the lists: the row itself, a group of 16 or one of 64
enum { ENTRY_ROW = 1, ENTRY_GROUP = 16, ENTRY_WIDE = 64 };
static __device__ __forceinline__ int64_t entry_row(uint32_t entry, int member, int kind)
{
    return kind == ENTRY_ROW    ? (int64_t)entry
           : kind == ENTRY_WIDE ? (int64_t)entry * 64 + member
                                : (int64_t)(entry >> 2) * 64 + 16 * (member >> 2) + 4 * (entry & 3) + (member & 3);
}

// A lower bound of the k-th largest (k <= 64) of the values of which most[0..3] are a thread's maxima of four
// sets: the k-th largest of the maxima of 256 sets, found bit by bit.
template <int NT>
static __device__ __forceinline__ float kth_set_max(FinishShared<NT> &sh, const float (&most)[4], int k, int tid)
{
    float set[4] = {most[0], most[1], most[2], most[3]};
    if constexpr (NT > 64) {                                          // NT / 256 threads' values to a set, for the first wave
        float mine = fmaxf(fmaxf(set[0], set[1]), fmaxf(set[2], set[3]));
#pragma unroll
        for (int x = 1; x < NT / 256; x <<= 1) mine = fmaxf(mine, __shfl_xor(mine, x));
        __syncthreads();
        if (tid % (NT / 256) == 0) sh.kth_in[tid / (NT / 256)] = mine;
        __syncthreads();
        if (tid < 64)
#pragma unroll
            for (int u = 0; u < 4; u++) set[u] = sh.kth_in[tid + 64 * u];
    }
    if (NT == 64 || tid < 64) {
        uint32_t key[4], cut = 0;
#pragma unroll
        for (int u = 0; u < 4; u++) key[u] = f32_key(set[u]);
        for (int bit = 31; bit >= 0; bit--) {
            const uint32_t cand = cut | (1u << bit);
            int n = 0;
#pragma unroll
            for (int u = 0; u < 4; u++) n += __popcll(__ballot(key[u] >= cand));
            if (n >= k) cut = cand;
        }
        if (tid == 0) sh.kth_out = key_f32(cut);
    }
    team_sync<NT>();
    return sh.kth_out;
}

template <class S>
struct DotLoad {                    // values per lane and step (eight bytes: sixteen and their float64 values are too many registers)
    static constexpr int CH = sizeof(S) == 1 ? 8 : 16 / sizeof(S);
};

// <q, t> in float64 for U rows at once by `lanes` lanes (1 to 64), whose own place is `sub`; the order of a
// sum depends on d alone, so equal rows get equal values
template <class S, class Q, bool VEC, int U>
static __device__ __forceinline__ void dot_exact(const S *const (&t)[U], const Q *q, int d, int sub, int lanes, double (&x)[U])
{
    constexpr int CH = DotLoad<S>::CH;
#pragma unroll
    for (int u = 0; u < U; u++) x[u] = 0.0;
#pragma unroll 1
    for (int k = sub * CH; k < d; k += lanes * CH) {
        FewFrag<S, CH> f[U];
#pragma unroll
        for (int u = 0; u < U; u++) f[u] = few_load<S, CH, VEC>(t[u], k, d);
        const FewFrag<Q, CH> g = few_load<Q, CH, VEC>(q, k, d);
#pragma unroll
        for (int e = 0; e < CH; e++) {
            const double y = (double)(float)g.e[e];
#pragma unroll
            for (int u = 0; u < U; u++) x[u] = fma((double)(float)f[u].e[e], y, x[u]);
        }
    }
    for (int s = lanes >> 1; s > 0; s >>= 1)
#pragma unroll
        for (int u = 0; u < U; u++) x[u] += __shfl_xor(x[u], s);
}

// scores the rows of the `cnt` entries in sh.take and merges those of at least `floor` into sh.best
template <class S, class Q, int NT>
static __device__ __forceinline__ void finish_batch(const FinishArgs &a, FinishShared<NT> &sh, int64_t row, int tid, int cnt, int kind,
                                                    double floor)
{
    const int lane = tid & 63, wave = tid >> 6, lanes = a.dot_lanes, sub = lane & (lanes - 1), at = lane / lanes, rows = 64 / lanes;
    const Q *q = (const Q *)a.q + row * a.ldq;
    const int old = sh.nbest;
    if (tid < old) {
        sh.val[tid] = sh.best[tid];
        sh.id[tid] = sh.best_id[tid];
    }
    if (tid == 0) sh.count = old;
    team_sync<NT>();
    const int items = cnt * kind;
    constexpr int U = sizeof(S) == 1 && NT == 64 ? 8 : 4;             // (a workgroup of 16 waves has half a wave's registers each)
#pragma unroll 1
    for (int i0 = wave * U * rows; i0 < items; i0 += NT / 64 * U * rows) {    // U times 64 / lanes rows per wave
        const S *t[U];
        int64_t v[U];
        double x[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int i = i0 + u * rows + at, ic = i < items ? i : items - 1;
            v[u] = entry_row(sh.take[ic / kind], ic % kind, kind);
            const bool in = i < items && v[u] < a.st.V && (!a.st.live || ((a.st.live[row * a.st.ld_live + (v[u] >> 5)] >> (v[u] & 31)) & 1u));
            v[u] = in ? v[u] : -1;
            t[u] = (const S *)a.table + (in ? v[u] : 0) * a.ldt;
        }
        if (a.vec) dot_exact<S, Q, true>(t, q, a.d, sub, lanes, x);
        else dot_exact<S, Q, false>(t, q, a.d, sub, lanes, x);
#pragma unroll
        for (int u = 0; u < U; u++)
            if (sub == 0 && v[u] >= 0 && x[u] >= floor) {             // (not a NaN either)
                const int slot = atomicAdd(&sh.count, 1);
                sh.val[slot] = x[u];
                sh.id[slot] = (uint32_t)v[u];
            }
    }
    team_sync<NT>();
    const int total = sh.count;
#pragma unroll 1
    for (int i = tid; i < total; i += NT) {
        const double x = sh.val[i];
        const uint32_t id = sh.id[i];
        int rank = 0;
        for (int j = 0; j < total; j++) rank += sh.val[j] > x || (sh.val[j] == x && sh.id[j] < id) ? 1 : 0;
        if (rank < a.top) {
            sh.best[rank] = x;
            sh.best_id[rank] = id;
        }
    }
    if (tid == 0) sh.nbest = total < a.top ? total : a.top;
    team_sync<NT>();
}

// the entries with want set, ITEMS rows at a time, until none is left (drop() is asked again before each time)
template <class S, class Q, int NT, class Drop>
static __device__ __forceinline__ void finish_entries(const FinishArgs &a, FinishShared<NT> &sh, int64_t row, int tid, bool want,
                                                      uint32_t entry, int kind, double floor, const Drop &drop)
{
    const int lane = tid & 63, wave = tid >> 6, most = FinishShared<NT>::ITEMS / kind;
    for (;;) {
        if (want && drop()) want = false;
        const unsigned long long b = __ballot(want);
        int at = __popcll(b & ((1ull << lane) - 1ull)), total = __popcll(b);
        if constexpr (NT > 64) {
            if (lane == 0) sh.wcnt[wave] = total;
            __syncthreads();
            total = 0;
            for (int w = 0; w < NT / 64; w++) {
                at += w < wave ? sh.wcnt[w] : 0;
                total += sh.wcnt[w];
            }
        }
        if (want && at < most) {
            sh.take[at] = entry;
            want = false;
        }
        team_sync<NT>();
        if (total == 0) return;                                       // (the same in every thread)
        finish_batch<S, Q, NT>(a, sh, row, tid, total < most ? total : most, kind, floor);
    }
}

// NT threads per query, `TEAMS` queries per workgroup
template <class S, class Q, int NT, int TEAMS>
__global__ __launch_bounds__(NT * TEAMS, NT == 64 ? 3 : 4) void logprob_finish_kernel(FinishArgs a)
{
    __shared__ FinishShared<NT> shared[TEAMS];
    FinishShared<NT> &sh = shared[threadIdx.x / NT];
    const int tid = threadIdx.x % NT;
    const int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / NT;
    if (row >= a.st.n) return;                                        // (teams of a workgroup do not wait for each other)
    const float4 *parts = a.st.parts + row * a.st.nparts;
    const float c = a.st.c;
    float m = HIDDEN, s = 0.0f, e = 0.0f;
    for (int i = tid; i < a.st.nparts; i += NT) {
        float4 p = parts[i];
        const float m1 = max_of(m, p.x);
        rebase(s, e, m, m1, c);
        rebase(p.y, p.z, p.x, m1, c);
        s += p.y;
        e += p.z;
        m = m1;
    }
    // |q|^2 and the table's largest squared norm, for the margin
    float q2 = 0.0f, x2 = 0.0f, zero = 1.0f;
    const Q *q = (const Q *)a.q + row * a.ldq;
    if (a.top) {
        for (int k = tid; k < a.d; k += NT) {
            const float x = (float)q[k];
            q2 = fmaf(x, x, q2);
            zero = x == 0.0f ? zero : 0.0f;
        }
#pragma unroll 8
        for (int i = tid; i < a.nxmax; i += NT) x2 = fmaxf(x2, a.xmax[i]);
    }
    const float top = team_fold(sh, m, [](float x, float y) { return max_of(x, y); });
    rebase(s, e, m, top, c);
    team_fold5<NT>(sh, s, e, q2, x2, zero);
    const bool empty = top == HIDDEN;
    const float logs = log2f(s);
    if (tid == 0) {
        const double ln_sum = (double)logs * 0.6931471805599453;
        sh.lse = (double)top * (double)a.scale + ln_sum;
        a.lse[row] = empty ? NEG_INF : (float)sh.lse;
        if (a.entropy) a.entropy[row] = empty ? 0.0f : fmaxf((logs - e / s) * LN2, 0.0f);
        const int64_t t = a.st.targets[row];
        float lp = 0.0f;
        if (t >= 0 && t < a.st.V) {
            const bool seen = !a.st.live || ((a.st.live[row * a.st.ld_live + (t >> 5)] >> (t & 31)) & 1u);
            lp = seen ? (float)(((double)a.st.zt[row] - (double)top) * (double)a.scale - ln_sum) : NEG_INF;
        }
        a.logp[row] = lp;
        sh.nbest = 0;
        sh.count = 0;
    }
    if (a.top == 0) return;

    // what a product may be off by (components whose squares underflow, and a group's row in the last bits of a
    // denormal, have terms of their own); not finite: nothing can be told apart
    const float under = sqrtf((float)a.d) * 1.1e-19f;
    const float eps = a.slack * (sqrtf(q2) + under) * (sqrtf(x2) + under) * 1.0001f + 4e-44f;
    const bool zeros = zero != 0.0f;                                  // a query of zeros: every product is 0

    // entry i of the query's groups: block i >> shift, its part i & 3 if it has four
    const int shift = a.st.wide ? 0 : 2, ngroups = a.st.nblocks << shift;
    const auto group_at = [&](int i) { return a.st.wide ? (int64_t)i : (((int64_t)(i >> 2) * a.st.n + row) << 2) + (i & 3); };
    const float *gmax = a.st.wide ? a.st.gmax + row * a.st.wstride : a.st.gmax;
    // A thread's groups are four sets; of each it keeps the largest value, where that is, and the second largest.
    // (loads first, then straight-line code: a load whose use is behind a branch is moved there, and loads then wait
    // for one another)
    float most[4] = {HIDDEN, HIDDEN, HIDDEN, HIDDEN}, second[4] = {HIDDEN, HIDDEN, HIDDEN, HIDDEN};
    int where[4] = {0, 0, 0, 0};
    const auto keep = [&](int set, float x, int i) {
        second[set] = __builtin_amdgcn_fmed3f(most[set], second[set], x);
        where[set] = x > most[set] ? i : where[set];
        most[set] = fmaxf(most[set], x);
    };
    // place k of set u of this thread: four sets are 16 bytes
    const auto group_of = [&](int u, int k) { return 4 * (tid + k * NT) + u; };
    const int fours = (ngroups + 3) / 4;
    for (int k = 0; tid + k * NT < fours; k += 8) {
        v4f x[8];
#pragma unroll
        for (int u = 0; u < 8; u++) x[u] = *(const v4f *)(gmax + group_at(4 * min(tid + (k + u) * NT, fours - 1)));
#pragma unroll
        for (int u = 0; u < 8; u++)
#pragma unroll
            for (int e = 0; e < 4; e++) keep(e, group_of(e, k + u) < ngroups ? x[u][e] : HIDDEN, group_of(e, k + u));
    }
    if (!empty && eps < 1e38f) {                                      // (the same in every thread)
        const float thr = kth_set_max<NT>(sh, most, a.top, tid) - 2.0f * eps;
        // exact products of the K best are at least this
        const double floor = (double)thr + (double)eps * 0.999;
        const auto note = [&](int i) {
            const int at = atomicAdd(&sh.count, 1);
            if (at < FinishShared<NT>::ITEMS) sh.id[at] = (uint32_t)i;
        };
#pragma unroll
        for (int u = 0; u < 4; u++) {
            if (!(most[u] >= thr && most[u] > HIDDEN)) continue;
            note(where[u]);
            if (!(second[u] >= thr && second[u] > HIDDEN)) continue;
            // (seldom: two of a set)
            for (int k = 0; group_of(u, k) < ngroups; k += 8) {
                float x[8];
#pragma unroll
                for (int w = 0; w < 8; w++) x[w] = gmax[group_at(min(group_of(u, k + w), ngroups - 1))];
                uint32_t hits = 0;
#pragma unroll
                for (int w = 0; w < 8; w++) {
                    const int i = group_of(u, k + w);
                    hits |= i < ngroups && i != where[u] && x[w] >= thr && x[w] > HIDDEN ? 1u << w : 0u;
                }
                for (; hits; hits &= hits - 1) note(group_of(u, k + __ffs(hits) - 1));
            }
        }
        team_sync<NT>();
        const int groups = sh.count;
        team_sync<NT>();
        if (tid == 0) sh.count = groups <= FinishShared<NT>::ITEMS ? 0 : FinishShared<NT>::LIST + 1;
        team_sync<NT>();
        if (groups <= FinishShared<NT>::ITEMS)
            for (int u0 = tid; u0 < groups; u0 += NT) {
                const int i = (int)sh.id[u0];
                const int64_t g = group_at(i);
                const float x = gmax[g];
                // the group's best row alone, or all of its rows if another may reach the bound too; wide: the group
                const int rows = !a.st.wide && a.st.gsecond[g] >= thr ? 16 : 1, at = atomicAdd(&sh.count, rows);
                for (int u = 0; u < rows && at + u < FinishShared<NT>::LIST; u++) {
                    sh.lval[at + u] = x;
                    sh.lid[at + u] = a.st.wide ? (uint32_t)i
                                               : (uint32_t)entry_row((uint32_t)i, rows == 1 ? (int)(__float_as_uint(x) & 15u) : u, ENTRY_GROUP);
                }
            }
        team_sync<NT>();
        const int found = sh.count;
        team_sync<NT>();
        if (found <= FinishShared<NT>::LIST) {
            for (int i0 = 0; i0 < found; i0 += NT) {
                const int i = i0 + tid;
                const float x = i < found ? sh.lval[i] : HIDDEN;
                // (an entry that cannot reach the K-th best so far is left out)
                finish_entries<S, Q, NT>(a, sh, row, tid, i < found, i < found ? sh.lid[i] : 0u, a.st.wide ? ENTRY_WIDE : ENTRY_ROW, floor, [&]() {
                    return sh.nbest == a.top && (double)x + (double)eps < sh.best[a.top - 1];
                });
            }
        } else {
            // so many equal products that the list does not hold them: all groups in order of their blocks of 64
            // rows, so that a block whose rows can only equal the K-th best comes too late to displace it
            for (int i0 = 0; i0 < ngroups; i0 += NT) {
                const int i = i0 + tid;
                const float x = i < ngroups ? gmax[group_at(i)] : HIDDEN;
                finish_entries<S, Q, NT>(a, sh, row, tid, x >= thr && x > HIDDEN, (uint32_t)i, a.st.wide ? ENTRY_WIDE : ENTRY_GROUP, floor, [&]() {
                    if (sh.nbest < a.top) return false;
                    const double k = sh.best[a.top - 1], up = zeros ? 0.0 : (double)x + (double)eps;
                    return up < k || (up == k && (int)(sh.best_id[a.top - 1] >> 6) < i >> shift);
                });
            }
        }
    }
    team_sync<NT>();
    if (tid < a.top) {
        const bool have = tid < sh.nbest;
        a.top_ids[row * a.top + tid] = have ? (int64_t)sh.best_id[tid] : -1;
        a.top_logp[row * a.top + tid] =
            have ? (float)(sh.best[tid] * (double)a.scale - sh.lse) : NEG_INF;
    }
}

// ---- gradient of the logits --------------------------------------------------------------------------

struct GradArgs {
    int n, V, v0;                   // the product's columns are rows v0 .. V - 1 of the table
    int vc, npad;                   // columns of g, of gt
    float scale;
    const uint32_t *live;
    int64_t ld_live;
    const int64_t *targets;
    const float *lse, *entropy, *dlogp, *dentropy;
    __bf16 *g, *gt;                 // [n][vc], [vc][npad]; either null
    PackLayout gto, gtto;
    const float2 *rows;             // fp32 (NP 3): row_stats_kernel's
};

// G = scale (dlogp (1[v = t] - p) - dentropy p (log p + H)) in registers, in NP bf16 pieces: two for bf16 rows (16 bits: at
// most 2^-16 of a value, so that a gradient is off by its own rounding and little else; one piece would be half the work of
// both products, 1.8 ms instead of 2.9 for 4,095 x 65,537 x 1024, and 2.3e-3 off instead of 1.7e-3) or three (fp32), written for the
// products with the table (rows of queries) and with the queries (rows of the table).  Both sum over what
// they have in common with the operand beside them, so their columns lie in the order that a wave holds
// them in (ORDER_TABLE, ORDER_QUERIES): a lane's values are 32 or 8 bytes in a row, the lanes of a row 128.
// (4,095 x 65,537 x 1024 bf16: 960 us, of which the product alone would take 400 and 2.1 GB of G are written, 4.4 TB/s beside it;
// with the pieces in planes of their own 957, but the products that read them 1,088 each instead of 1,038.)
template <int NP, bool ENT>
struct GradEpi {
    GradArgs a;
    template <class T>
    struct State {
        float da[T::QT], db[T::QT], H[T::QT], lse[T::QT], m[NP == 3 ? T::QT : 1];
        int32_t target[T::QT];      // from the chunk's first row on, or far below it
    };
    template <class T>
    __device__ __forceinline__ void begin(State<T> &st, int64_t q0, int lane) const
    {
#pragma unroll
        for (int j = 0; j < T::QT; j++) {
            const int q = (int)q0 + 16 * j + (lane & 15);
            const bool in = q < a.n;
            const int row = in ? q : a.n - 1;
            const int64_t t = a.targets[row];
            const bool seen = t >= 0 && t < a.V && (!a.live || ((a.live[row * a.ld_live + (t >> 5)] >> (t & 31)) & 1u));
            st.da[j] = in && seen ? a.dlogp[row] * a.scale : 0.0f;
            st.db[j] = ENT && in ? a.dentropy[row] * a.scale : 0.0f;
            st.H[j] = ENT && st.db[j] != 0.0f ? a.entropy[row] : 0.0f;
            if constexpr (NP == 3) {
                const float2 r = a.rows[row];
                st.m[j] = r.x;
                st.lse[j] = r.y;
            } else {
                st.lse[j] = a.lse[row];
            }
            st.target[j] = in && seen ? (int32_t)(t - a.v0) : -0x7FFFFFFF;
        }
    }
    template <class T>
    __device__ __forceinline__ void end(State<T> &, int, int, int64_t, int) const {}
    template <class T>
    __device__ __forceinline__ void tile(State<T> &st, RowAcc<T> &acc, int64_t p0l, int64_t q0l, int lane, int) const
    {
        static_assert(T::QT == 4 && T::PT % 4 == 0, "a wave has whole groups of 64");
        const int p0 = (int)p0l, q0 = (int)q0l, h = lane >> 4, c = lane & 15;
        if (p0 >= a.vc || q0 >= a.npad) return;                       // uniform
        const bool checked = a.live || a.v0 + p0 + 16 * T::PT > a.V;  // uniform: a mask, or the table's end
#pragma unroll
        for (int b = 0; b < T::PT / 4; b++) {                         // 64 rows of the table
            if (p0 + 64 * b >= a.vc) break;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int q = q0 + 16 * j + c;
                const bool in = q < a.n;
                const float da = st.da[j], db = st.db[j];
                const bool dead = da == 0.0f && db == 0.0f;
                const uint32_t dp = (uint32_t)(st.target[j] - p0 - 64 * b);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    v4f &x = acc.v[4 * b + i][j];
                    const v4f z = x;
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        const float lp = log_p(st, z[r], j), pr = exp2_fast(lp * LOG2E);
                        float g = -da * pr;
                        if constexpr (ENT) g -= db * pr * (fmaxf(lp, -1e4f) + st.H[j]);
                        x[r] = g;
                    }
                    if (__any(dp >= (uint32_t)(16 * i) && dp < (uint32_t)(16 * i + 16))) {   // (seldom)
                        uint32_t at = dp - 16 * i - 4 * h;
                        asm volatile("" : "+v"(at));
#pragma unroll
                        for (int r = 0; r < 4; r++)
                            if (at == (uint32_t)r) {
                                const float lp = log_p(st, z[r], j), pr = exp2_fast(lp * LOG2E);
                                float g = da * (1.0f - pr);
                                if constexpr (ENT) g -= db * pr * (fmaxf(lp, -1e4f) + st.H[j]);
                                x[r] = g;
                            }
                    }
                    uint32_t bits = dead ? 0u : 0xFu;
                    if (checked) {
                        const int v = a.v0 + p0 + 64 * b + 16 * i + 4 * h, left = a.V - v;
                        if (left < 4) bits &= left <= 0 ? 0u : (1u << left) - 1u;
                        if (a.live && left > 0) bits &= a.live[(in ? q : 0) * a.ld_live + (v >> 5)] >> (v & 31);
                    }
#pragma unroll
                    for (int r = 0; r < 4; r++) x[r] = (bits >> r) & 1u ? x[r] : 0.0f;
                }
            }
            if constexpr (NP == 2) {
                // both pieces of a value in one register, where the value was: beside them they would not fit a wave's with the
                // largest tile
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++)
#pragma unroll
                        for (int r = 0; r < 4; r++) {
                            const float x = acc.v[4 * b + i][j][r], hi = (float)(__bf16)x;
                            acc.v[4 * b + i][j][r] = __builtin_bit_cast(float, (v2bf){(__bf16)(x - hi), (__bf16)hi});
                        }
                const auto pair = [](int u, float x, float y) {      // of two registers: the upper halves are first pieces
                    return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), u ? 0x05040100u : 0x07060302u);
                };
                write<T, 2>(
                    0, p0 + 64 * b, q0, lane,
                    [&](int u, int i, int j) {
                        const v4f x = acc.v[4 * b + i][j];
                        return (v2u){pair(u, x[0], x[1]), pair(u, x[2], x[3])};
                    },
                    [&](int u, int i, int r) {
                        return (v2u){pair(u, acc.v[4 * b + i][0][r], acc.v[4 * b + i][1][r]), pair(u, acc.v[4 * b + i][2][r], acc.v[4 * b + i][3][r])};
                    });
            } else {
                // pieces, one after the other: rounded off what is left
#pragma unroll 1
                for (int u = 0; u < NP; u++) {
                    v4bf o[4][4];
#pragma unroll
                    for (int i = 0; i < 4; i++)
#pragma unroll
                        for (int j = 0; j < 4; j++)
#pragma unroll
                            for (int r = 0; r < 4; r++) {
                                o[i][j][r] = (__bf16)acc.v[4 * b + i][j][r];
                                acc.v[4 * b + i][j][r] -= (float)o[i][j][r];
                            }
                    write<T, 1>(
                        u, p0 + 64 * b, q0, lane, [&](int, int i, int j) { return __builtin_bit_cast(v2u, o[i][j]); },
                        [&](int, int i, int r) { return __builtin_bit_cast(v2u, (v4bf){o[i][0][r], o[i][1][r], o[i][2][r], o[i][3][r]}); });
                }
            }
        }
    }
    // log p of a product, in natural units.  fp32: scale times a difference is exact inside the sum, which log2(e) is not.
    // bf16: the logit is rounded as lse is, so that a row that has all of the probability has 1 - p = 0 however large both are
    template <class S>
    __device__ __forceinline__ float log_p(const S &st, float z, int j) const
    {
        if constexpr (NP == 3) return fmaf(z - st.m[j], a.scale, -st.lse[j]);
        else return z * a.scale - st.lse[j];
    }
    // pieces u0 .. u0 + U - 1 of 64 x 64 values: by_row(u, i, j) a query's four, by_col(u, i, r) a row's.  (The pieces of a line
    // follow each other)
    template <class T, int U, class R, class C>
    __device__ __forceinline__ void write(int u0, int p, int q0, int lane, const R &by_row, const C &by_col) const
    {
        const int h = lane >> 4, c = lane & 15;
        if (a.g)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int q = q0 + 16 * j + c;
                __bf16 *to = a.g + (int64_t)q * a.gto.ld + (int64_t)(p / 32 + h / 2) * a.gto.block + u0 * a.gto.piece + 16 * (h & 1);
                if (q < a.n)
#pragma unroll
                    for (int u = 0; u < U; u++) {
                        *(v4u *)(to + 32 * u) = __builtin_shufflevector(by_row(u, 0, j), by_row(u, 1, j), 0, 1, 2, 3);
                        *(v4u *)(to + 32 * u + 8) = __builtin_shufflevector(by_row(u, 2, j), by_row(u, 3, j), 0, 1, 2, 3);
                    }
            }
        if (a.gt)
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    __bf16 *to = a.gt + (int64_t)(p + 16 * i + 4 * h + r) * a.gtto.ld + (q0 / 32 + c / 8) * a.gtto.block + u0 * a.gtto.piece + 4 * (c & 7);
#pragma unroll
                    for (int u = 0; u < U; u++) *(v2u *)(to + 32 * u) = by_col(u, i, r);
                }
    }
};

// For log p of fp32 rows: {largest product m, ln s} where m and s say the same as the lse that is given, to eight
// half steps of it, else {0, lse}: what is given counts.  lse is rounded at its own size, 2^-24 |lse|, which log p of a
// likely row inherits and 1 - p then magnifies (1,000 x 1,024 x 96, lse about 20: gradients off by 7e-6, with the pair
// 3e-6); scale (z - m) - ln s is rounded at the size of log p.  A wave per query.
__global__ __launch_bounds__(WG) void row_stats_kernel(StatsArgs a, float scale, const float *__restrict__ lse, float2 *__restrict__ out)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * (WG / 64) + (threadIdx.x >> 6);
    if (row >= a.n) return;
    const float4 *parts = a.parts + row * a.nparts;
    float m = HIDDEN, s = 0.0f, e = 0.0f;
    const auto add = [&](float pm, float ps) {
        float pe = 0.0f;
        const float m1 = max_of(m, pm);
        rebase(s, e, m, m1, a.c);
        rebase(ps, pe, pm, m1, a.c);
        s += ps;
        m = m1;
    };
    for (int i = lane; i < a.nparts; i += 64) add(parts[i].x, parts[i].y);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float pm = __shfl_xor(m, o), ps = __shfl_xor(s, o);
        add(pm, ps);
    }
    if (lane) return;
    const float given = lse[row];
    const double logs = log((double)s), own = (double)m * scale + logs;
    const bool same = m > HIDDEN && fabs(own - given) < 0x1p-21 * (fabs((double)given) + 1.0);
    out[row] = same ? make_float2(m, (float)logs) : make_float2(0.0f, given);
}

// sums of the splits, in their order; rows of dpad values, a multiple of four
__global__ __launch_bounds__(WG) void join_splits_kernel(const float *__restrict__ part, int splits, int64_t n, int cols, int dpad,
                                                         void *__restrict__ out, int64_t ld, int bf16_out)
{
    const int64_t total = n * dpad;
    for (int64_t t = (int64_t)blockIdx.x * WG + threadIdx.x; t * 4 < total; t += (int64_t)gridDim.x * WG) {
        v4f x = *(const v4f *)(part + t * 4);
        for (int s = 1; s < splits; s++) x += *(const v4f *)(part + s * total + t * 4);
        const int64_t r = t * 4 / dpad, o = r * ld;
        const int c = (int)(t * 4 - r * dpad);
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (c + e < cols) {
                if (bf16_out) ((__bf16 *)out)[o + c + e] = (__bf16)x[e];
                else ((float *)out)[o + c + e] = x[e];
            }
    }
}

__global__ __launch_bounds__(WG) void clear_rows_kernel(void *out, int64_t n, int64_t cols, int64_t ld, int width)
{
    for (int64_t t = (int64_t)blockIdx.x * WG + threadIdx.x; t < n * cols; t += (int64_t)gridDim.x * WG) {
        const int64_t r = t / cols, o = r * ld + (t - r * cols);
        if (width == 4) ((float *)out)[o] = 0.0f;
        else ((uint16_t *)out)[o] = 0;
    }
}

// workgroups for `threads` threads whose kernel goes on from there (a grid of 2^32 threads is none)
static unsigned capped(int64_t threads) { return (unsigned)std::min<int64_t>((threads + WG - 1) / WG, 1 << 20); }

// ---- launches ----------------------------------------------------------------------------------------

// Up to here a tile has all of the queries, so that the table is read once and as it is, and a query is finished by a
// whole workgroup.  So / by the larger tiles, us: 64 queries, 131,071 x 1024 bf16 72 / 133, 1M x 128 fp32 279 / 619, bytes
// 237 / 283; one query 64 / 125, 125 / 596 and 81 / 279.
#define FEW_ROWS 64

static int lies_vec(const void *p, int dtype, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld * dtype_width(dtype) % 16 == 0; }

static const uint32_t *any_live(const LogprobArgs &a, uint32_t *room, hipStream_t s, int *rc)
{
    if (!a.live || a.ld_live == 0) return a.live;
    const int64_t words = (a.V + 31) / 32;
    hipLaunchKernelGGL(any_live_kernel, dim3((unsigned)((words + WG - 1) / WG)), dim3(WG), 0, s, a.live, a.ld_live, a.n, words, room);
    if (hipGetLastError() != hipSuccess) {
        rairs_set_error("launch failed");
        *rc = RAIRS_EHIP;
    }
    return room;
}

#define NORM_WGS 1024

template <class S, class Q, bool VEC, bool NORM>
static void few_stats_launch(const FewStatsArgs &fa, hipStream_t s)
{
    const dim3 grid((unsigned)((fa.st.nparts + WG / 64 - 1) / (WG / 64)));
    if (fa.st.n <= 16) hipLaunchKernelGGL((few_stats_kernel<S, Q, 1, VEC, NORM>), grid, dim3(WG), 0, s, fa);
    else if (fa.st.n <= 32) hipLaunchKernelGGL((few_stats_kernel<S, Q, 2, VEC, NORM>), grid, dim3(WG), 0, s, fa);
    else hipLaunchKernelGGL((few_stats_kernel<S, Q, 4, VEC, NORM>), grid, dim3(WG), 0, s, fa);
}

template <class S, class Q>
static int few_stats(const FewStatsArgs &fa, bool vec, bool norm, hipStream_t s)
{
    if (vec && norm) few_stats_launch<S, Q, true, true>(fa, s);
    else if (vec) few_stats_launch<S, Q, true, false>(fa, s);
    else if (norm) few_stats_launch<S, Q, false, true>(fa, s);
    else few_stats_launch<S, Q, false, false>(fa, s);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

// A product of fp32 sums may be off by: every addition may round (or cut) at 2^-23 of a partial sum, which
// |q||t| bounds; the 64 covers the products of pieces that are left out and the smaller ones' sums, and the
// last term the bits that say which row of a group it is.
static float product_slack(int d) { return (1.1f * (float)d + 64.0f) * 1.1920929e-7f + 1.9073486e-6f; }

template <class S, class Q>
static int finish_launch(FinishArgs &f, hipStream_t s)
{
    f.dot_lanes = 1;
    while (f.dot_lanes < 64 && f.dot_lanes * DotLoad<S>::CH < f.d) f.dot_lanes *= 2;
    if (f.st.n <= FEW_ROWS) hipLaunchKernelGGL((logprob_finish_kernel<S, Q, 1024, 1>), dim3((unsigned)f.st.n), dim3(1024), 0, s, f);
    else hipLaunchKernelGGL((logprob_finish_kernel<S, Q, 64, 4>), dim3((unsigned)((f.st.n + 3) / 4)), dim3(256), 0, s, f);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

template <bool ENT, int TOP>
static int stats_launch(RowProd &rp, const StatsArgs &st, bool threes, bool large, int prun, hipStream_t s)
{
    if (threes)
        return large ? rowprod_launch<TileT, ROW_THREES>(rp, StatsEpi<ENT, TOP>{st, nullptr, nullptr}, s, prun)
                     : rowprod_launch<TileW, ROW_THREES>(rp, StatsEpi<ENT, TOP>{st, nullptr, nullptr}, s, prun);
    return large ? rowprod_launch<TileL>(rp, StatsEpi<ENT, TOP>{st, nullptr, nullptr}, s, prun)
                 : rowprod_launch<TileW>(rp, StatsEpi<ENT, TOP>{st, nullptr, nullptr}, s, prun);
}

// a few queries over rows that lie right
template <class T, int FLAGS>
static int few_tiles_launch(RowProd &rp, const StatsArgs &st, const uint32_t *any_live, float *xmax, int prun, hipStream_t s)
{
    return xmax ? rowprod_launch<T, FLAGS | ROW_NORM>(rp, StatsEpi<true, 2, true>{st, any_live, xmax}, s, prun)
                : rowprod_launch<T, FLAGS>(rp, StatsEpi<true, 0>{st, nullptr, nullptr}, s, prun);
}

template <int FLAGS>
static int few_tiles(RowProd &rp, const StatsArgs &st, const uint32_t *any_live, float *xmax, int prun, hipStream_t s)
{
    return st.n <= 16   ? few_tiles_launch<TileF1, FLAGS>(rp, st, any_live, xmax, prun, s)
           : st.n <= 32 ? few_tiles_launch<TileF2, FLAGS>(rp, st, any_live, xmax, prun, s)
                        : few_tiles_launch<TileF4, FLAGS>(rp, st, any_live, xmax, prun, s);
}

// The forward pass holds the parts and groups of as many queries at a time as this (10,000 queries over 1M rows in groups of
// 16: 5 GB); the table is laid out once.
#define STATS_BYTES (8ll << 30)

int rairs_run_logprob(const LogprobArgs &a, void *ws, size_t *bytes, hipStream_t s)
{
    const bool few = a.n <= FEW_ROWS;
    const int64_t blocks = (a.V + 63) / 64, kpad = pad_to(a.d, ROWPROD_K);
    // rounds of 64 rows per wave, up to 16, for 4,096 waves (four a SIMD) or a multiple
    const int64_t fills = (blocks + 16 * 4096 - 1) / (16 * 4096);
    const int rounds = few ? (int)((blocks + fills * 4096 - 1) / (fills * 4096)) : 1;
    const bool threes = !few && a.ttype == RAIRS_F32;
    const double ksum = (double)kpad * (dtype_pieces(a.ttype) * dtype_pieces(a.qtype) == 9 ? 6 : dtype_pieces(a.qtype));
    const int few_parts = (int)((blocks + rounds - 1) / rounds);
    bool large;
    int prun, runs, most_parts;
    const auto plan = [&](int64_t n) {
        large = rowprod_size(a.V, n) == 2;
        const int bp = few || large ? 256 : 128, bq = few ? 64 : threes ? 128 : bp;
        const int64_t ptiles = (a.V + bp - 1) / bp, qtiles = (n + bq - 1) / bq;
        // (a start costs a few microseconds, a tile 27 at K = 1024 and 256 x 256; one workgroup of the large tile
        // fits a CU, two of the smaller)
        prun = rowprod_run(ptiles, qtiles, few || large || threes ? 256 : 512, few ? 0.3 : 100.0 / (ksum + 200.0), 64);
        // (a few queries: by tiles, four waves along P, or rows straight from memory; there is room for either's parts)
        runs = (int)((ptiles + prun - 1) / prun);
        most_parts = few ? std::max(4 * runs, few_parts) : (threes && large ? 4 : 2) * runs;
    };
    // Groups of 16 rows or of 64.  Per query, the smaller ones cost two more operations a row and 8 bytes for 16 rows
    // instead of 4 for 64, about 0.14 ps times V; the larger ones 64 rows of the table for each of the `top`, at about
    // 6 TB/s.  (A few queries: the vector units have nothing else to do.)
    const int wide = !few && a.V > 76ll * a.top * a.d * dtype_width(a.ttype);
    plan(a.n);
    int64_t nc = a.n;                                                 // queries at a time: whole tiles, about as many each time
    const int64_t each = 16ll * most_parts + (!a.top ? 0 : wide ? pad_to(blocks, 4) * 4 : blocks * 32);
    if (!few && a.n * each > STATS_BYTES) {
        const int64_t fit = std::max<int64_t>(STATS_BYTES / each / 256 * 256, 256), times = (a.n + fit - 1) / fit;
        nc = pad_to((a.n + times - 1) / times, 256);
        plan(nc);
    }
    Carve w(ws);
    StatsArgs st = {};
    st.V = (int)a.V; st.c = a.scale * LOG2E; st.ld_live = a.ld_live;
    st.parts = w.take<float4>(nc * most_parts);
    st.wstride = (int)pad_to(blocks, 4);
    st.gmax = a.top ? w.take<float>(wide ? nc * st.wstride : nc * blocks * 4) : nullptr;
    st.gsecond = a.top && !wide ? w.take<float>(nc * blocks * 4) : nullptr;
    st.nblocks = (int)blocks;
    st.wide = wide;
    st.zt = w.take<float>(nc);
    float *xmax = w.take<float>(few ? most_parts : NORM_WGS);
    uint32_t *seen = w.take<uint32_t>(a.ld_live ? (a.V + 31) / 32 : 0);
    // (packed whether they need it or not, so that the size does not depend on where the rows lie)
    __bf16 *qroom = few ? nullptr : w.take<__bf16>(pack_room(a.qtype, a.n, a.d));
    __bf16 *troom = few ? nullptr : w.take<__bf16>(pack_room(a.ttype, a.V, a.d));
    uint32_t *piece_flags = w.take<uint32_t>(2);
    if (bytes) *bytes = w.used;
    if (!ws) return RAIRS_OK;

    int rc = RAIRS_OK;
    const uint32_t *seen_by_any = any_live(a, seen, s, &rc);
    if (rc) return rc;
    st.nparts = most_parts;
    FinishArgs f = {};
    f.table = a.table; f.ldt = a.ldt; f.ldq = a.ldq; f.d = a.d;
    f.vec = lies_vec(a.q, a.qtype, a.ldq) && lies_vec(a.table, a.ttype, a.ldt);
    f.scale = a.scale;
    f.slack = product_slack(a.d);
    f.xmax = xmax;
    f.top = a.top;
    // the queries from q0 on: of their statistics, and of what they are finished with
    const auto queries = [&](int64_t q0, int64_t n) {
        st.n = (int)n;
        st.targets = a.targets + q0;
        st.live = a.live ? a.live + q0 * a.ld_live : nullptr;
        f.q = (const char *)a.q + q0 * a.ldq * dtype_width(a.qtype);
        f.logp = a.logp + q0; f.lse = a.lse + q0; f.entropy = a.entropy ? a.entropy + q0 : nullptr;
        f.top_ids = a.top ? a.top_ids + q0 * a.top : nullptr;
        f.top_logp = a.top ? a.top_logp + q0 * a.top : nullptr;
    };
    const auto finish = [&]() {
        f.st = st;
        f.nxmax = few ? st.nparts : NORM_WGS;
        return a.ttype == RAIRS_BF16 ? finish_launch<__bf16, __bf16>(f, s)
               : a.ttype == RAIRS_F32 ? finish_launch<float, float>(f, s)
                                      : finish_launch<uint8_t, float>(f, s);
    };
    queries(0, nc < a.n ? nc : a.n);
    if (few && (f32_lies_right(a.table, a.ttype, a.ldt, a.d) && f32_lies_right(a.q, a.qtype, a.ldq, a.d))) {
        st.nparts = 4 * runs;
        RowProd rp = {};
        rowprod_pieces(rp, 1, 1);
        rp.ksteps = a.d / (ROWPROD_K / 2);
        rp.P = f32_operand(a.table, a.ldt, a.V);
        rp.Q = f32_operand(a.q, a.ldq, a.n);
        rc = few_tiles<ROW_F32>(rp, st, seen_by_any, a.top ? xmax : nullptr, prun, s);
        if (rc) return rc;
    } else if (few && rows_lie_right(a.table, a.ttype, a.ldt, a.d) && rows_lie_right(a.q, a.qtype, a.ldq, a.d)) {
        st.nparts = 4 * runs;
        RowProd rp = {};
        rowprod_pieces(rp, 1, 1);
        rp.ksteps = a.d / ROWPROD_K;
        rp.P = RowOperand{(const __bf16 *)a.table, a.ldt, 0, a.V, nullptr, nullptr};
        rp.Q = RowOperand{(const __bf16 *)a.q, a.ldq, 0, a.n, nullptr, nullptr};
        rc = few_tiles<0>(rp, st, seen_by_any, a.top ? xmax : nullptr, prun, s);
        if (rc) return rc;
    } else if (few) {
        st.nparts = few_parts;
        FewStatsArgs fa = {st, a.table, a.q, a.ldt, a.ldq, a.d, rounds, seen_by_any, xmax};
        const bool vec = lies_vec(a.table, a.ttype, a.ldt) && lies_vec(a.q, a.qtype, a.ldq);
        rc = a.ttype == RAIRS_BF16 ? few_stats<__bf16, __bf16>(fa, vec, a.top != 0, s)
             : a.ttype == RAIRS_F32 ? few_stats<float, float>(fa, vec, a.top != 0, s)
                                    : few_stats<uint8_t, float>(fa, vec, a.top != 0, s);
        if (rc) return rc;
    } else {
        if (a.top) {
            const int vec = lies_vec(a.table, a.ttype, a.ldt);
            if (a.ttype == RAIRS_BF16)
                hipLaunchKernelGGL(table_norm_kernel<__bf16>, dim3(NORM_WGS), dim3(WG), 0, s, (const __bf16 *)a.table, a.ldt, a.V, a.d, seen_by_any, vec, xmax);
            else if (a.ttype == RAIRS_F32)
                hipLaunchKernelGGL(table_norm_kernel<float>, dim3(NORM_WGS), dim3(WG), 0, s, (const float *)a.table, a.ldt, a.V, a.d, seen_by_any, vec, xmax);
            else
                hipLaunchKernelGGL(table_norm_kernel<uint8_t>, dim3(NORM_WGS), dim3(WG), 0, s, (const uint8_t *)a.table, a.ldt, a.V, a.d, seen_by_any, vec, xmax);
            RAIRS_HIP(hipGetLastError());
        }
        RowProd rp = {};
        rowprod_sums(rp, dtype_pieces(a.ttype), dtype_pieces(a.qtype), threes ? pad_to(a.d, 32) : kpad);
        // (queries of byte vectors are whole numbers as a rule, whose lower pieces are zero: packing them says so, and
        // the products of those pieces are left out)
        const bool flags = a.ttype == RAIRS_U8;
        if ((rc = rairs_operand(a.table, a.ttype, a.ldt, a.V, a.d, nullptr, threes, troom, rp.P, s, flags ? piece_flags : nullptr, true))) return rc;
        if ((rc = rairs_operand(a.q, a.qtype, a.ldq, a.n, a.d, nullptr, threes, qroom, rp.Q, s, flags ? piece_flags : nullptr, false))) return rc;
        if (flags) rp.Q.pieces_there = piece_flags;
        const bool ent = a.entropy != nullptr;
        const __bf16 *q = rp.Q.p;
        for (int64_t q0 = 0; q0 < a.n; q0 += nc) {
            queries(q0, std::min(nc, a.n - q0));
            rp.Q.p = q + q0 * rp.Q.ld;
            rp.Q.rows = st.n;
            if (a.top == 0) rc = ent ? stats_launch<true, 0>(rp, st, threes, large, prun, s) : stats_launch<false, 0>(rp, st, threes, large, prun, s);
            else if (wide) rc = ent ? stats_launch<true, 1>(rp, st, threes, large, prun, s) : stats_launch<false, 1>(rp, st, threes, large, prun, s);
            else rc = ent ? stats_launch<true, 2>(rp, st, threes, large, prun, s) : stats_launch<false, 2>(rp, st, threes, large, prun, s);
            if (rc || (rc = finish())) return rc;
        }
        return RAIRS_OK;
    }
    return finish();
}

// G is made for as many of the table's rows at a time as this holds, with what is laid out of the rows themselves beside it.
// (In pieces of 128 MB, which the last-level cache would keep, 4,095 x 65,537 x 1024 took 2.5 ms instead of 1.9, with G in one
// piece: five launches of each product that fill the card less well, and partial sums read again each time.)
#define GRAD_CHUNK_BYTES (8ll << 30)

template <int NP, bool ENT>
static int grad_launch(RowProd &rp, const GradArgs &ga, bool threes, hipStream_t s)
{
    if constexpr (NP == 3)
        if (threes)
            return rowprod_size(rp.P.rows, rp.Q.rows) == 2 ? rowprod_launch<TileT, ROW_THREES>(rp, GradEpi<NP, ENT>{ga}, s)
                                                           : rowprod_launch<TileW, ROW_THREES>(rp, GradEpi<NP, ENT>{ga}, s);
    // (three pieces of bytes' gradients: 128 x 128 alone, whose pieces fit the registers)
    if constexpr (NP == 3) return rowprod_launch<TileW>(rp, GradEpi<NP, ENT>{ga}, s);
    else
    return rowprod_size(rp.P.rows, rp.Q.rows) == 2
               ? rowprod_launch<TileL>(rp, GradEpi<NP, ENT>{ga}, s, rowprod_run((rp.P.rows + 255) / 256, (rp.Q.rows + 255) / 256, 256, 0.2, 64))
               : rowprod_launch<TileW>(rp, GradEpi<NP, ENT>{ga}, s);
}

int rairs_run_logprob_backward(const LogprobArgs &a, void *ws, size_t *bytes, hipStream_t s)
{
    const int np = dtype_pieces(a.qtype), tp = dtype_pieces(a.ttype);
    const int gp = np == 3 ? 3 : 2;                                   // pieces of the logits' gradient
    const bool threes = tp == 3, twos = gp == 2, again = np == 3;
    const int64_t kpad = pad_to(a.d, threes ? 32 : ROWPROD_K), npad = pad_to(a.n, ROWPROD_K), dpad = pad_to(a.d, 4);
    const bool need_dt = a.dtable != nullptr, need_dq = a.dq != nullptr;
    // bytes of a row of the table: G both ways, the row as it lies and turned
    const int64_t row = 2 * tp * pad_to(a.d, ROWPROD_K), each = 2 * gp * npad * (int64_t)(need_dq + need_dt) + row + (need_dq ? 2 * tp * a.d : 0);
    int64_t vc = GRAD_CHUNK_BYTES / each / 1024 * 1024;
    vc = vc < 1024 ? 1024 : std::min<int64_t>(vc, 1 << 20);           // (rows of threes: below 2^22 values)
    const int64_t chunks = (a.V + vc - 1) / vc;
    vc = pad_to((a.V + chunks - 1) / chunks, ROWPROD_K);              // of about one size
    // (fp32: the statistics need no G, and rows that are all laid out for them stay for the gradient)
    const int64_t vs = !again ? vc : std::max(vc, std::min(a.V, std::max<int64_t>(GRAD_CHUNK_BYTES / row / 1024 * 1024, 1024)));
    // the queries' product: its sum over the chunk is cut so that there are workgroups for every CU, of large tiles if
    // pieces of 2,048 rows (of the small tiles' 512) are enough for that
    const int64_t tl = rowprod_tiles(a.d, a.n, 256), tm = rowprod_tiles(a.d, a.n, 128), ts = rowprod_tiles(a.d, a.n, 64);
    int64_t splits = (256 + tl - 1) / tl;
    if (splits > vc / 2048) splits = std::min((256 + tm - 1) / tm, vc / 1024);
    if (splits * tm < 160) splits = std::min((512 + ts - 1) / ts, vc / (threes ? 128 : 512));
    if (splits < 1) splits = 1;
    Carve w(ws);
    __bf16 *qroom = w.take<__bf16>(pack_room(a.qtype, a.n, a.d));
    __bf16 *troom = w.take<__bf16>(pack_room(a.ttype, vs, a.d));
    __bf16 *tcols = need_dq ? w.take<__bf16>((int64_t)a.d * vc * tp) : nullptr;
    __bf16 *qcols = need_dt ? w.take<__bf16>((int64_t)a.d * npad * np) : nullptr;
    __bf16 *g = need_dq ? w.take<__bf16>(a.n * vc * gp) : nullptr;
    __bf16 *gt = need_dt ? w.take<__bf16>(vc * npad * gp) : nullptr;
    float *sums = need_dq ? w.take<float>(splits * a.n * dpad) : nullptr;
    uint32_t *seen = w.take<uint32_t>(a.ld_live ? (a.V + 31) / 32 : 0);
    // fp32: the statistics once more, by tiles as in the forward pass
    StatsArgs st = {};
    const auto large_of = [&](int64_t rows) { return rowprod_size(rows, a.n) == 2; };
    const auto run_of = [&](int64_t rows) {
        const bool l = large_of(rows);
        const int64_t side = l ? 256 : 128, ptiles = (rows + side - 1) / side, qtiles = (a.n + (threes ? 127 : side - 1)) / (threes ? 128 : side);
        return rowprod_run(ptiles, qtiles, l || threes ? 256 : 512, 100.0 / ((double)kpad * (threes ? 6 : 3) + 200.0), 64);
    };
    const auto parts_of = [&](int64_t rows) {
        const bool l = large_of(rows);
        const int64_t ptiles = (rows + (l ? 255 : 127)) / (l ? 256 : 128);
        return (threes && l ? 4 : 2) * ((ptiles + run_of(rows) - 1) / run_of(rows));
    };
    if (again) {
        for (int64_t v0 = 0; v0 < a.V; v0 += vs) st.nparts += (int)parts_of(std::min(vs, a.V - v0));
        st.parts = w.take<float4>(a.n * st.nparts);
        st.zt = w.take<float>(a.n);
    }
    float2 *rows_stats = again ? w.take<float2>(a.n) : nullptr;
    if (bytes) *bytes = w.used;
    if (!ws) return RAIRS_OK;

    int rc = RAIRS_OK;
    const uint32_t *seen_by_any = any_live(a, seen, s, &rc);
    if (rc) return rc;
    RowOperand Q = {};
    const PackLayout qto = pack_layout(a.d, npad, threes);
    const auto chunk = [&](int64_t v0) { return (const char *)a.table + v0 * a.ldt * dtype_width(a.ttype); };
    // what is laid out first: the queries and the table's first rows, both ways round
    PackJobs jobs = {};
    RowOperand P0 = {};
    const auto turn_table = [&](int64_t v0, int64_t rows, int64_t cpad) {
        PackJob &j = jobs.job[jobs.n++];
        j = PackJob{};
        j.src = chunk(v0); j.dst = tcols; j.dtype = a.ttype; j.turned = 1; j.ld = a.ldt; j.rows = rows; j.cols = a.d; j.pad = cpad;
        j.to = pack_layout(a.d, cpad, threes); j.order = ORDER_TABLE;
        // (rows that nobody sees are zero here: their G is zero, and they may hold anything)
        j.live = seen_by_any ? seen_by_any + v0 / 32 : nullptr;
    };
    rairs_operand_job(a.q, a.qtype, a.ldq, a.n, a.d, threes, qroom, Q, jobs);
    if (need_dt) {
        PackJob &j = jobs.job[jobs.n++];
        j = PackJob{};
        j.src = a.q; j.dst = qcols; j.dtype = a.qtype; j.turned = 1; j.ld = a.ldq; j.rows = a.n; j.cols = a.d; j.pad = npad;
        j.to = qto; j.order = ORDER_QUERIES;
        j.live = a.live; j.ld_live = a.ld_live; j.targets = a.targets; j.V = a.V; j.dlogp = a.dlogp; j.dentropy = a.dentropy;
    }
    if (again) {
        st.n = (int)a.n; st.c = a.scale * LOG2E; st.ld_live = a.ld_live; st.targets = a.targets;
        float4 *parts = st.parts;
        for (int64_t v0 = 0; v0 < a.V; v0 += vs) {
            const int64_t rows = std::min(vs, a.V - v0);
            RowProd rp = {};
            rairs_operand_job(chunk(v0), a.ttype, a.ldt, rows, a.d, threes, troom, rp.P, jobs);
            if (need_dq && vc >= a.V) turn_table(0, rows, pad_to(rows, ROWPROD_K));
            if ((rc = rairs_launch_pack(jobs, s))) return rc;
            jobs.n = 0;
            P0 = rp.P;
            rowprod_sums(rp, tp, np, kpad);
            rp.Q = Q;
            st.V = (int)rows;
            st.live = a.live ? a.live + v0 / 32 : nullptr;
            if ((rc = stats_launch<false, 0>(rp, st, threes, large_of(rows), run_of(rows), s))) return rc;
            st.parts += parts_of(rows);
        }
        st.parts = parts;
        hipLaunchKernelGGL(row_stats_kernel, dim3((unsigned)((a.n + WG / 64 - 1) / (WG / 64))), dim3(WG), 0, s, st, a.scale, a.lse_in, rows_stats);
        RAIRS_HIP(hipGetLastError());
    }
    for (int64_t v0 = 0; v0 < a.V; v0 += vc) {
        const int64_t rows = a.V - v0 < vc ? a.V - v0 : vc, cpad = pad_to(rows, ROWPROD_K);
        RowProd rp = {};
        if (again && vs >= a.V) {
            rp.P = P0;                                                // (laid out above)
            rp.P.p += v0 * P0.ld;
            rp.P.rows = rows;
        } else {
            rairs_operand_job(chunk(v0), a.ttype, a.ldt, rows, a.d, threes, troom, rp.P, jobs);
        }
        if (need_dq && !(again && vc >= a.V)) turn_table(v0, rows, cpad);
        if ((rc = rairs_launch_pack(jobs, s))) return rc;
        jobs.n = 0;
        rowprod_sums(rp, tp, np, kpad);
        rp.Q = Q;
        GradArgs ga = {};
        ga.n = (int)a.n; ga.V = (int)a.V; ga.v0 = (int)v0; ga.vc = (int)cpad; ga.npad = (int)npad;
        ga.scale = a.scale;
        ga.live = a.live; ga.ld_live = a.ld_live; ga.targets = a.targets;
        ga.rows = rows_stats;
        ga.lse = a.lse_in; ga.entropy = a.entropy_in; ga.dlogp = a.dlogp; ga.dentropy = a.dentropy;
        ga.g = g; ga.gt = gt;
        ga.gto = twos ? pack_twos(cpad) : pack_layout(a.n, cpad, threes);
        ga.gtto = twos ? pack_twos(npad) : pack_layout(cpad, npad, threes);
        const bool ent = a.dentropy != nullptr;
        if (np == 3) rc = ent ? grad_launch<3, true>(rp, ga, threes, s) : grad_launch<3, false>(rp, ga, threes, s);
        else rc = ent ? grad_launch<2, true>(rp, ga, threes, s) : grad_launch<2, false>(rp, ga, threes, s);
        if (rc) return rc;
        // (products of G with pieces of a table or of queries)
        const auto sums_of = [&](RowProd &rp, int pieces, int64_t values) {
            if (!twos) return rowprod_sums(rp, pieces, gp, values);
            rowprod_pieces(rp, 1, 1);
            rp.ksteps = (int)(values / 32);
        };
        const auto launch = [&](RowProd &rp, const StoreEpi &e) {
            return threes ? rowprod_launch_any<ROW_THREES>(rp, e, s) : twos ? rowprod_launch_any<ROW_TWOS>(rp, e, s) : rowprod_launch_any(rp, e, s);
        };
        RowProd pq = {}, pt = {};
        StoreEpi eq = {}, et = {};
        if (need_dq) {
            const PackLayout tto = pack_layout(a.d, cpad, threes);
            sums_of(pq, tp, cpad);
            pq.P = RowOperand{tcols, tto.ld, tto.piece, a.d, nullptr, nullptr};
            pq.Q = RowOperand{g, ga.gto.ld, twos ? 0 : ga.gto.piece, a.n, nullptr, nullptr};
            pq.splits = (int)splits;
            eq = StoreEpi{sums, dpad, a.n * dpad, a.d, a.n, nullptr, 0, v0 > 0};
        }
        if (need_dt) {
            sums_of(pt, np, npad);
            pt.P = RowOperand{qcols, qto.ld, qto.piece, a.d, nullptr, nullptr};
            pt.Q = RowOperand{gt, ga.gtto.ld, twos ? 0 : ga.gtto.piece, rows, nullptr, nullptr};
            et = StoreEpi{(char *)a.dtable + v0 * a.lddt * dtype_width(a.ttype), a.lddt, 0, a.d, rows, nullptr, a.ttype == RAIRS_BF16, 0};
        }
        // (both of small tiles: side by side; fp32 1,000 x 1,024 x 96 22.5 us, one after the other 26.6)
        if (need_dq && need_dt && rowprod_size(a.d, a.n, (int)splits) == 0 && rowprod_size(a.d, rows) == 0) {
            if ((rc = threes ? rowprod_launch_pair<TileU, ROW_THREES>(pq, eq, pt, et, s) : rowprod_launch_pair<TileS, ROW_TWOS>(pq, eq, pt, et, s))) return rc;
            continue;
        }
        if (need_dq && (rc = launch(pq, eq))) return rc;
        if (need_dt && (rc = launch(pt, et))) return rc;
    }
    if (need_dq) {
        hipLaunchKernelGGL(join_splits_kernel, dim3(capped(a.n * dpad / 4)), dim3(WG), 0, s, sums, (int)splits, a.n, a.d,
                           (int)dpad, a.dq, a.lddq, (int)(a.qtype == RAIRS_BF16));
        RAIRS_HIP(hipGetLastError());
    }
    return RAIRS_OK;
}

int rairs_launch_clear_rows(void *out, int64_t n, int64_t cols, int64_t ld, int dtype, hipStream_t s)
{
    if (n == 0 || cols == 0) return RAIRS_OK;
    hipLaunchKernelGGL(clear_rows_kernel, dim3(capped(n * cols)), dim3(WG), 0, s, out, n, cols, ld, dtype_width(dtype));
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}
