// Products of a few rows with many that lie otherwise than rowprod.h's tiles need them (any stride, alignment and
// length; bytes), and products that are small altogether: a wave takes 16 PT of the many rows and all of the few,
// and both operands go from memory straight into the matrix instruction's registers.  A load costs a cache access for
// each lane's row, which is what bounds these calls (16 queries against 131,071 x 1024 bf16: 80 us, by tiles 65; 64 queries
// against 1M x 128 fp32: 321 us, by tiles 279; 1M x 128 bytes, which have no tiles here: 80 us for one query, 100 for 16, 237
// for 64); the few come from the caches.  A lane holds 16 bytes of a row
// per load, so that four lanes read 64 consecutive bytes of it, and the four loads in flight a line.
//
// bf16 rows use the 16 x 16 x 32 instruction, fp32 rows the fp32 one (16 x 16 x 4: 64 operations a cycle
// and SIMD are enough next to memory for up to 64 rows), byte rows are widened to fp32.  The order in
// which the summed dimension is taken does not matter to the instruction as long as both operands
// agree: lane group g takes values g CH .. g CH + CH - 1 of a step.
#pragma once
#include "rowprod.h"

template <class S>
struct FewLoad {                    // values per lane and step, by the type of the many rows
    static constexpr int CH = 16 / sizeof(S);
};

template <class S, int CH>
struct FewFrag {
    S e[CH];
};

// CH values of a row from k on, zero from d on; ONCE: they are not read again
template <class S, int CH, bool VEC, bool ONCE = false>
static __device__ __forceinline__ FewFrag<S, CH> few_load(const S *row, int k, int d)
{
    FewFrag<S, CH> f;
    if (VEC && k <= d - CH) {
        if constexpr (CH * sizeof(S) == 8) {
            const v2u x = *(const v2u *)(row + k);
            __builtin_memcpy(f.e, &x, 8);
        } else {
#pragma unroll
            for (int w = 0; w < CH * (int)sizeof(S) / 16; w++) {
                const v4u *from = (const v4u *)(row + k + w * (16 / sizeof(S)));
                const v4u x = ONCE ? __builtin_nontemporal_load(from) : *from;
                __builtin_memcpy(&f.e[w * (16 / sizeof(S))], &x, 16);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < CH; e++) f.e[e] = k + e < d ? row[k + e] : (S)0;
    }
    return f;
}

// instruction e of a step's products (bf16: one; fp32: one for each value of a lane)
template <class S, int CH>
struct FewMfma {
    static constexpr int N = CH;
    static __device__ __forceinline__ v4f go(const FewFrag<S, CH> &a, const FewFrag<float, CH> &b, int e, v4f c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x4f32((float)a.e[e], b.e[e], c, 0, 0, 0);
    }
};
template <int CH>
struct FewMfma<__bf16, CH> {
    static constexpr int N = 1;
    static __device__ __forceinline__ v4f go(const FewFrag<__bf16, CH> &a, const FewFrag<__bf16, CH> &b, int, v4f c)
    {
        v8bf x, y;
        __builtin_memcpy(&x, a.e, 16);
        __builtin_memcpy(&y, b.e, 16);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
    }
};

// KU steps: 4 KU CH values of every row, from value k on for this lane.  The loads of a row follow each other, so
// that the pieces of a line are asked for at once (asked for a row tile later they cost a third of the
// bandwidth: 4.6 TB/s instead of 6.5 for rows of 512 bytes).
template <class S, class Q, int PT, int QT, int KU, bool VEC, bool NORM>
static __device__ __forceinline__ void few_steps(const S *const (&prow)[PT], const Q *const (&qrow)[QT], int k, int d, v4f (&acc)[PT][QT],
                                                 float (&nrm)[PT])
{
    constexpr int CH = FewLoad<S>::CH, STEP = 4 * CH;
    FewFrag<S, CH> a[PT][KU];
    FewFrag<Q, CH> b[KU][QT];
#pragma unroll
    for (int i = 0; i < PT; i++)
#pragma unroll
        for (int s = 0; s < KU; s++) a[i][s] = few_load<S, CH, VEC, true>(prow[i], k + s * STEP, d);
#pragma unroll
    for (int s = 0; s < KU; s++)
#pragma unroll
        for (int j = 0; j < QT; j++) b[s][j] = few_load<Q, CH, VEC, false>(qrow[j], k + s * STEP, d);
    __builtin_amdgcn_sched_barrier(0);                                // (all of them are under way first)
    // (products onto the same sums as far apart as can be: each waits for the one before it)
#pragma unroll
    for (int s = 0; s < KU; s++)
#pragma unroll
        for (int e = 0; e < FewMfma<S, CH>::N; e++)
#pragma unroll
            for (int i = 0; i < PT; i++)
#pragma unroll
                for (int j = 0; j < QT; j++) acc[i][j] = FewMfma<S, CH>::go(a[i][s], b[s][j], e, acc[i][j]);
    if constexpr (NORM) {
#pragma unroll
        for (int i = 0; i < PT; i++)
#pragma unroll
            for (int s = 0; s < KU; s++)
#pragma unroll
                for (int e = 0; e < CH; e++) nrm[i] = fmaf((float)a[i][s].e[e], (float)a[i][s].e[e], nrm[i]);
    }
}

// acc += rows prow (many) times rows qrow (few) over the steps [s0, s1); prow/qrow: this lane's rows
// (p tile i: row lane & 15 of it).  NORM: nrm[i] collects this lane's part of |p row|^2.
template <class S, class Q, int PT, int QT, bool VEC, bool NORM>
static __device__ __forceinline__ void few_dot(const S *const (&prow)[PT], const Q *const (&qrow)[QT], int s0, int s1, int d, int lane,
                                               v4f (&acc)[PT][QT], float (&nrm)[PT])
{
    // as many steps at once as registers hold: the few rows' operands are QT (bytes: 4 QT) registers of four each
    constexpr int STEP = 4 * FewLoad<S>::CH, KU = QT * (int)(sizeof(Q) / sizeof(S)) <= 2 ? 4 : QT * (int)(sizeof(Q) / sizeof(S)) <= 4 ? 2 : 1;
    const int off = (lane >> 4) * FewLoad<S>::CH, whole = VEC ? (d / STEP < s1 ? d / STEP : s1) : s0;
    int s = s0;
    // (the bound that few_load compares with is out of reach in whole steps: no comparison is left)
#pragma unroll 1
    for (; s + KU <= whole; s += KU) few_steps<S, Q, PT, QT, KU, VEC, NORM>(prow, qrow, s * STEP + off, 0x7FFFFFFF, acc, nrm);
#pragma unroll 1
    for (; s < s1; s++) few_steps<S, Q, PT, QT, 1, VEC, NORM>(prow, qrow, s * STEP + off, d, acc, nrm);
}
