// Products of rows with rows on the bf16 matrix cores: out[q][p] = sum_k Q[q][k] P[p][k], the form that
// every large product of the projection and of the log probabilities is brought into (both operands
// with the summed dimension contiguous), with what is done to a tile's results left to a functor.
//
// Values of more than 8 bits go in as sums of bf16 pieces, three for fp32 (24 bits), and a product is
// the sum of the products of pieces that matter: of nine the six with the larger factors, the small
// ones first (what is left out is below 2^-23 |P||Q|).  A piece list is only a longer sum, so bf16
// rows, fp32 rows and byte rows share one kernel.
//
// A workgroup stages 64 values of each of its rows in LDS, two buffers, fetched straight into LDS by
// 16-byte loads.  Such a load writes lane l's bytes at base + 16 l, so the order in LDS is chosen by
// the address that each lane reads: slot s of row r holds the row's 16-byte chunk s ^ (r & 7), which
// keeps a global access 128 bytes long and the operand reads (16 rows, one chunk) free of bank conflicts.
#pragma once
#include "device_util.h"

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

#define ROWPROD_K 64                // values of a row in LDS at a time

// Rows of bf16 pieces: value k of piece i of row r at p[i * piece + r * ld + k]; ld a multiple of 8,
// p 16-byte aligned, k up to a multiple of ROWPROD_K readable (zero beyond the row).
struct RowOperand {
    const __bf16 *p;
    int64_t ld, piece;
    int64_t rows;
    const int32_t *perm;            // row r of the product is row perm[r] here (null: r)
};

// The part of a sum that depends on the row's adapter: rows are sorted by adapter, a tile runs over
// the adapters of its rows, with the other rows' u taken from a row of zeros.
struct AdapterPart {
    const __bf16 *u;                // [q rows][kpad]
    const __bf16 *b;                // [adapters][p rows][kpad]
    const __bf16 *zero;             // [kpad] zeros
    const int32_t *of_row;          // [q rows] adapter of each row in product order, -1: none
    const int32_t *end;             // [adapters] one past an adapter's last row
    int kpad;                       // multiple of ROWPROD_K; 0: no adapters
};

struct RowProd {
    RowOperand P, Q;
    int nseg;                       // products of pieces
    uint8_t sp[6], sq[6];           // piece of P and of Q of each
    int ksteps;                     // steps of ROWPROD_K per product
    int splits;                     // workgroups that share a tile's sum
    int ptiles, qtiles;
    AdapterPart ad;
};

static inline void rowprod_pieces(RowProd &a, int np, int nq)
{
    a.nseg = 0;
    for (int s = (np - 1) + (nq - 1); s >= 0; s--)                   // the smallest products first
        for (int i = np - 1; i >= 0; i--) {
            const int j = s - i;
            if (j < 0 || j >= nq || s > (np > nq ? np : nq) - 1) continue;
            a.sp[a.nseg] = (uint8_t)i;
            a.sq[a.nseg] = (uint8_t)j;
            a.nseg++;
        }
}

// PT x QT tiles of 16 x 16 per wave, WP x WQ waves.
template <int PT_, int QT_, int WP_, int WQ_>
struct RowTile {
    static constexpr int PT = PT_, QT = QT_, WP = WP_, WQ = WQ_, NT = 64 * WP * WQ;
    static constexpr int BP = 16 * PT * WP, BQ = 16 * QT * WQ;
    static constexpr int LP = BP * 8 / NT, LQ = BQ * 8 / NT;          // 16-byte loads per thread and step
    static constexpr int BYTES = (BP + BQ) * 128;                     // of one LDS buffer
};

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

template <class T>
struct RowAcc {
    v4f v[T::PT][T::QT];
};

// one step's 16-byte chunks of both operands, straight into LDS
template <class T>
static __device__ __forceinline__ void rowprod_fetch(char *buf, const __bf16 *const (&pp)[T::LP], const __bf16 *const (&qp)[T::LQ],
                                                     int64_t op, int64_t oq, int wave)
{
#pragma unroll
    for (int i = 0; i < T::LP; i++)
        __builtin_amdgcn_global_load_lds((global_void *)(pp[i] + op), (lds_void *)(buf + (i * T::NT + wave * 64) * 16), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < T::LQ; i++)
        __builtin_amdgcn_global_load_lds((global_void *)(qp[i] + oq), (lds_void *)(buf + T::BP * 128 + (i * T::NT + wave * 64) * 16), 16,
                                         0, 0);
}

// every load into LDS of this wave has landed, then every wave's
static __device__ __forceinline__ void rowprod_landed()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

template <class T>
static __device__ __forceinline__ void rowprod_step(const char *buf, int wp, int wq, int lane, RowAcc<T> &acc)
{
#pragma unroll
    for (int kk = 0; kk < 2; kk++) {
        const int slot = ((kk * 4 + (lane >> 4)) ^ (lane & 7)) * 16 + (lane & 15) * 128;
        v8bf a[T::PT], b[T::QT];
#pragma unroll
        for (int i = 0; i < T::PT; i++) a[i] = *(const v8bf *)(buf + (wp * T::PT + i) * 2048 + slot);
#pragma unroll
        for (int j = 0; j < T::QT; j++) b[j] = *(const v8bf *)(buf + T::BP * 128 + (wq * T::QT + j) * 2048 + slot);
#pragma unroll
        for (int i = 0; i < T::PT; i++)
#pragma unroll
            for (int j = 0; j < T::QT; j++) acc.v[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], acc.v[i][j], 0, 0, 0);
    }
}

// Workgroup's tile: neighbouring workgroups of one XCD (they are handed out round robin over the
// eight) take the q tiles of the same p tile one after the other, so that its rows come from that
// XCD's L2 cache after the first.
static __device__ __forceinline__ bool rowprod_tile(const RowProd &a, int &pt, int &qt, int &split)
{
    const uint32_t total = (uint32_t)(a.ptiles * a.qtiles * a.splits), per = (total + 7) / 8;
    const uint32_t id = (blockIdx.x % 8) * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || id >= total) return false;
    qt = (int)(id % a.qtiles);
    pt = (int)(id / a.qtiles % a.ptiles);
    split = (int)(id / (a.qtiles * a.ptiles));
    return true;
}
static inline unsigned rowprod_grid(const RowProd &a)
{
    const uint32_t total = (uint32_t)(a.ptiles * a.qtiles * a.splits);
    return (total + 7) / 8 * 8;
}

// The epilogue is called as epi(acc, p0, q0, lane, split): lane l holds, for its tiles (i, j), rows
// q0 + 16 j + (l & 15) and columns p0 + 16 i + 4 (l >> 4) + 0..3.
template <class T, class Epi>
__global__ __launch_bounds__(T::NT) void rowprod_kernel(RowProd a, Epi epi)
{
    extern __shared__ __align__(16) char rowprod_lds[];
    int pt, qt, split;
    if (!rowprod_tile(a, pt, qt, split)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = wave % T::WP, wq = wave / T::WP;
    const int64_t p0 = (int64_t)pt * T::BP, q0 = (int64_t)qt * T::BQ;

    const int chunk = ((tid & 7) ^ ((tid >> 3) & 7)) * 8;             // (NT / 8 is a multiple of 8: the same for every load)
    const __bf16 *pp[T::LP], *qp[T::LQ];
#pragma unroll
    for (int i = 0; i < T::LP; i++) {
        int64_t r = p0 + i * (T::NT / 8) + (tid >> 3);
        r = r < a.P.rows ? r : a.P.rows - 1;                          // (rows beyond the last: computed, not stored)
        if (a.P.perm) r = a.P.perm[r];
        pp[i] = a.P.p + r * a.P.ld + chunk;
    }
#pragma unroll
    for (int i = 0; i < T::LQ; i++) {
        int64_t r = q0 + i * (T::NT / 8) + (tid >> 3);
        r = r < a.Q.rows ? r : a.Q.rows - 1;
        if (a.Q.perm) r = a.Q.perm[r];
        qp[i] = a.Q.p + r * a.Q.ld + chunk;
    }
    RowAcc<T> acc;
#pragma unroll
    for (int i = 0; i < T::PT; i++)
#pragma unroll
        for (int j = 0; j < T::QT; j++) acc.v[i][j] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};

    const int steps = a.nseg * a.ksteps;
    const int s0 = (int)((int64_t)steps * split / a.splits), s1 = (int)((int64_t)steps * (split + 1) / a.splits);
    char *b0 = rowprod_lds, *b1 = rowprod_lds + T::BYTES;
    if (s0 < s1) {
        int seg = s0 / a.ksteps, k = s0 % a.ksteps;
        rowprod_fetch<T>(b0, pp, qp, a.sp[seg] * a.P.piece + k * ROWPROD_K, a.sq[seg] * a.Q.piece + k * ROWPROD_K, wave);
        rowprod_landed();
        for (int s = s0; s < s1; s++) {
            if (s + 1 < s1) {
                if (++k == a.ksteps) { k = 0; seg++; }
                rowprod_fetch<T>(b1, pp, qp, a.sp[seg] * a.P.piece + k * ROWPROD_K, a.sq[seg] * a.Q.piece + k * ROWPROD_K, wave);
            }
            rowprod_step<T>(b0, wp, wq, lane, acc);
            rowprod_landed();
            char *t = b0; b0 = b1; b1 = t;
        }
    }
    if (a.ad.kpad) {                                                  // uniform
        const int64_t qend = q0 + T::BQ < a.Q.rows ? q0 + T::BQ : a.Q.rows;
        for (int64_t pos = q0; pos < qend;) {
            const int ad = a.ad.of_row[pos];
            if (ad < 0) break;                                        // rows without an adapter are the last
            pos = a.ad.end[ad];
#pragma unroll
            for (int i = 0; i < T::LP; i++) {
                int64_t r = p0 + i * (T::NT / 8) + (tid >> 3);
                r = r < a.P.rows ? r : a.P.rows - 1;
                pp[i] = a.ad.b + ((int64_t)ad * a.P.rows + r) * a.ad.kpad + chunk;
            }
#pragma unroll
            for (int i = 0; i < T::LQ; i++) {
                int64_t r = q0 + i * (T::NT / 8) + (tid >> 3);
                r = r < a.Q.rows ? r : a.Q.rows - 1;
                qp[i] = (a.ad.of_row[r] == ad ? a.ad.u + r * a.ad.kpad : a.ad.zero) + chunk;
            }
            for (int k = 0; k < a.ad.kpad; k += ROWPROD_K) {
                rowprod_fetch<T>(b0, pp, qp, k, k, wave);
                rowprod_landed();
                rowprod_step<T>(b0, wp, wq, lane, acc);
                rowprod_landed();
            }
        }
    }
    epi(acc, p0 + wp * (16 * T::PT), q0 + wq * (16 * T::QT), lane, split);
}

template <class T, class Epi>
static int rowprod_launch(RowProd &a, const Epi &epi, hipStream_t s)
{
    a.ptiles = (int)((a.P.rows + T::BP - 1) / T::BP);
    a.qtiles = (int)((a.Q.rows + T::BQ - 1) / T::BQ);
    if (a.splits < 1) a.splits = 1;
    auto kern = rowprod_kernel<T, Epi>;
    RAIRS_HIP(hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * T::BYTES));
    hipLaunchKernelGGL(kern, dim3(rowprod_grid(a)), dim3(T::NT), 2 * T::BYTES, s, a, epi);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

// ---- epilogues -------------------------------------------------------------------------------------

// out[row][p] = value, as fp32 or bf16; splits write their own sums, `split` elements apart
struct StoreEpi {
    void *out;
    int64_t ld, split_stride;
    int64_t np, nq;                 // columns, rows
    const int32_t *perm;            // row r goes to row perm[r] (null: r)
    int bf16_out, add;              // add (fp32 only): onto what is there
    template <class T>
    __device__ __forceinline__ void operator()(const RowAcc<T> &acc, int64_t p0, int64_t q0, int lane, int split) const
    {
        // four values at once where every row starts on a multiple of four elements
        const bool four = ld % 4 == 0 && (bf16_out ? ((uintptr_t)out & 7) == 0 : ((uintptr_t)out & 15) == 0) && split_stride % 4 == 0;
#pragma unroll
        for (int j = 0; j < T::QT; j++) {
            const int64_t q = q0 + 16 * j + (lane & 15);
            if (q >= nq) continue;
            const int64_t row = (perm ? perm[q] : q) * ld + split * split_stride;
#pragma unroll
            for (int i = 0; i < T::PT; i++) {
                const int64_t p = p0 + 16 * i + 4 * (lane >> 4);
                v4f x = acc.v[i][j];
                if (four && p + 4 <= np) {
                    if (bf16_out) {
                        const v4bf y = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
                        *(v4bf *)((__bf16 *)out + row + p) = y;
                    } else {
                        v4f *o = (v4f *)((float *)out + row + p);
                        if (add) x += *o;
                        *o = x;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (p + e < np) {
                            if (bf16_out) ((__bf16 *)out)[row + p + e] = (__bf16)x[e];
                            else ((float *)out)[row + p + e] = add ? ((float *)out)[row + p + e] + x[e] : x[e];
                        }
                }
            }
        }
    }
};
