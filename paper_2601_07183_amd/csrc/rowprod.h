// Products of rows with rows on the bf16 matrix cores: out[q][p] = sum_k Q[q][k] P[p][k], the form that
// every large product of the projection and of the log probabilities is brought into (both operands
// with the summed dimension contiguous), with what is done to a tile's results left to a functor.
//
// Values of more than 8 bits go in as sums of bf16 pieces, three for fp32 (24 bits), and a product is
// the sum of the products of pieces that matter: of nine the six with the larger factors (what is left out is
// below 2^-23 |P||Q|).  A piece list is only a longer sum, so bf16 rows, byte rows and fp32 rows share one kernel.
//
// fp32 with fp32 ("threes") goes by steps of 32 values with all three pieces of both in LDS, from rows in which each
// 32 values' pieces follow each other: six products of what is read once, which halves the traffic (2,999 x 1024 x 960
// with adapters: 49 us, 66 as six sums one after the other).  The products with smaller factors have sums of their own, added at the end, so that they
// do not round the large one's.
//
// Rows of bf16 against values in two pieces ("twos": the gradient of the logits) go by steps of 32 values too, with both
// pieces of Q in LDS and P once.
//
// Small products of fp32 rows take the rows as they are and the fp32 matrix instruction (a sixteenth of the
// bf16 rate, against six products of pieces and the packing): lengths, strides and steps are then counted in
// units of two bytes all the same, so that a step is 32 values.
//
// A workgroup stages 64 values of each of its rows in LDS, fetched straight into LDS by 16-byte loads into a ring
// of two buffers (large tiles, whose products take longer than a load) to four (small ones).  Such a load writes
// lane l's bytes at base + 16 l, so the order in LDS is chosen by the address that each lane reads: slot s of row r holds the row's 16-byte chunk s ^ (r & 7), which
// keeps a global access 128 bytes long and the operand reads (16 rows, one chunk) free of bank conflicts.
#pragma once
#include <algorithm>

#include "device_util.h"

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

#define ROWPROD_K 64                // values of a row in LDS at a time

// Rows of bf16 pieces: value k of piece i of row r at p[i * piece + r * ld + k]; ld a multiple of 8, below
// 2^22, p 16-byte aligned, k up to a multiple of ROWPROD_K readable (zero beyond the row).  Rows of fp32: units of
// two bytes in place of values.  Threes: 32 values of piece 0, of piece 1, of piece 2, then the next 32 values; twos likewise.
struct RowOperand {
    const __bf16 *p;
    int64_t ld, piece;
    int64_t rows;
    const int32_t *perm;            // Q only: row r of the product is row perm[r] here (null: r); then rows * ld below 2^31
    const uint32_t *pieces_there;   // Q only: word i is 0 if piece i + 1 is zero everywhere (null: not known)
};

// The part of a sum that depends on the row's adapter: rows are sorted by adapter, a tile runs over
// the adapters of its rows, with the other rows' u taken from a row of zeros.
struct AdapterPart {
    const __bf16 *u;                // [q rows][kpad]
    const __bf16 *b;                // [adapters][p rows][kpad]
    const __bf16 *zero;             // [kpad] zeros
    const int32_t *of_row;          // [q rows] adapter of each row in product order, -1: none
    const int32_t *end;             // [adapters] one past an adapter's last row
    int kpad;                       // multiple of ROWPROD_K (threes: of 96); 0: no adapters
};

struct RowProd {
    RowOperand P, Q;
    int nseg;                       // products of pieces
    uint32_t sp, sq;                // piece of P and of Q of each, four bits a product
    int ksteps;                     // steps of ROWPROD_K (threes and fp32: 32 values) per product
    int splits;                     // workgroups that share a tile's sum
    int ptiles, qtiles;             // tiles, and workgroups along P: each takes prun tiles
    int prun, pruns;
    int band;                       // q tiles whose workgroups take the runs together
    AdapterPart ad;
};

static inline void rowprod_pieces(RowProd &a, int np, int nq)
{
    a.nseg = 0;
    a.sp = a.sq = 0;
    for (int s = (np - 1) + (nq - 1); s >= 0; s--)                   // the smallest products first
        for (int i = np - 1; i >= 0; i--) {
            const int j = s - i;
            if (j < 0 || j >= nq || s > (np > nq ? np : nq) - 1) continue;
            a.sp |= (uint32_t)i << (4 * a.nseg);
            a.sq |= (uint32_t)j << (4 * a.nseg);
            a.nseg++;
        }
}

// PT x QT tiles of 16 x 16 per wave, WP x WQ waves; a ring of ST buffers.
template <int PT_, int QT_, int WP_, int WQ_, int ST_>
struct RowTile {
    static constexpr int PT = PT_, QT = QT_, WP = WP_, WQ = WQ_, NT = 64 * WP * WQ, ST = ST_;
    static constexpr int BP = 16 * PT * WP, BQ = 16 * QT * WQ;
    static constexpr int LP = BP * 8 / NT, LQ = BQ * 8 / NT ? BQ * 8 / NT : 1;   // 16-byte loads per thread and step
    static constexpr bool SOME_Q = BQ * 8 < NT;                       // (the first waves alone load Q)
    static constexpr int LEAST = LP + (SOME_Q ? 0 : LQ);              // loads that every wave makes
    static constexpr int BYTES = (BP + BQ) * 128;                     // of one LDS buffer
};

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

// What bounds a tile is LDS next to the matrix cores: a step of 256 x 256 is 64 KB to write and 192 KB to read for
// 2,048 cycles of products, of 128 x 128 32 and 96 KB for 512.  Large tiles need less of the caches, small ones give more
// workgroups.  Measured (bf16, us, 256 / 128 / 64): 4096 x 8191 x 4096 251 / 339 / 600; 1024 x 4096 x 13120 270 / 126 / 239;
// 1024 x 512 x 1024 30 / 14 / 9.  The largest reach 1.1 PFLOP/s (4096 x 128,000 x 1024 with the statistics: 1.0 ms).
typedef RowTile<8, 4, 2, 4, 2> TileL;       // 256 x 256, 8 waves
typedef RowTile<4, 2, 2, 4, 3> TileM;       // 128 x 128, 8 waves
typedef RowTile<2, 2, 2, 2, 4> TileS;       // 64 x 64, 4 waves
typedef RowTile<4, 4, 4, 2, 2> TileT;       // 256 x 128, 8 waves: what threes have for TileL
typedef RowTile<2, 2, 2, 2, 3> TileU;       // 64 x 64: and for TileS (two workgroups a CU)
typedef RowTile<4, 4, 2, 2, 2> TileW;       // 128 x 128, 4 waves: 64 x 64 to a wave, for epilogues that want that
// few queries, whose rows' loads are what counts: about 100 KB of them on the way in a workgroup that has a CU to
// itself (two workgroups with half of that each: the same time).  1M x 128 fp32 and one query: 94 us, 5.5 TB/s, with the
// norms; 131,071 x 1024 bf16 and 16 queries: 46 us, 5.8 TB/s.
typedef RowTile<4, 1, 4, 1, 4> TileF1;      // 256 x 16
typedef RowTile<4, 2, 4, 1, 4> TileF2;      // 256 x 32
typedef RowTile<4, 4, 4, 1, 3> TileF4;      // 256 x 64
static inline int64_t rowprod_tiles(int64_t p, int64_t q, int side) { return ((p + side - 1) / side) * ((q + side - 1) / side); }
// The size by the workgroups there are for 256 CUs, measured on either side of both limits (rows x K x columns, us, large / middle /
// small, bf16; fp32 in three pieces): 8,191 x 1000 x 2048, 256 tiles of 256, 50 / 68 / 84; 170 / 189 / 231.  4,096 x 1000 x 2048, 128 of
// them, 46 / 42 / 50; 92 / 100 / 126 (three pieces' large tile is half that size: 256 x 128 would still do).  2,999 x 1000 x 960, 192
// tiles of 128, 42 / 27 / 28; 83 / 55 / 62.  1,024 x 1000 x 1024, 64 of them, 37 / 21 / 16; 79 / 51 / 34.
static inline int rowprod_size(int64_t p, int64_t q, int splits = 1)
{
    return rowprod_tiles(p, q, 256) * splits >= 200 ? 2 : rowprod_tiles(p, q, 128) * splits >= 160 ? 1 : 0;
}

template <class T>
struct RowAcc {
    v4f v[T::PT][T::QT];
    float nrm[T::PT];               // ROW_NORM: this lane's part of the squared norm of row 16 i + (lane & 15) of P
};

// with adapters; fp32 rows; norms wanted; three pieces together; two pieces of Q together
enum { ROW_ADAPT = 1, ROW_F32 = 2, ROW_NORM = 4, ROW_THREES = 8, ROW_TWOS = 16 };
// bytes of one LDS buffer, loads that every wave makes for it
template <class T, int FLAGS>
struct RowStep {
    static constexpr bool THREES = FLAGS & ROW_THREES, TWOS = FLAGS & ROW_TWOS;
    static constexpr int PL = TWOS ? T::LP / 2 : T::LP, PB = TWOS ? 64 : 128;             // loads of P, bytes of a row of P
    static constexpr int BYTES = THREES ? T::BYTES * 3 / 2 : T::BP * PB + T::BQ * 128, LOADS = THREES ? T::LEAST * 3 / 2 : T::LEAST - T::LP + PL;
    static constexpr int LP2 = THREES ? T::LP / 2 : 1, LQ2 = THREES ? T::LQ / 2 : 1;      // loads of third pieces
    static constexpr int WAVES = T::NT == 256 && T::ST * BYTES > 80 * 1024 ? 1 : 2;       // per SIMD: four waves that have a CU to themselves
    static_assert(!THREES || (!T::SOME_Q && T::LP % 2 == 0 && T::LQ % 2 == 0), "");
    static_assert(!TWOS || (!THREES && T::LP % 2 == 0), "");
};

// Threes in LDS: pieces 0 and 1 of a row as any row's 128 bytes, then the third pieces (`at` bytes into the row's), two rows to
// 128 bytes: slot s of pair r holds chunk s ^ (r & 3) of the two.
template <class T, int L>
static __device__ __forceinline__ void rowprod_thirds(int64_t r0, int64_t rows, int64_t ld, int tid, uint32_t (&o)[L], int64_t (&row)[L], int at = 128)
{
    const uint32_t last = (uint32_t)(rows - 1 - r0 < 0x7FFFFFFF ? rows - 1 - r0 : 0x7FFFFFFF);
#pragma unroll
    for (int i = 0; i < L; i++) {
        const uint32_t pair = i * (T::NT / 8) + (tid >> 3), x = (tid & 7) ^ (pair & 3), r = 2 * pair + (x >> 2);
        row[i] = r0 + r;
        o[i] = (r < last ? r : last) * (uint32_t)(ld * 2) + at + (x & 3) * 16;
    }
}

// one step's 16-byte chunks of both operands, straight into LDS: a row's place is a 32-bit offset from an
// address that the workgroup shares
template <class T, int PL>
static __device__ __forceinline__ void rowprod_fetch(char *buf, const char *pb, const uint32_t (&po)[PL], const char *qb,
                                                     const uint32_t (&qo)[T::LQ], int wave)
{
#pragma unroll
    for (int i = 0; i < PL; i++)
        __builtin_amdgcn_global_load_lds((global_void *)(pb + po[i]), (lds_void *)(buf + (i * T::NT + wave * 64) * 16), 16, 0, 0);
    if (!T::SOME_Q || wave * 64 < T::BQ * 8)                          // uniform
#pragma unroll
        for (int i = 0; i < T::LQ; i++)
            __builtin_amdgcn_global_load_lds((global_void *)(qb + qo[i]), (lds_void *)(buf + (PL * T::NT + i * T::NT + wave * 64) * 16), 16,
                                             0, 0);
}

template <class T, int L>
static __device__ __forceinline__ void rowprod_fetch_thirds(char *buf, const char *base, const uint32_t (&o)[L], int wave)
{
#pragma unroll
    for (int i = 0; i < L; i++)
        __builtin_amdgcn_global_load_lds((global_void *)(base + o[i]), (lds_void *)(buf + (i * T::NT + wave * 64) * 16), 16, 0, 0);
}

// All but the last N loads into LDS of this wave have landed, then every wave's; and every wave has read what it
// reads.  (The compiler's own barrier would wait for all of the loads.)
template <int N>
static __device__ __forceinline__ void rowprod_landed()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// One step's products.  The operand that more products follow each other with stays: the longer side's tiles
// are the inner loop.  `fetch`, the next step's loads, is issued in the middle of the first half's products,
// where the operand reads of that half are out of its way.  128,000 x 4096 x 1024 at 256 x 256: 854 us so, 859
// with the loads first, 922 with the loops the other way round; with both halves' operands read first, or
// products and reads interleaved by hand, 960 to 1,025.
template <class T, int FLAGS, class F>
static __device__ __forceinline__ void rowprod_step(const char *buf, int wp, int wq, int lane, RowAcc<T> &acc, const F &fetch)
{
#pragma unroll
    for (int kk = 0; kk < 2; kk++) {
        const int slot = ((kk * 4 + (lane >> 4)) ^ (lane & 7)) * 16 + (lane & 15) * 128;
        v4u a[T::PT], b[T::QT];
#pragma unroll
        for (int i = 0; i < T::PT; i++) a[i] = *(const v4u *)(buf + (wp * T::PT + i) * 2048 + slot);
#pragma unroll
        for (int j = 0; j < T::QT; j++) b[j] = *(const v4u *)(buf + T::BP * 128 + (wq * T::QT + j) * 2048 + slot);
#pragma unroll
        for (int e = 0; e < (FLAGS & ROW_F32 ? 4 : 1); e++)
#pragma unroll
            for (int x = 0; x < T::PT * T::QT; x++) {
                if (kk == 0 && e == 0 && x == T::PT * T::QT / 2) {
                    __builtin_amdgcn_sched_barrier(0);
                    fetch();
                    __builtin_amdgcn_sched_barrier(0);
                }
                const int i = T::PT >= T::QT ? x % T::PT : x / T::QT, j = T::PT >= T::QT ? x / T::PT : x % T::QT;
                if constexpr (FLAGS & ROW_F32)
                    acc.v[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i][e]), __uint_as_float(b[j][e]), acc.v[i][j], 0, 0, 0);
                else
                    acc.v[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a[i]), __builtin_bit_cast(v8bf, b[j]),
                                                                          acc.v[i][j], 0, 0, 0);
            }
        if constexpr (FLAGS & ROW_NORM)
#pragma unroll
            for (int i = 0; i < T::PT; i++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    if constexpr (FLAGS & ROW_F32) {
                        acc.nrm[i] = fmaf(__uint_as_float(a[i][e]), __uint_as_float(a[i][e]), acc.nrm[i]);
                    } else {
                        const uint32_t word = a[i][e];                // (a cast of a vector's element as it stands takes the vector's first)
                        const v2bf x = __builtin_bit_cast(v2bf, word);
                        acc.nrm[i] = __builtin_amdgcn_fdot2_f32_bf16(x, x, acc.nrm[i], false);
                    }
                }
    }
}

// One step of threes: 32 values.  Fragments are read as they are needed, the largest products first.
template <class T, class F>
static __device__ __forceinline__ void rowprod_step_threes(const char *buf, int wp, int wq, int lane, RowAcc<T> &acc, v4f (&low)[T::PT][T::QT],
                                                           const F &fetch)
{
    const int r = lane & 15, h = lane >> 4;
    const int slot = (h ^ (r & 7)) * 16 + r * 128, slot1 = ((4 + h) ^ (r & 7)) * 16 + r * 128;
    const int slot2 = ((4 * (r & 1) + h) ^ ((r >> 1) & 3)) * 16 + (r >> 1) * 128;
    const char *pa = buf + wp * T::PT * 2048, *qa = buf + T::BP * 128 + wq * T::QT * 2048;
    const char *pc = buf + T::BYTES + wp * T::PT * 1024, *qc = buf + T::BYTES + T::BP * 64 + wq * T::QT * 1024;
    v8bf a0[T::PT], a1[T::PT], b0[T::QT], b1[T::QT];
    const auto mul = [&](const v8bf (&a)[T::PT], const v8bf (&b)[T::QT], v4f (&c)[T::PT][T::QT]) {
#pragma unroll
        for (int i = 0; i < T::PT; i++)
#pragma unroll
            for (int j = 0; j < T::QT; j++) c[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], c[i][j], 0, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < T::PT; i++) a0[i] = *(const v8bf *)(pa + i * 2048 + slot);
#pragma unroll
    for (int j = 0; j < T::QT; j++) b0[j] = *(const v8bf *)(qa + j * 2048 + slot);
#pragma unroll
    for (int j = 0; j < T::QT; j++) b1[j] = *(const v8bf *)(qa + j * 2048 + slot1);
#pragma unroll
    for (int i = 0; i < T::PT; i++) a1[i] = *(const v8bf *)(pa + i * 2048 + slot1);
    mul(a0, b0, acc.v);
    __builtin_amdgcn_sched_barrier(0);
    fetch();
    __builtin_amdgcn_sched_barrier(0);
    mul(a0, b1, low);
    mul(a1, b1, low);
#pragma unroll
    for (int j = 0; j < T::QT; j++) b1[j] = *(const v8bf *)(qc + j * 1024 + slot2);      // the third pieces
    mul(a1, b0, low);
#pragma unroll
    for (int i = 0; i < T::PT; i++) a1[i] = *(const v8bf *)(pc + i * 1024 + slot2);
    mul(a0, b1, low);
    mul(a1, b0, low);
}

// One step of twos: 32 values, of P once and of Q in both pieces, each value of P against two of Q.
template <class T, class F>
static __device__ __forceinline__ void rowprod_step_twos(const char *buf, int wp, int wq, int lane, RowAcc<T> &acc, const F &fetch)
{
    const int r = lane & 15, h = lane >> 4;
    const char *pa = buf + wp * T::PT * 1024 + ((4 * (r & 1) + h) ^ ((r >> 1) & 3)) * 16 + (r >> 1) * 128;
    const char *qa = buf + T::BP * 64 + wq * T::QT * 2048 + r * 128;
    v8bf a[T::PT], b[T::QT];
#pragma unroll
    for (int i = 0; i < T::PT; i++) a[i] = *(const v8bf *)(pa + i * 1024);
#pragma unroll
    for (int u = 1; u >= 0; u--) {                                    // (the smaller products first)
#pragma unroll
        for (int j = 0; j < T::QT; j++) b[j] = *(const v8bf *)(qa + j * 2048 + ((4 * u + h) ^ (r & 7)) * 16);
#pragma unroll
        for (int x = 0; x < T::PT * T::QT; x++) {
            if (u == 1 && x == T::PT * T::QT / 2) {
                __builtin_amdgcn_sched_barrier(0);
                fetch();
                __builtin_amdgcn_sched_barrier(0);
            }
            const int i = T::PT >= T::QT ? x % T::PT : x / T::QT, j = T::PT >= T::QT ? x / T::PT : x % T::QT;
            acc.v[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], acc.v[i][j], 0, 0, 0);
        }
    }
}

// A workgroup's q tile and run of p tiles.  Workgroups are handed out round robin over the eight XCDs, each with
// its own L2 cache: one XCD takes consecutive ids, and ids go over a band of q tiles, then to the next run, so that
// what runs on an XCD at a time is about a square of tiles, whose rows its cache fetches once.
static __device__ __forceinline__ bool rowprod_tile(const RowProd &a, uint32_t block, int &run, int &qt, int &split)
{
    const uint32_t all = (uint32_t)(a.pruns * a.qtiles), total = all * a.splits, per = (total + 7) / 8;
    const uint32_t id = (block % 8) * per + block / 8;
    if (block / 8 >= per || id >= total) return false;
    split = (int)(id / all);
    const uint32_t in = id % all, b = in / (uint32_t)(a.band * a.pruns), rest = in % (uint32_t)(a.band * a.pruns);
    const uint32_t h = min((uint32_t)a.band, a.qtiles - b * a.band);
    qt = (int)(b * a.band + rest % h);
    run = (int)(rest / h);
    return true;
}
static inline unsigned rowprod_grid(const RowProd &a)
{
    const uint32_t total = (uint32_t)(a.pruns * a.qtiles * a.splits);
    return (total + 7) / 8 * 8;
}

// offsets of a tile's rows from its first one, `ld` elements apart; rows beyond the last of `rows` read it
// (they are computed, not stored)
template <class T, int L>
static __device__ __forceinline__ void rowprod_rows(int64_t r0, int64_t rows, int64_t ld, int tid, uint32_t (&o)[L])
{
    const uint32_t chunk = ((tid & 7) ^ ((tid >> 3) & 7)) * 16, last = (uint32_t)(rows - 1 - r0 < 0x7FFFFFFF ? rows - 1 - r0 : 0x7FFFFFFF);
#pragma unroll
    for (int i = 0; i < L; i++) {
        const uint32_t r = i * (T::NT / 8) + (tid >> 3);              // (NT / 8 is a multiple of 8: chunk is the same for every load)
        o[i] = (r < last ? r : last) * (uint32_t)(ld * 2) + chunk;
    }
}

// A workgroup takes a q tile and a run of p tiles one after the other; the loads of a tile's first step
// are under way while the tile before it is finished.  The epilogue keeps a state of its own over the
// run: epi.begin(state, q0, lane), epi.tile(state, acc, p0, q0, lane, split) per tile, epi.end(state, run, wp,
// q0, lane): lane l holds, for its tiles (i, j), rows q0 + 16 j + (l & 15) and columns p0 + 16 i +
// 4 (l >> 4) + 0..3.
template <class T, class Epi, int FLAGS>
static __device__ __forceinline__ void rowprod_run_tiles(const RowProd &a, const Epi &epi, uint32_t block)
{
    constexpr bool ADAPT = FLAGS & ROW_ADAPT, THREES = FLAGS & ROW_THREES, TWOS = FLAGS & ROW_TWOS;
    static_assert(!TWOS || !ADAPT, "");
    constexpr int BYTES = RowStep<T, FLAGS>::BYTES, LP2 = RowStep<T, FLAGS>::LP2, LQ2 = RowStep<T, FLAGS>::LQ2;
    constexpr int STEP = THREES ? 192 : ROWPROD_K * 2, PSTEP = TWOS ? 64 : STEP;          // bytes of a row per step, of P's
    constexpr int PL = RowStep<T, FLAGS>::PL;
    extern __shared__ __align__(16) char rowprod_lds[];
    int run, qt, split;
    if (!rowprod_tile(a, block, run, qt, split)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = wave % T::WP, wq = wave / T::WP;
    const int t0 = run * a.prun, t1 = min(t0 + a.prun, a.ptiles);
    const int64_t q0 = (int64_t)qt * T::BQ, qw = q0 + wq * (16 * T::QT);

    // what is fetched, a step at a time, ahead of what is multiplied: the run's tiles one after the other, then (the run is
    // one tile) the adapters of the tile's rows
    uint32_t po[PL], qo[T::LQ];
    const auto place_p = [&](int tile) {
        if constexpr (TWOS) {
            int64_t row[PL];
            rowprod_thirds<T>((int64_t)tile * T::BP, a.P.rows, a.P.ld, tid, po, row, 0);
        } else {
            rowprod_rows<T>((int64_t)tile * T::BP, a.P.rows, a.P.ld, tid, po);
        }
    };
    place_p(t0);
    const char *pb = (const char *)(a.P.p + (int64_t)t0 * T::BP * a.P.ld), *qb = (const char *)a.Q.p;
    const uint32_t chunk = ((tid & 7) ^ ((tid >> 3) & 7)) * 16;
    if (a.Q.perm) {
#pragma unroll
        for (int i = 0; i < T::LQ; i++) {
            const int64_t r = q0 + i * (T::NT / 8) + (tid >> 3);
            qo[i] = (uint32_t)a.Q.perm[r < a.Q.rows ? r : a.Q.rows - 1] * (uint32_t)(a.Q.ld * 2) + chunk;
        }
    } else {
        rowprod_rows<T>(q0, a.Q.rows, a.Q.ld, tid, qo);
        qb += q0 * a.Q.ld * 2;
    }
    uint32_t po3[LP2], qo3[LQ2];                                      // of third pieces
    int64_t prow3[LP2], qrow3[LQ2];
    if constexpr (THREES) {
        rowprod_thirds<T>((int64_t)t0 * T::BP, a.P.rows, a.P.ld, tid, po3, prow3);
        rowprod_thirds<T>(q0, a.Q.rows, a.Q.ld, tid, qo3, qrow3);
        if (a.Q.perm)
#pragma unroll
            for (int i = 0; i < LQ2; i++) {
                const uint32_t place = (tid & 7) ^ ((tid >> 3) & 3);  // (the pair's, as in rowprod_thirds)
                qo3[i] = (uint32_t)a.Q.perm[qrow3[i] < a.Q.rows ? qrow3[i] : a.Q.rows - 1] * (uint32_t)(a.Q.ld * 2) + 128 + (place & 3) * 16;
            }
    }
    uint32_t sp = a.sp, sq = a.sq;
    int nseg = a.nseg;
    if (a.Q.pieces_there) {
        const uint32_t there = 1u | (a.Q.pieces_there[0] ? 2u : 0u) | (a.Q.pieces_there[1] ? 4u : 0u);
        sp = sq = 0;
        nseg = 0;
        for (int i = 0; i < a.nseg; i++) {
            const uint32_t u = (a.sp >> (4 * i)) & 15, v = (a.sq >> (4 * i)) & 15;
            if (!((there >> v) & 1u)) continue;
            sp |= u << (4 * nseg);
            sq |= v << (4 * nseg);
            nseg++;
        }
    }
    const int steps = nseg * a.ksteps;
    const int s0 = (int)((int64_t)steps * split / a.splits), s1 = (int)((int64_t)steps * (split + 1) / a.splits);
    const int seg0 = s0 / a.ksteps, k0 = s0 % a.ksteps;

    int f_tile = t0, f_step = s0, seg = seg0, k = k0;                 // the next step to fetch
    // of the adapters: the one being fetched, its next values, where its rows end; -1: none left
    int f_ad = -1, f_k = 0;
    int64_t f_end = q0;
    int32_t own[ADAPT ? T::LQ : 1], own3[ADAPT ? LQ2 : 1];            // adapters of this thread's rows
    const int64_t qend = q0 + T::BQ < a.Q.rows ? q0 + T::BQ : a.Q.rows;
    if constexpr (ADAPT) {
#pragma unroll
        for (int i = 0; i < T::LQ; i++) {
            const int64_t r = q0 + i * (T::NT / 8) + (tid >> 3);
            own[i] = a.ad.of_row[r < a.Q.rows ? r : a.Q.rows - 1];
        }
        if constexpr (THREES)
#pragma unroll
            for (int i = 0; i < LQ2; i++) own3[i] = a.ad.of_row[qrow3[i] < a.Q.rows ? qrow3[i] : a.Q.rows - 1];
        f_ad = a.ad.of_row[q0];                                       // (rows without an adapter are the last)
        f_end = f_ad >= 0 ? a.ad.end[f_ad] : qend;
    }
    char *f_buf = rowprod_lds;
    int fetched = 0, total = 0x7FFFFFFF;                              // steps so far; all there are, once that is known
    // (when nothing is left the last step's addresses are read again: a wave always has as many loads on the way as the
    // wait counts)
    auto fetch = [&]() {
        bool base = true;
        if constexpr (ADAPT) base = f_tile < t1;
        if (base) {
            const int64_t ps = (sp >> (4 * seg)) & 15, qs = (sq >> (4 * seg)) & 15;
            const char *pk = pb + ps * a.P.piece * 2 + (int64_t)k * PSTEP, *qk = qb + qs * a.Q.piece * 2 + (int64_t)k * STEP;
            rowprod_fetch<T>(f_buf, pk, po, qk, qo, wave);
            if constexpr (THREES) {
                rowprod_fetch_thirds<T>(f_buf + T::BYTES, pk, po3, wave);
                rowprod_fetch_thirds<T>(f_buf + T::BYTES + T::BP * 64, qk, qo3, wave);
            }
            if (f_tile < t1) {
                fetched++;
                if (++f_step < s1) {
                    if (++k == a.ksteps) { k = 0; seg++; }
                } else {
                    f_tile++;
                    if (f_tile < t1) {
                        f_step = s0; seg = seg0; k = k0;
                        pb += (int64_t)T::BP * a.P.ld * 2;
                        if (f_tile + 1 == a.ptiles) {
                            place_p(f_tile);
                            if constexpr (THREES) rowprod_thirds<T>((int64_t)f_tile * T::BP, a.P.rows, a.P.ld, tid, po3, prow3);
                        }
                    } else if (!ADAPT || f_ad < 0) {
                        total = fetched;
                    }
                }
            }
        } else if constexpr (ADAPT) {
            const int64_t p0 = (int64_t)t0 * T::BP;
            const int ad = f_ad < 0 ? 0 : f_ad;
            uint32_t ao[T::LP], uo[T::LQ];
            rowprod_rows<T>(p0, a.P.rows, a.ad.kpad, tid, ao);
            rowprod_rows<T>(q0, a.Q.rows, a.ad.kpad, tid, uo);
            const char *bb = (const char *)(a.ad.b + ((int64_t)ad * a.P.rows + p0) * a.ad.kpad + f_k), *ub = (const char *)(a.ad.u + q0 * a.ad.kpad + f_k);
#pragma unroll
            for (int i = 0; i < T::LP; i++)
                __builtin_amdgcn_global_load_lds((global_void *)(bb + ao[i]), (lds_void *)(f_buf + (i * T::NT + wave * 64) * 16), 16, 0, 0);
#pragma unroll
            for (int i = 0; i < T::LQ; i++) {
                const char *src = own[i] == ad ? ub + uo[i] : (const char *)a.ad.zero;
                __builtin_amdgcn_global_load_lds((global_void *)src, (lds_void *)(f_buf + T::BP * 128 + (i * T::NT + wave * 64) * 16), 16, 0, 0);
            }
            if constexpr (THREES) {
                uint32_t ao3[LP2], uo3[LQ2];
                rowprod_thirds<T>(p0, a.P.rows, a.ad.kpad, tid, ao3, prow3);
                rowprod_thirds<T>(q0, a.Q.rows, a.ad.kpad, tid, uo3, qrow3);
                rowprod_fetch_thirds<T>(f_buf + T::BYTES, bb, ao3, wave);
#pragma unroll
                for (int i = 0; i < LQ2; i++) {
                    const char *src = own3[i] == ad ? ub + uo3[i] : (const char *)a.ad.zero;
                    __builtin_amdgcn_global_load_lds((global_void *)src, (lds_void *)(f_buf + T::BYTES + T::BP * 64 + (i * T::NT + wave * 64) * 16), 16,
                                                     0, 0);
                }
            }
            if (f_ad >= 0) {
                fetched++;
                f_k += STEP / 2;
                if (f_k == a.ad.kpad) {
                    f_k = 0;
                    f_ad = f_end < qend ? a.ad.of_row[f_end] : -1;
                    if (f_ad >= 0) f_end = a.ad.end[f_ad];
                    else total = fetched;
                }
            }
        }
        f_buf = f_buf == rowprod_lds + (T::ST - 1) * BYTES ? rowprod_lds : f_buf + BYTES;
    };
    for (int i = 0; i < T::ST - 1; i++) fetch();
    typename Epi::template State<T> state;
    epi.begin(state, qw, lane);
    const char *buf = rowprod_lds;
    int done = 0;
    for (int t = t0; t < t1; t++) {
        RowAcc<T> acc;
#pragma unroll
        for (int i = 0; i < T::PT; i++)
#pragma unroll
            for (int j = 0; j < T::QT; j++) acc.v[i][j] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < T::PT; i++) acc.nrm[i] = 0.0f;
        v4f low[T::PT][T::QT];
        if constexpr (THREES)
#pragma unroll
            for (int i = 0; i < T::PT; i++)
#pragma unroll
                for (int j = 0; j < T::QT; j++) low[i][j] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
        // (a run of several tiles: a tile's steps; else all that is fetched)
        const int stop = done + (s1 - s0);
        while (ADAPT ? done < total : done < stop) {
            // (this also says that every wave is past the step before, whose buffer the next fetch writes)
            rowprod_landed<(T::ST - 2) * RowStep<T, FLAGS>::LOADS>();
            if constexpr (THREES) rowprod_step_threes<T>(buf, wp, wq, lane, acc, low, fetch);
            else if constexpr (TWOS) rowprod_step_twos<T>(buf, wp, wq, lane, acc, fetch);
            else rowprod_step<T, FLAGS>(buf, wp, wq, lane, acc, fetch);
            buf = buf == rowprod_lds + (T::ST - 1) * BYTES ? rowprod_lds : buf + BYTES;
            done++;
        }
        if constexpr (THREES)
#pragma unroll
            for (int i = 0; i < T::PT; i++)
#pragma unroll
                for (int j = 0; j < T::QT; j++) acc.v[i][j] += low[i][j];
        epi.tile(state, acc, (int64_t)t * T::BP + wp * (16 * T::PT), qw, lane, split);
    }
    epi.end(state, run, wp, qw, lane);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                  // (LDS is given away when the workgroup ends)
}

template <class T, class Epi, int FLAGS>
__global__ __launch_bounds__(T::NT, (RowStep<T, FLAGS>::WAVES)) void rowprod_kernel(RowProd a, Epi epi)
{
    rowprod_run_tiles<T, Epi, FLAGS>(a, epi, blockIdx.x);
}

// two products that do not wait for each other, of few workgroups each; `first`: the first one's
template <class Epi>
struct RowProdPair {
    RowProd a[2];
    Epi epi[2];
    uint32_t first;
};
template <class T, class Epi, int FLAGS>
__global__ __launch_bounds__(T::NT, (RowStep<T, FLAGS>::WAVES)) void rowprod_pair_kernel(RowProdPair<Epi> p)
{
    const int which = blockIdx.x >= p.first;
    rowprod_run_tiles<T, Epi, FLAGS>(p.a[which], p.epi[which], which ? blockIdx.x - p.first : blockIdx.x);
}

// p tiles that a workgroup takes one after the other, at most `most`: what the last round of workgroups leaves
// idle against the start of each (about `start` tiles' time), with room for `slots` workgroups at once
static inline int rowprod_run(int64_t ptiles, int64_t qtiles, int slots, double start, int most)
{
    int best = 1;
    double least = 1e300;
    for (int r = 1; r <= most && r <= ptiles; r++) {
        const int64_t wgs = (ptiles + r - 1) / r * qtiles;
        const double t = (double)((wgs + slots - 1) / slots) * (r + start);
        if (t < least) { least = t; best = r; }
    }
    return best;
}

// the launch's part of a product; `prun`: p tiles that a workgroup takes one after the other
template <class T, int FLAGS>
static void rowprod_plan(RowProd &a, int prun)
{
    a.ptiles = (int)((a.P.rows + T::BP - 1) / T::BP);
    a.qtiles = (int)((a.Q.rows + T::BQ - 1) / T::BQ);
    a.prun = prun;
    a.pruns = (a.ptiles + prun - 1) / prun;
    if (a.splits < 1) a.splits = 1;
    // the square: of the workgroups that an XCD has at a time, 32 or (small tiles: two a CU) 64
    const int64_t total = (int64_t)a.pruns * a.qtiles;
    const int64_t at_once = std::min<int64_t>((total * a.splits + 7) / 8, T::ST * RowStep<T, FLAGS>::BYTES > 80 * 1024 ? 32 : 64);
    double least = 1e300;
    for (int bands = 1; bands <= a.qtiles; bands++) {
        const int h = (a.qtiles + bands - 1) / bands;
        const double rows = (double)h * T::BQ + (double)at_once / h * T::BP;
        if (rows < least) { least = rows; a.band = h; }
    }
}

template <class T, int FLAGS = 0, class Epi>
static int rowprod_launch(RowProd &a, const Epi &epi, hipStream_t s, int prun = 1)
{
    rowprod_plan<T, FLAGS>(a, prun);
    constexpr int lds = T::ST * RowStep<T, FLAGS>::BYTES;
    auto kern = rowprod_kernel<T, Epi, FLAGS>;
    RAIRS_HIP(hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kern, dim3(rowprod_grid(a)), dim3(T::NT), lds, s, a, epi);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

template <class T, int FLAGS = 0, class Epi>
static int rowprod_launch_pair(const RowProd &a, const Epi &ea, const RowProd &b, const Epi &eb, hipStream_t s)
{
    RowProdPair<Epi> p = {{a, b}, {ea, eb}, 0};
    rowprod_plan<T, FLAGS>(p.a[0], 1);
    rowprod_plan<T, FLAGS>(p.a[1], 1);
    p.first = rowprod_grid(p.a[0]);
    constexpr int lds = T::ST * RowStep<T, FLAGS>::BYTES;
    auto kern = rowprod_pair_kernel<T, Epi, FLAGS>;
    RAIRS_HIP(hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kern, dim3(p.first + rowprod_grid(p.a[1])), dim3(T::NT), lds, s, p);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

// the same with the tile chosen by rowprod_size
template <int FLAGS = 0, class Epi>
static int rowprod_launch_any(RowProd &a, const Epi &epi, hipStream_t s)
{
    const int size = rowprod_size(a.P.rows, a.Q.rows, a.splits > 1 ? a.splits : 1);
    if constexpr (FLAGS & ROW_THREES)
        return size == 2 ? rowprod_launch<TileT, FLAGS>(a, epi, s) : size == 1 ? rowprod_launch<TileM, FLAGS>(a, epi, s) : rowprod_launch<TileU, FLAGS>(a, epi, s);
    else
        return size == 2 ? rowprod_launch<TileL, FLAGS>(a, epi, s) : size == 1 ? rowprod_launch<TileM, FLAGS>(a, epi, s) : rowprod_launch<TileS, FLAGS>(a, epi, s);
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
    struct State {
        int64_t row[T::QT];         // of the output, -1: none
    };
    template <class T>
    __device__ __forceinline__ void begin(State<T> &st, int64_t q0, int lane) const
    {
#pragma unroll
        for (int j = 0; j < T::QT; j++) {
            const int64_t q = q0 + 16 * j + (lane & 15);
            st.row[j] = q >= nq ? -1 : perm ? perm[q] : q;
        }
    }
    template <class T>
    __device__ __forceinline__ void end(State<T> &, int, int, int64_t, int) const {}
    template <class T>
    __device__ __forceinline__ void tile(State<T> &st, const RowAcc<T> &acc, int64_t p0, int64_t q0, int lane, int split) const
    {
        // four values at once where every row starts on a multiple of four elements
        const bool four = ld % 4 == 0 && (bf16_out ? ((uintptr_t)out & 7) == 0 : ((uintptr_t)out & 15) == 0) && split_stride % 4 == 0;
#pragma unroll
        for (int j = 0; j < T::QT; j++) {
            if (st.row[j] < 0) continue;
            const int64_t row = st.row[j] * ld + split * split_stride;
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
