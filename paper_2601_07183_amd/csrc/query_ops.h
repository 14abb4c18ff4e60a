// The operators on the query side of an index: internal declarations of their translation units.
#pragma once
#include "rowprod.h"

static inline int dtype_width(int dtype) { return dtype == RAIRS_F32 ? 4 : dtype == RAIRS_BF16 ? 2 : 1; }
static inline int dtype_pieces(int dtype) { return dtype == RAIRS_F32 ? 3 : 1; }
static inline int64_t pad_to(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Hands out 256-byte aligned parts of a workspace; without one it only counts.
struct Carve {
    char *base;
    size_t used;
    explicit Carve(void *p) : base((char *)p), used(0) {}
    template <class X>
    X *take(int64_t count)
    {
        X *p = base ? (X *)(base + used) : nullptr;
        used += ((size_t)count * sizeof(X) + 255) / 256 * 256;
        return p;
    }
};

// Where packed values go: value k of piece u of row r at r * ld + k / 32 * block + u * piece + k % 32
struct PackLayout {
    int64_t ld, piece;
    int block;
};
// pieces one after the other, or (threes) together in every 32 values; kpad a multiple of 32
static inline PackLayout pack_layout(int64_t rows, int64_t kpad, bool threes)
{
    return threes ? PackLayout{3 * kpad, 32, 96} : PackLayout{kpad, rows * kpad, 32};
}
// two pieces together in every 32 values
static inline PackLayout pack_twos(int64_t kpad) { return PackLayout{2 * kpad, 32, 64}; }
// rows of a matrix as bf16 pieces with rows of kpad values, zero from `cols` on (and where live says so)
// (perm: row r is src's row perm[r]; flags[i], if given: cleared if `clear`, else set if piece i + 1 of any value is
// not zero)
int rairs_launch_pack_rows(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, const int32_t *perm, __bf16 *dst,
                           int64_t kpad, PackLayout to, hipStream_t s, uint32_t *flags, bool clear);
// the same, transposed: dst[c][place of r] = src[r][c], zero for r in [rows, rpad) and where live says so; rows keep
// their places (order 0), or change them among their 64 as the gradient of the logits does (rowpack.h)
enum { ORDER_SAME = 0, ORDER_TABLE = 1, ORDER_QUERIES = 2 };
int rairs_launch_pack_cols(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, const uint32_t *live, int order, __bf16 *dst,
                           int64_t rpad, PackLayout to, hipStream_t s);

// A matrix as an operand of rowprod: bf16 rows that lie right already are taken where they are, others
// are packed into `room` (pack_room elements of it).  With a permutation (the product's row r is row
// perm[r]) rows are packed in its order, or, if a 32-bit offset reaches them all, taken through it.
static inline bool rows_lie_right(const void *p, int dtype, int64_t ld, int64_t cols)
{
    return dtype == RAIRS_BF16 && (uintptr_t)p % 16 == 0 && ld % 8 == 0 && ld < (1 << 22) && cols % ROWPROD_K == 0;
}
// fp32 rows that lie right for the fp32 instruction: whole steps of 32 values
static inline bool f32_lies_right(const void *p, int dtype, int64_t ld, int64_t cols)
{
    return dtype == RAIRS_F32 && (uintptr_t)p % 16 == 0 && ld % 4 == 0 && ld < (1 << 21) && cols % (ROWPROD_K / 2) == 0;
}
static inline RowOperand f32_operand(const void *p, int64_t ld, int64_t rows) { return RowOperand{(const __bf16 *)p, 2 * ld, 0, rows, nullptr, nullptr}; }
static inline int64_t pack_room(int dtype, int64_t rows, int64_t cols) { return rows * pad_to(cols, ROWPROD_K) * dtype_pieces(dtype); }
// (threes: both operands of the product are fp32)
int rairs_operand(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, const int32_t *perm, bool threes, __bf16 *room,
                  RowOperand &out, hipStream_t s, uint32_t *flags = nullptr, bool clear = false);
// Several matrices laid out by one launch.
struct PackJob {
    const void *src;
    __bf16 *dst;
    int dtype, turned;              // turned: as rairs_launch_pack_cols does, else as rairs_launch_pack_rows
    int64_t ld, rows, cols, pad;    // pad: values of a row of dst
    PackLayout to;
    int order;
    const uint32_t *live;
    // turned, if targets are given: rows that pass no gradient (their target outside the mask `live`, [ld_live] words a row,
    // or dlogp 0, and dentropy 0) are zero instead
    const int64_t *targets;
    int64_t ld_live, V;
    const float *dlogp, *dentropy;
    int vec;                        // (set by the launch, as is what follows)
    unsigned blocks;
};
#define PACK_JOBS 4
struct PackJobs {
    PackJob job[PACK_JOBS];
    int n;
};
int rairs_launch_pack(PackJobs &jobs, hipStream_t s);
// an operand as rairs_operand makes it, its packing (if it needs any) left to `jobs`
void rairs_operand_job(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, bool threes, __bf16 *room, RowOperand &out, PackJobs &jobs);
// the products of an np-piece operand with an nq-piece one over kpad values
static inline void rowprod_sums(RowProd &rp, int np, int nq, int64_t kpad)
{
    const bool threes = np == 3 && nq == 3;
    rowprod_pieces(rp, threes ? 1 : np, threes ? 1 : nq);
    rp.ksteps = (int)(kpad / (threes ? 32 : ROWPROD_K));
}

struct LogprobArgs {
    const void *q, *table;
    int qtype, ttype;
    int64_t ldq, ldt, n, V;
    int d;
    float scale;
    const uint32_t *live;
    int64_t ld_live;
    const int64_t *targets;
    // forward
    float *logp, *lse, *entropy;
    int top;
    int64_t *top_ids;
    float *top_logp;
    // backward
    const float *lse_in, *entropy_in, *dlogp, *dentropy;
    void *dq, *dtable;
    int64_t lddq, lddt;
};
// (with ws null both only count the bytes they need)
int rairs_run_logprob(const LogprobArgs &a, void *ws, size_t *bytes, hipStream_t s);
int rairs_run_logprob_backward(const LogprobArgs &a, void *ws, size_t *bytes, hipStream_t s);

int rairs_launch_clear_rows(void *out, int64_t n, int64_t cols, int64_t ld, int dtype, hipStream_t s);

struct ProjectArgs {
    rairs_projection_t p;
    const void *x, *dy;
    int64_t ldx, lddy, n;
    const int32_t *adapter;
    void *y, *dx, *da, *db;
    int64_t ldy, lddx;
    int ytype;
};
int rairs_run_project(const ProjectArgs &a, void *ws, size_t *bytes, hipStream_t s);
int rairs_run_project_backward(const ProjectArgs &a, void *ws, size_t *bytes, hipStream_t s);
