// The steps of laying rows out for the products of rowprod.h, shared by the kernels that do it.
#pragma once
#include "query_ops.h"

// eight consecutive values of a row, zero from `cols` on; `vec`: rows are 16-byte aligned (8 for bytes)
template <class S>
static __device__ __forceinline__ void load8(const S *row, int64_t i0, int64_t cols, bool vec, float (&x)[8])
{
    if (vec && i0 + 8 <= cols) {
        struct __align__(sizeof(S) == 1 ? 8 : 16) V { S e[8]; };
        const V v = *(const V *)(row + i0);
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = (float)v.e[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = i0 + e < cols ? (float)row[i0 + e] : 0.0f;
    }
}

// The pieces of a value: what is left after each is exact.  An infinity or NaN is its own first piece
// and the others are zero; a finite value that rounds to infinity keeps its upper 16 bits instead.
template <int NP>
static __device__ __forceinline__ void split_pieces(float x, __bf16 (&out)[NP])
{
    if constexpr (NP == 1) {
        out[0] = (__bf16)x;
    } else {
        __bf16 a = (__bf16)x;
        const uint32_t mag = __float_as_uint(x) & 0x7FFFFFFFu;
        if (mag > 0x7F7F7FFFu && mag < 0x7F800000u) a = (__bf16)__uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
        const float ra = mag < 0x7F800000u ? x - (float)a : 0.0f;
        const __bf16 b = (__bf16)ra;
        out[0] = a;
        out[1] = b;
        if constexpr (NP > 2) out[2] = (__bf16)(ra - (float)b);
    }
}

static __device__ __forceinline__ bool row_live(const uint32_t *live, int64_t r)
{
    return !live || ((live[r >> 5] >> (r & 31)) & 1u);
}

// 64 x 64 tiles turned through LDS: dst[c][r] = src[r][c], rows from `rows` to rpad zero.  `order`: the place of
// a row among its 64 (the order of a sum's terms does not matter as long as both operands keep it; gradients of
// logits are written in the orders that a wave holds them in): 0 its own; 1: row 16 i + 4 h + r at 16 h + 4 i + r;
// 2: row 16 j + c at 4 c + j.
static __device__ __forceinline__ int place_of(int r, int order)
{
    return order == 0 ? r : order == 1 ? 16 * ((r >> 2) & 3) + 4 * (r >> 4) + (r & 3) : 4 * (r & 15) + (r >> 4);
}

// one tile, by NT threads, rows that are not live zero (barriers are the workgroup's: all of it is in here); `inside`: there is such a tile
template <class S, int NP>
struct PackCols {
    __bf16 tile[NP][64][72];        // [piece][column][row], rows of 144 bytes
};
template <class S, int NP, int NT, class Live>
static __device__ __forceinline__ void pack_cols_tile(PackCols<S, NP> &sh, int tid, bool inside, const S *__restrict__ src, int64_t ld, int64_t rows,
                                                      int64_t cols, int order, int vec, __bf16 *__restrict__ dst, int64_t rpad,
                                                      const PackLayout &to, int64_t r0, int64_t c0, const Live &live)
{
#pragma unroll
    for (int h = 0; h < 512 / NT; h++) {
        const int t = tid + h * NT, r = t >> 3, i0 = (t & 7) * 8;
        float x[8];
        const bool in = inside && r0 + r < rows && live(r0 + r);
        if (in) load8(src + (r0 + r) * ld, c0 + i0, cols, vec, x);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            __bf16 pc[NP];
            split_pieces<NP>(in ? x[e] : 0.0f, pc);
#pragma unroll
            for (int u = 0; u < NP; u++) sh.tile[u][i0 + e][place_of(r, order)] = pc[u];
        }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 512 / NT; h++) {
        const int t = tid + h * NT, c = t >> 3, i0 = (t & 7) * 8;
        if (inside && c0 + c < cols && r0 + i0 < rpad)
#pragma unroll
            for (int u = 0; u < NP; u++)
                *(v8bf *)(dst + (c0 + c) * to.ld + (r0 + i0) / 32 * to.block + u * to.piece + i0 % 32) = *(const v8bf *)&sh.tile[u][c][i0];
    }
}

// rows of a job, by the workgroup `block` of its `blocks`, of NT threads
template <class S, int NP, int NT>
static __device__ __forceinline__ void pack_rows_job(const PackJob &a, int64_t block)
{
    const int64_t per = a.pad / 8, total = a.rows * per;
    for (int64_t t = block * NT + threadIdx.x; t < total; t += (int64_t)a.blocks * NT) {
        const int64_t r = t / per, i0 = (t - r * per) * 8;
        float x[8];
        load8((const S *)a.src + r * a.ld, i0, a.cols, a.vec, x);
        v8bf o[NP];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            __bf16 pc[NP];
            split_pieces<NP>(x[e], pc);
#pragma unroll
            for (int u = 0; u < NP; u++) o[u][e] = pc[u];
        }
#pragma unroll
        for (int u = 0; u < NP; u++) *(v8bf *)(a.dst + r * a.to.ld + i0 / 32 * a.to.block + u * a.to.piece + i0 % 32) = o[u];
    }
}

static int is_vec(const void *p, int64_t ld, int width)
{
    const int64_t a = width == 1 ? 8 : 16;
    return (uintptr_t)p % a == 0 && ld * width % a == 0;
}
