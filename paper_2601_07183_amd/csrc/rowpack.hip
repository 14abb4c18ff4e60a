// Rows laid out for the products of rowprod.h: as bf16 pieces with every row filled up with zeros to
// a multiple of 64 values, in their own order or transposed.  Both kernels are bound by memory: they
// read a value once and write 2 bytes (bf16, bytes) or 6 (fp32) for it.
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

template <class S, int NP>
__global__ __launch_bounds__(WG) void pack_rows_kernel(const S *__restrict__ src, int64_t ld, int64_t rows, int64_t cols,
                                                       const int32_t *__restrict__ perm, int vec, __bf16 *__restrict__ dst,
                                                       int64_t kpad, int64_t piece, uint32_t *__restrict__ flags, int clear)
{
    if (flags && clear && blockIdx.x == 0 && threadIdx.x < 2) flags[threadIdx.x] = 0;
    uint32_t there = 0;
    const int64_t per = kpad / 8, total = rows * per;
    for (int64_t t = (int64_t)blockIdx.x * WG + threadIdx.x; t < total; t += (int64_t)gridDim.x * WG) {
        const int64_t r = t / per, i0 = (t - r * per) * 8;
        float x[8];
        load8(src + (perm ? (int64_t)perm[r] : r) * ld, i0, cols, vec, x);
        v8bf o[NP];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            __bf16 pc[NP];
            split_pieces<NP>(x[e], pc);
#pragma unroll
            for (int u = 0; u < NP; u++) o[u][e] = pc[u];
#pragma unroll
            for (int u = 1; u < NP; u++) there |= (float)pc[u] != 0.0f ? 1u << (u - 1) : 0u;
        }
#pragma unroll
        for (int u = 0; u < NP; u++) *(v8bf *)(dst + u * piece + r * kpad + i0) = o[u];
    }
    if (NP > 1 && flags && !clear) {
        if (__any(there & 1u) && (threadIdx.x & 63) == 0) flags[0] = 1;      // (all that do write the same)
        if (__any(there & 2u) && (threadIdx.x & 63) == 0) flags[1] = 1;
    }
}

// 64 x 64 tiles turned through LDS: dst[c][r] = src[r][c], rows from `rows` to rpad zero.  `order`: the place of
// a row among its 64 (the order of a sum's terms does not matter as long as both operands keep it; gradients of
// logits are written in the orders that a wave holds them in): 0 its own; 1: row 16 i + 4 h + r at 16 h + 4 i + r;
// 2: row 16 j + c at 4 c + j.
static __device__ __forceinline__ int place_of(int r, int order)
{
    return order == 0 ? r : order == 1 ? 16 * ((r >> 2) & 3) + 4 * (r >> 4) + (r & 3) : 4 * (r & 15) + (r >> 4);
}

template <class S, int NP>
__global__ __launch_bounds__(WG) void pack_cols_kernel(const S *__restrict__ src, int64_t ld, int64_t rows, int64_t cols,
                                                       const uint32_t *__restrict__ live, int order, int vec,
                                                       __bf16 *__restrict__ dst, int64_t rpad, int64_t piece)
{
    __shared__ __bf16 tile[NP][64][72];                  // [piece][column][row], rows of 144 bytes
    const int64_t r0 = (int64_t)blockIdx.x * 64, c0 = (int64_t)blockIdx.y * 64;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int t = threadIdx.x + h * WG, r = t >> 3, i0 = (t & 7) * 8;
        float x[8];
        const bool in = r0 + r < rows && row_live(live, r0 + r);
        if (in) load8(src + (r0 + r) * ld, c0 + i0, cols, vec, x);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            __bf16 pc[NP];
            split_pieces<NP>(in ? x[e] : 0.0f, pc);
#pragma unroll
            for (int u = 0; u < NP; u++) tile[u][i0 + e][place_of(r, order)] = pc[u];
        }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int t = threadIdx.x + h * WG, c = t >> 3, i0 = (t & 7) * 8;
        if (c0 + c < cols && r0 + i0 < rpad)
#pragma unroll
            for (int u = 0; u < NP; u++)
                *(v8bf *)(dst + u * piece + (c0 + c) * rpad + r0 + i0) = *(const v8bf *)&tile[u][c][i0];
    }
}

static int is_vec(const void *p, int64_t ld, int width)
{
    const int64_t a = width == 1 ? 8 : 16;
    return (uintptr_t)p % a == 0 && ld * width % a == 0;
}

int rairs_launch_pack_rows(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, const int32_t *perm, __bf16 *dst,
                           int64_t kpad, hipStream_t s, uint32_t *flags, bool clear)
{
    if (rows == 0) return RAIRS_OK;
    const int64_t piece = rows * kpad, want = (rows * (kpad / 8) + WG - 1) / WG;
    const dim3 grid((unsigned)(want < 8192 ? want : 8192));
    const int vec = is_vec(src, ld, dtype_width(dtype));
    if (dtype == RAIRS_F32)
        hipLaunchKernelGGL((pack_rows_kernel<float, 3>), grid, dim3(WG), 0, s, (const float *)src, ld, rows, cols, perm, vec, dst, kpad, piece, flags,
                           (int)clear);
    else if (dtype == RAIRS_BF16)
        hipLaunchKernelGGL((pack_rows_kernel<__bf16, 1>), grid, dim3(WG), 0, s, (const __bf16 *)src, ld, rows, cols, perm, vec, dst, kpad, piece, flags,
                           (int)clear);
    else
        hipLaunchKernelGGL((pack_rows_kernel<uint8_t, 1>), grid, dim3(WG), 0, s, (const uint8_t *)src, ld, rows, cols, perm, vec, dst, kpad, piece, flags,
                           (int)clear);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

int rairs_launch_pack_cols(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, const uint32_t *live, int order, __bf16 *dst,
                           int64_t rpad, hipStream_t s)
{
    if (cols == 0 || rpad == 0) return RAIRS_OK;
    const int vec = is_vec(src, ld, dtype_width(dtype));
    const int64_t piece = cols * rpad;
    const dim3 grid((unsigned)((rpad + 63) / 64), (unsigned)((cols + 63) / 64));
    if (dtype == RAIRS_F32)
        hipLaunchKernelGGL((pack_cols_kernel<float, 3>), grid, dim3(WG), 0, s, (const float *)src, ld, rows, cols, live, order, vec, dst, rpad, piece);
    else if (dtype == RAIRS_BF16)
        hipLaunchKernelGGL((pack_cols_kernel<__bf16, 1>), grid, dim3(WG), 0, s, (const __bf16 *)src, ld, rows, cols, live, order, vec, dst, rpad, piece);
    else
        hipLaunchKernelGGL((pack_cols_kernel<uint8_t, 1>), grid, dim3(WG), 0, s, (const uint8_t *)src, ld, rows, cols, live, order, vec, dst, rpad, piece);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

int rairs_operand(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, const int32_t *perm, __bf16 *room, RowOperand &out,
                  hipStream_t s, uint32_t *flags, bool clear)
{
    const int64_t kpad = pad_to(cols, ROWPROD_K);
    out.rows = rows;
    out.perm = nullptr;
    out.pieces_there = nullptr;
    if (rows_lie_right(src, dtype, ld, cols) && (!perm || rows * ld < (1ll << 31))) {
        out.p = (const __bf16 *)src;
        out.ld = ld;
        out.piece = 0;
        out.perm = perm;
        return RAIRS_OK;
    }
    out.p = room;
    out.ld = kpad;
    out.piece = rows * kpad;
    return rairs_launch_pack_rows(src, dtype, ld, rows, cols, perm, room, kpad, s, flags, clear);
}
