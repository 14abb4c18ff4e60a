// Rows laid out for the products of rowprod.h: as bf16 pieces with every row filled up with zeros to
// a multiple of 64 values (of 32 where all three pieces lie together), in their own order or transposed.  The
// kernels are bound by memory: they read a value once and write 2 bytes (bf16, bytes) or 6 (fp32) for it
// (65,537 x 1024 bf16 turned: 68 us, 3.9 TB/s).
#include <algorithm>

#include "rowpack.h"

template <class S, int NP>
__global__ __launch_bounds__(WG) void pack_rows_kernel(const S *__restrict__ src, int64_t ld, int64_t rows, int64_t cols,
                                                       const int32_t *__restrict__ perm, int vec, __bf16 *__restrict__ dst,
                                                       int64_t kpad, PackLayout to, uint32_t *__restrict__ flags, int clear)
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
        for (int u = 0; u < NP; u++) *(v8bf *)(dst + r * to.ld + i0 / 32 * to.block + u * to.piece + i0 % 32) = o[u];
    }
    if (NP > 1 && flags && !clear) {
        if (__any(there & 1u) && (threadIdx.x & 63) == 0) flags[0] = 1;      // (all that do write the same)
        if (__any(there & 2u) && (threadIdx.x & 63) == 0) flags[1] = 1;
    }
}

template <class S, int NP>
static __device__ __forceinline__ void pack_job(const PackJob &a, int64_t block, char *lds)
{
    if (!a.turned) {
        pack_rows_job<S, NP, WG>(a, block);
        return;
    }
    const int64_t rt = (a.pad + 63) / 64;
    pack_cols_tile<S, NP, WG>(*(PackCols<S, NP> *)lds, threadIdx.x, true, (const S *)a.src, a.ld, a.rows, a.cols, a.order, a.vec, a.dst, a.pad, a.to,
                              block % rt * 64, block / rt * 64, [&](int64_t r) {
                                  if (!a.targets) return row_live(a.live, r);
                                  const int64_t t = a.targets[r];
                                  const bool seen = t >= 0 && t < a.V && row_live(a.live ? a.live + r * a.ld_live : nullptr, t);
                                  return (seen && a.dlogp[r] != 0.0f) || (a.dentropy && a.dentropy[r] != 0.0f);
                              });
}

__global__ __launch_bounds__(WG) void pack_jobs_kernel(PackJobs a)
{
    __shared__ __align__(16) char lds[sizeof(PackCols<float, 3>)];
    int64_t block = blockIdx.x;
    int i = 0;
    while (i + 1 < a.n && block >= a.job[i].blocks) block -= a.job[i++].blocks;
    const PackJob &job = a.job[i];
    if (job.dtype == RAIRS_F32) pack_job<float, 3>(job, block, lds);
    else if (job.dtype == RAIRS_BF16) pack_job<__bf16, 1>(job, block, lds);
    else pack_job<uint8_t, 1>(job, block, lds);
}

int rairs_launch_pack(PackJobs &jobs, hipStream_t s)
{
    unsigned blocks = 0;
    for (int i = 0; i < jobs.n; i++) {
        PackJob &j = jobs.job[i];
        const int64_t want = j.turned ? (j.pad + 63) / 64 * ((j.cols + 63) / 64) : std::min<int64_t>((j.rows * (j.pad / 8) + WG - 1) / WG, 8192);
        j.blocks = (unsigned)want;
        j.vec = is_vec(j.src, j.ld, dtype_width(j.dtype));
        blocks += j.blocks;
    }
    if (!blocks) return RAIRS_OK;
    hipLaunchKernelGGL(pack_jobs_kernel, dim3(blocks), dim3(WG), 0, s, jobs);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

void rairs_operand_job(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, bool threes, __bf16 *room, RowOperand &out, PackJobs &jobs)
{
    out = RowOperand{};
    out.rows = rows;
    if (rows_lie_right(src, dtype, ld, cols)) {
        out.p = (const __bf16 *)src;
        out.ld = ld;
        return;
    }
    const int64_t kpad = pad_to(cols, threes ? 32 : ROWPROD_K);
    const PackLayout to = pack_layout(rows, kpad, threes);
    out.p = room;
    out.ld = to.ld;
    out.piece = threes ? 0 : to.piece;
    PackJob &j = jobs.job[jobs.n++];
    j = PackJob{};
    j.src = src; j.dst = room; j.dtype = dtype; j.ld = ld; j.rows = rows; j.cols = cols; j.pad = kpad; j.to = to;
}

int rairs_launch_pack_rows(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, const int32_t *perm, __bf16 *dst,
                           int64_t kpad, PackLayout to, hipStream_t s, uint32_t *flags, bool clear)
{
    if (rows == 0) return RAIRS_OK;
    const int64_t want = (rows * (kpad / 8) + WG - 1) / WG;
    const dim3 grid((unsigned)(want < 8192 ? want : 8192));
    const int vec = is_vec(src, ld, dtype_width(dtype));
    if (dtype == RAIRS_F32)
        hipLaunchKernelGGL((pack_rows_kernel<float, 3>), grid, dim3(WG), 0, s, (const float *)src, ld, rows, cols, perm, vec, dst, kpad, to, flags,
                           (int)clear);
    else if (dtype == RAIRS_BF16)
        hipLaunchKernelGGL((pack_rows_kernel<__bf16, 1>), grid, dim3(WG), 0, s, (const __bf16 *)src, ld, rows, cols, perm, vec, dst, kpad, to, flags,
                           (int)clear);
    else
        hipLaunchKernelGGL((pack_rows_kernel<uint8_t, 1>), grid, dim3(WG), 0, s, (const uint8_t *)src, ld, rows, cols, perm, vec, dst, kpad, to, flags,
                           (int)clear);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

int rairs_launch_pack_cols(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, const uint32_t *live, int order, __bf16 *dst,
                           int64_t rpad, PackLayout to, hipStream_t s)
{
    PackJobs jobs = {};
    jobs.n = 1;
    PackJob &j = jobs.job[0];
    j.src = src; j.dst = dst; j.dtype = dtype; j.turned = 1; j.ld = ld; j.rows = rows; j.cols = cols; j.pad = rpad; j.to = to;
    j.order = order; j.live = live;
    return rairs_launch_pack(jobs, s);
}

int rairs_operand(const void *src, int dtype, int64_t ld, int64_t rows, int64_t cols, const int32_t *perm, bool threes, __bf16 *room,
                  RowOperand &out, hipStream_t s, uint32_t *flags, bool clear)
{
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
    const int64_t kpad = pad_to(cols, threes ? 32 : ROWPROD_K);
    const PackLayout to = pack_layout(rows, kpad, threes);
    out.p = room;
    out.ld = to.ld;
    out.piece = threes ? 0 : to.piece;
    return rairs_launch_pack_rows(src, dtype, ld, rows, cols, perm, room, kpad, to, s, flags, clear);
}
