// A shared projection with low-rank adapters of many tenants in one batch: y = W x + s_a B_a (A_a x).
//
// Rows are put in order of their adapter (a counting sort on the device; nothing is read back), so
// that an adapter's rows lie together: u = s_a A_a x is then one small product per run of up to 16
// rows, and in the large product a tile adds the terms of the few adapters that its rows have, as
// further steps of the same sum in the same registers.  u enters that product as bf16 pieces (two or
// three, 16 or 24 bits), so it is as exact as the result's type can show.
//
// Up to 64 rows are bound by reading W once: no sort, the rows of W go straight into registers.
#include "fewrows.h"
#include "query_ops.h"

#define FEW_ROWS 64
#define SORT_ROWS 1024              // rows per workgroup of the sort
#define UNIT_ROWS 16                // rows of one adapter that one workgroup multiplies by A
#define CHUNK_ROWS 128              // rows of one adapter in one partial sum of its gradient

// ---- rows in order of their adapter ------------------------------------------------------------------

struct SortView {
    int64_t n, nb;                  // rows, workgroups of SORT_ROWS
    int na;
    const int32_t *adapter;
    int32_t *cnt;                   // [na + 1][nb], then first positions; key na: no adapter
    int32_t *first;                 // [na + 2] first position of each key, n at the end
    int32_t *unit0, *chunk0;        // [na + 1] first unit and first chunk of each adapter
    int32_t *perm, *of_row;         // [n]
    int4 *units, *chunks;           // {adapter, first position, rows, 0}
};

static __device__ __forceinline__ int sort_key(const SortView &v, int64_t i)
{
    const int a = v.adapter[i];
    return a >= 0 && a < v.na ? a : v.na;
}

__global__ __launch_bounds__(WG) void clear_words_kernel(int32_t *p, int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * WG + threadIdx.x;
    if (i < n) p[i] = 0;
}

__global__ __launch_bounds__(SORT_ROWS) void sort_count_kernel(SortView v)
{
    const int64_t i = (int64_t)blockIdx.x * SORT_ROWS + threadIdx.x;
    if (i < v.n) atomicAdd(&v.cnt[sort_key(v, i) * v.nb + blockIdx.x], 1);
}

// exclusive prefix sum of n words by one workgroup of 1024; every thread takes a run of them
static __device__ int32_t prefix_1024(int32_t *p, int64_t n, int32_t *sums)
{
    const int tid = threadIdx.x;
    const int64_t per = (n + 1023) / 1024, lo = tid * per < n ? tid * per : n, hi = lo + per < n ? lo + per : n;
    int32_t s = 0;
    for (int64_t i = lo; i < hi; i++) s += p[i];
    sums[tid] = s;
    __syncthreads();
    for (int o = 1; o < 1024; o <<= 1) {
        const int32_t x = tid >= o ? sums[tid - o] : 0;
        __syncthreads();
        sums[tid] += x;
        __syncthreads();
    }
    s = tid ? sums[tid - 1] : 0;
    const int32_t total = sums[1023];
    for (int64_t i = lo; i < hi; i++) {
        const int32_t x = p[i];
        p[i] = s;
        s += x;
    }
    __syncthreads();
    return total;
}

__global__ __launch_bounds__(1024) void sort_prefix_kernel(SortView v)
{
    __shared__ int32_t sums[1024];
    prefix_1024(v.cnt, (v.na + 1) * v.nb, sums);
    for (int k = threadIdx.x; k <= v.na + 1; k += 1024) v.first[k] = k <= v.na ? v.cnt[k * v.nb] : (int32_t)v.n;
    __syncthreads();
    for (int k = threadIdx.x; k <= v.na; k += 1024) {
        const int32_t rows = k < v.na ? v.first[k + 1] - v.first[k] : 0;
        v.unit0[k] = (rows + UNIT_ROWS - 1) / UNIT_ROWS;
        v.chunk0[k] = (rows + CHUNK_ROWS - 1) / CHUNK_ROWS;
    }
    __syncthreads();
    prefix_1024(v.unit0, v.na + 1, sums);
    prefix_1024(v.chunk0, v.na + 1, sums);
}

// (a row's place among its workgroup's rows of the same key keeps their order: the sums of the
// gradients are taken in the order of the batch, whatever order workgroups run in)
__global__ __launch_bounds__(SORT_ROWS) void sort_place_kernel(SortView v)
{
    __shared__ int32_t keys[SORT_ROWS];
    const int tid = threadIdx.x;
    const int64_t i = (int64_t)blockIdx.x * SORT_ROWS + tid;
    const int key = i < v.n ? sort_key(v, i) : -1;
    keys[tid] = key;
    __syncthreads();
    if (i >= v.n) return;
    int rank = 0;
    for (int j = 0; j < tid; j++) rank += keys[j] == key ? 1 : 0;
    const int32_t pos = v.cnt[key * v.nb + blockIdx.x] + rank;
    v.perm[pos] = (int32_t)i;
    v.of_row[pos] = key < v.na ? key : -1;
    if (key < v.na) {
        const int32_t at = pos - v.first[key], rows = v.first[key + 1] - v.first[key];
        if (at % UNIT_ROWS == 0) v.units[v.unit0[key] + at / UNIT_ROWS] = make_int4(key, pos, min(UNIT_ROWS, rows - at), 0);
        if (at % CHUNK_ROWS == 0) v.chunks[v.chunk0[key] + at / CHUNK_ROWS] = make_int4(key, pos, min(CHUNK_ROWS, rows - at), 0);
    }
}

static int64_t max_units(int64_t n, int na, int rows) { return n / rows + (na < n ? na : n) + 1; }

static SortView sort_carve(Carve &w, const int32_t *adapter, int64_t n, int na)
{
    SortView v = {};
    v.n = n;
    v.na = na;
    v.nb = (n + SORT_ROWS - 1) / SORT_ROWS;
    v.adapter = adapter;
    v.cnt = w.take<int32_t>((na + 1) * v.nb);
    v.first = w.take<int32_t>(na + 2);
    v.unit0 = w.take<int32_t>(na + 1);
    v.chunk0 = w.take<int32_t>(na + 1);
    v.perm = w.take<int32_t>(n);
    v.of_row = w.take<int32_t>(n);
    v.units = w.take<int4>(max_units(n, na, UNIT_ROWS));
    v.chunks = w.take<int4>(max_units(n, na, CHUNK_ROWS));
    return v;
}

static int sort_launch(const SortView &v, hipStream_t s)
{
    const int64_t words = (v.na + 1) * v.nb;
    hipLaunchKernelGGL(clear_words_kernel, dim3((unsigned)((words + WG - 1) / WG)), dim3(WG), 0, s, v.cnt, words);
    hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)v.nb), dim3(SORT_ROWS), 0, s, v);
    hipLaunchKernelGGL(sort_prefix_kernel, dim3(1), dim3(1024), 0, s, v);
    hipLaunchKernelGGL(sort_place_kernel, dim3((unsigned)v.nb), dim3(SORT_ROWS), 0, s, v);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

// ---- u = s_a A_a x for runs of up to 16 rows of one adapter -------------------------------------------

// products of pieces of u and of B (or A) laid side by side: columns t r .. t r + r - 1 hold piece pu[t]
// of u against piece pb[t]
struct SideBySide {
    int np, r, kpad;
    uint8_t pu[6], pb[6];
};

static SideBySide side_by_side(int upieces, int bpieces, int r)
{
    SideBySide x = {};
    RowProd rp = {};
    rowprod_pieces(rp, bpieces, upieces);
    x.np = rp.nseg;
    x.r = r;
    x.kpad = (int)pad_to(x.np * r, ROWPROD_K);
    for (int t = 0; t < rp.nseg; t++) {
        x.pb[t] = (rp.sp >> (4 * t)) & 15;
        x.pu[t] = (rp.sq >> (4 * t)) & 15;
    }
    return x;
}

static __device__ __forceinline__ void three_pieces(float x, __bf16 (&o)[3])
{
    o[0] = (__bf16)x;
    const float r = x - (float)o[0];
    o[1] = (__bf16)r;
    o[2] = (__bf16)(r - (float)o[1]);
}

struct ShrinkArgs {
    const void *x, *a;              // rows [n] of d; [adapters][r][d]
    int64_t ldx;
    int d, r;
    const float *scale;
    const int32_t *perm;
    const int4 *units;
    const int32_t *nunits;
    float *u;                       // [n][r] in sorted order, or null
    __bf16 *up;                     // [n][kpad] in sorted order, or null
    SideBySide side;
};

// a workgroup per unit; its waves share the sum, which is joined in LDS
template <class S, int RT, bool VEC>
__global__ __launch_bounds__(WG) void shrink_kernel(ShrinkArgs a)
{
    __shared__ float part[4][16][16 * RT + 1];           // [wave][row][rank]
    if ((int)blockIdx.x >= *a.nunits) return;
    const int4 unit = a.units[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = min(lane & 15, unit.z - 1);
    const S *qrow[1] = {(const S *)a.x + (int64_t)a.perm[unit.y + row] * a.ldx};
    const S *prow[RT];
    v4f acc[RT][1];
    float nrm[RT];
#pragma unroll
    for (int i = 0; i < RT; i++) {
        const int j = min(16 * i + (lane & 15), a.r - 1);
        prow[i] = (const S *)a.a + ((int64_t)unit.x * a.r + j) * a.d;
        acc[i][0] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int steps = (a.d + 4 * FewLoad<S>::CH - 1) / (4 * FewLoad<S>::CH);
    few_dot<S, S, RT, 1, VEC, false>(prow, qrow, steps * wave / 4, steps * (wave + 1) / 4, a.d, lane, acc, nrm);
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) part[wave][lane & 15][16 * i + 4 * (lane >> 4) + e] = acc[i][0][e];
    __syncthreads();
    const float sc = a.scale ? a.scale[unit.x] : 1.0f;
    for (int t = threadIdx.x; t < unit.z * a.r; t += WG) {
        const int i = t / a.r, j = t - i * a.r;
        const float x = ((part[0][i][j] + part[1][i][j]) + (part[2][i][j] + part[3][i][j])) * sc;
        part[0][i][j] = x;
        if (a.u) a.u[(int64_t)(unit.y + i) * a.r + j] = x;
    }
    if (!a.up) return;
    __syncthreads();
    for (int t = threadIdx.x; t < unit.z * a.side.kpad; t += WG) {
        const int i = t / a.side.kpad, k = t - i * a.side.kpad, b = k / a.r;
        __bf16 o = (__bf16)0.0f;
        if (b < a.side.np) {
            __bf16 pc[3];
            three_pieces(part[0][i][k - b * a.r], pc);
            const int w = a.side.pu[b];
            o = w == 0 ? pc[0] : w == 1 ? pc[1] : pc[2];
        }
        a.up[(int64_t)(unit.y + i) * a.side.kpad + k] = o;
    }
}

template <class S>
static int shrink_launch(const ShrinkArgs &a, int64_t units, bool vec, hipStream_t s)
{
    const dim3 grid((unsigned)units);
#define RAIRS_SHRINK(RT_)                                                                        \
    if (vec) hipLaunchKernelGGL((shrink_kernel<S, RT_, true>), grid, dim3(WG), 0, s, a);         \
    else hipLaunchKernelGGL((shrink_kernel<S, RT_, false>), grid, dim3(WG), 0, s, a)
    if (a.r <= 16) { RAIRS_SHRINK(1); }
    else if (a.r <= 32) { RAIRS_SHRINK(2); }
    else if (a.r <= 64) { RAIRS_SHRINK(4); }
    else { RAIRS_SHRINK(8); }
#undef RAIRS_SHRINK
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

// dst[a][o][t r + j] = piece pb[t] of src[a * batch + o * so + j * sj], zero up to kpad; and the row of
// zeros behind them
template <class S>
__global__ __launch_bounds__(WG) void pack_side_kernel(const S *__restrict__ src, int64_t batch, int64_t so, int64_t sj, int64_t rows,
                                                       int64_t total, SideBySide side, __bf16 *__restrict__ dst, __bf16 *__restrict__ zero)
{
    if (blockIdx.x == 0)
        for (int k = threadIdx.x; k < side.kpad; k += WG) zero[k] = (__bf16)0.0f;
    const int64_t t = (int64_t)blockIdx.x * WG + threadIdx.x;
    if (t >= total) return;
    const int64_t a = t / rows, o = t - a * rows;
    const S *p = src + a * batch + o * so;
    __bf16 *d = dst + t * side.kpad;
    for (int k0 = 0; k0 < side.kpad; k0 += 8) {
        v8bf x;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const int k = k0 + e, b = k / side.r;
            __bf16 v = (__bf16)0.0f;
            if (b < side.np) {
                __bf16 pc[3];
                three_pieces((float)p[(k - b * side.r) * sj], pc);
                const int w = side.pb[b];
                v = w == 0 ? pc[0] : w == 1 ? pc[1] : pc[2];
            }
            x[e] = v;
        }
        *(v8bf *)(d + k0) = x;
    }
}

static int pack_side_launch(const void *src, int dtype, int64_t batch, int64_t so, int64_t sj, int64_t rows, int64_t adapters,
                            const SideBySide &side, __bf16 *dst, __bf16 *zero, hipStream_t s)
{
    const int64_t total = rows * adapters;
    const dim3 grid((unsigned)((total + WG - 1) / WG));
    if (dtype == RAIRS_F32)
        hipLaunchKernelGGL(pack_side_kernel<float>, grid, dim3(WG), 0, s, (const float *)src, batch, so, sj, rows, total, side, dst, zero);
    else
        hipLaunchKernelGGL(pack_side_kernel<__bf16>, grid, dim3(WG), 0, s, (const __bf16 *)src, batch, so, sj, rows, total, side, dst, zero);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

// ---- a few rows ----------------------------------------------------------------------------------------

struct FewProjectArgs {
    const void *x, *w, *a, *b;
    int64_t ldx, ldy, n;
    int d_in, d_out, r, na;
    const int32_t *adapter;         // null: none
    const float *scale;
    float *u;                       // [n][r]
    void *y;
    int bf16_out;
};

// u: a wave per row and rank
template <class S>
__global__ __launch_bounds__(WG) void few_shrink_kernel(FewProjectArgs a, int vec)
{
    const int lane = threadIdx.x & 63, j = blockIdx.y * (WG / 64) + (threadIdx.x >> 6);
    const int64_t row = blockIdx.x;
    const int ad = a.adapter[row];
    if (j >= a.r || ad < 0 || ad >= a.na) return;
    constexpr int CH = FewLoad<S>::CH;
    const S *x = (const S *)a.x + row * a.ldx, *w = (const S *)a.a + ((int64_t)ad * a.r + j) * a.d_in;
    float s = 0.0f;
    for (int k = lane * CH; k < a.d_in; k += 64 * CH) {
        const FewFrag<S, CH> f = vec ? few_load<S, CH, true>(x, k, a.d_in) : few_load<S, CH, false>(x, k, a.d_in);
        const FewFrag<S, CH> g = vec ? few_load<S, CH, true>(w, k, a.d_in) : few_load<S, CH, false>(w, k, a.d_in);
#pragma unroll
        for (int e = 0; e < CH; e++) s = fmaf((float)f.e[e], (float)g.e[e], s);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) a.u[row * a.r + j] = a.scale ? s * a.scale[ad] : s;
}

// 16 columns of y per workgroup: its waves share the sum over d_in, then each finishes one tile of 16 rows
template <class S, int QT, bool VEC>
__global__ __launch_bounds__(WG) void few_project_kernel(FewProjectArgs a)
{
    __shared__ v4f part[4][QT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int p0 = blockIdx.x * 16;
    const S *prow[1] = {(const S *)a.w + (int64_t)min(p0 + (lane & 15), a.d_out - 1) * a.d_in};
    const S *qrow[QT];
    v4f acc[1][QT];
    float nrm[1];
#pragma unroll
    for (int j = 0; j < QT; j++) {
        const int64_t q = min((int64_t)(16 * j + (lane & 15)), a.n - 1);
        qrow[j] = (const S *)a.x + q * a.ldx;
        acc[0][j] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int steps = (a.d_in + 4 * FewLoad<S>::CH - 1) / (4 * FewLoad<S>::CH);
    few_dot<S, S, 1, QT, VEC, false>(prow, qrow, steps * wave / 4, steps * (wave + 1) / 4, a.d_in, lane, acc, nrm);
#pragma unroll
    for (int j = 0; j < QT; j++) part[wave][j][lane] = acc[0][j];
    __syncthreads();
    if (wave >= QT) return;
    const int64_t q = 16 * wave + (lane & 15);
    if (q >= a.n) return;
    v4f y = (part[0][wave][lane] + part[1][wave][lane]) + (part[2][wave][lane] + part[3][wave][lane]);
    const int o0 = p0 + 4 * (lane >> 4);
    const int ad = a.adapter ? a.adapter[q] : -1;
    if (ad >= 0 && ad < a.na) {
        const float *u = a.u + q * a.r;
        v4f z = {0.0f, 0.0f, 0.0f, 0.0f};
        const S *b = (const S *)a.b + (int64_t)ad * a.d_out * a.r;
        for (int j = 0; j < a.r; j++) {
            const float uj = u[j];
#pragma unroll
            for (int e = 0; e < 4; e++) z[e] = fmaf((float)b[(int64_t)min(o0 + e, a.d_out - 1) * a.r + j], uj, z[e]);
        }
        y += z;
    }
#pragma unroll
    for (int e = 0; e < 4; e++)
        if (o0 + e < a.d_out) {
            if (a.bf16_out) ((__bf16 *)a.y)[q * a.ldy + o0 + e] = (__bf16)y[e];
            else ((float *)a.y)[q * a.ldy + o0 + e] = y[e];
        }
}

template <class S>
static int few_project(const FewProjectArgs &a, hipStream_t s)
{
    const bool vec = (uintptr_t)a.x % 16 == 0 && a.ldx * sizeof(S) % 16 == 0 && (uintptr_t)a.w % 16 == 0 && a.d_in * sizeof(S) % 16 == 0 &&
                     (!a.adapter || (uintptr_t)a.a % 16 == 0);
    if (a.adapter) {
        hipLaunchKernelGGL(few_shrink_kernel<S>, dim3((unsigned)a.n, (unsigned)((a.r + 3) / 4)), dim3(WG), 0, s, a, (int)vec);
        RAIRS_HIP(hipGetLastError());
    }
    const dim3 grid((unsigned)((a.d_out + 15) / 16));
#define RAIRS_FEW(QT_)                                                                               \
    if (vec) hipLaunchKernelGGL((few_project_kernel<S, QT_, true>), grid, dim3(WG), 0, s, a);        \
    else hipLaunchKernelGGL((few_project_kernel<S, QT_, false>), grid, dim3(WG), 0, s, a)
    if (a.n <= 16) { RAIRS_FEW(1); }
    else if (a.n <= 32) { RAIRS_FEW(2); }
    else { RAIRS_FEW(4); }
#undef RAIRS_FEW
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

// ---- forward -------------------------------------------------------------------------------------------

static bool row_vec(const void *p, int64_t ld, int dtype) { return (uintptr_t)p % 16 == 0 && ld * dtype_width(dtype) % 16 == 0; }

int rairs_run_project(const ProjectArgs &g, void *ws, size_t *bytes, hipStream_t s)
{
    const rairs_projection_t &p = g.p;
    const bool adapters = p.n_adapters > 0;
    Carve w(ws);
    int rc = RAIRS_OK;
    if (g.n <= FEW_ROWS) {
        FewProjectArgs a = {};
        a.u = adapters ? w.take<float>(g.n * p.rank) : nullptr;
        if (bytes) *bytes = w.used;
        if (!ws) return RAIRS_OK;
        a.x = g.x; a.w = p.W; a.a = p.A; a.b = p.B;
        a.ldx = g.ldx; a.ldy = g.ldy; a.n = g.n;
        a.d_in = p.d_in; a.d_out = p.d_out; a.r = p.rank; a.na = p.n_adapters;
        a.adapter = adapters ? g.adapter : nullptr;
        a.scale = p.scale; a.y = g.y; a.bf16_out = g.ytype == RAIRS_BF16;
        return p.dtype == RAIRS_BF16 ? few_project<__bf16>(a, s) : few_project<float>(a, s);
    }
    const int np = dtype_pieces(p.dtype);
    __bf16 *xroom = w.take<__bf16>(pack_room(p.dtype, g.n, p.d_in)), *wroom = w.take<__bf16>(pack_room(p.dtype, p.d_out, p.d_in));
    SortView sv = {};
    SideBySide side = {};
    __bf16 *up = nullptr, *bp = nullptr, *zero = nullptr;
    if (adapters) {
        sv = sort_carve(w, g.adapter, g.n, p.n_adapters);
        side = side_by_side(3, np, p.rank);
        up = w.take<__bf16>(g.n * side.kpad);
        bp = w.take<__bf16>((int64_t)p.n_adapters * p.d_out * side.kpad);
        zero = w.take<__bf16>(side.kpad);
    }
    if (bytes) *bytes = w.used;
    if (!ws) return RAIRS_OK;

    const bool use = adapters && g.adapter;
    RowProd rp = {};
    rowprod_pieces(rp, np, np);
    rp.ksteps = (int)(pad_to(p.d_in, ROWPROD_K) / ROWPROD_K);
    if (use && (rc = sort_launch(sv, s))) return rc;
    if ((rc = rairs_operand(p.W, p.dtype, p.d_in, p.d_out, p.d_in, nullptr, wroom, rp.P, s))) return rc;
    if ((rc = rairs_operand(g.x, p.dtype, g.ldx, g.n, p.d_in, use ? sv.perm : nullptr, xroom, rp.Q, s))) return rc;
    if (use) {
        ShrinkArgs sa = {g.x, p.A, g.ldx, p.d_in, p.rank, p.scale, sv.perm, sv.units, sv.unit0 + p.n_adapters, nullptr, up, side};
        const bool vec = row_vec(g.x, g.ldx, p.dtype) && row_vec(p.A, p.d_in, p.dtype);
        const int64_t units = max_units(g.n, p.n_adapters, UNIT_ROWS);
        if ((rc = p.dtype == RAIRS_BF16 ? shrink_launch<__bf16>(sa, units, vec, s) : shrink_launch<float>(sa, units, vec, s))) return rc;
        if ((rc = pack_side_launch(p.B, p.dtype, (int64_t)p.d_out * p.rank, p.rank, 1, p.d_out, p.n_adapters, side, bp, zero, s))) return rc;
        rp.ad = AdapterPart{up, bp, zero, sv.of_row, sv.first + 1, side.kpad};
    }
    StoreEpi e = {g.y, g.ldy, 0, p.d_out, g.n, use ? sv.perm : nullptr, g.ytype == RAIRS_BF16, 0};
    return use ? rowprod_launch_any<true>(rp, e, s) : rowprod_launch_any(rp, e, s);
}

// ---- backward ------------------------------------------------------------------------------------------

// dst[b][c][r] = src[b][r][c]
template <class S>
__global__ __launch_bounds__(WG) void transpose_kernel(const S *__restrict__ src, int rows, int cols, S *__restrict__ dst)
{
    __shared__ S tile[32][33];
    const int64_t batch = (int64_t)blockIdx.z * rows * cols;
    const int r0 = blockIdx.x * 32, c0 = blockIdx.y * 32, x = threadIdx.x & 31, y = threadIdx.x >> 5;
    for (int i = y; i < 32; i += 8)
        if (r0 + i < rows && c0 + x < cols) tile[i][x] = src[batch + (int64_t)(r0 + i) * cols + c0 + x];
    __syncthreads();
    for (int i = y; i < 32; i += 8)
        if (c0 + i < cols && r0 + x < rows) dst[batch + (int64_t)(c0 + i) * rows + r0 + x] = tile[x][i];
}

// Partial sums of an adapter's gradient over a chunk of its rows: part[chunk][j][i] = sum_rows u[row][j]
// x[row][i].  A thread has one column and 16 ranks; u comes through scalar registers.
#define GRAD_RANKS 16
template <class S>
__global__ __launch_bounds__(WG) void adapter_grad_kernel(const S *__restrict__ x, int64_t ldx, const int32_t *__restrict__ perm,
                                                          const float *__restrict__ u, int r, int cols, const int4 *__restrict__ chunks,
                                                          const int32_t *__restrict__ nchunks, float *__restrict__ part)
{
    if ((int)blockIdx.x >= *nchunks) return;
    const int4 ch = chunks[blockIdx.x];
    const int i = blockIdx.y * WG + threadIdx.x, j0 = blockIdx.z * GRAD_RANKS;
    const int ic = min(i, cols - 1), nj = min(GRAD_RANKS, r - j0);
    float acc[GRAD_RANKS];
#pragma unroll
    for (int j = 0; j < GRAD_RANKS; j++) acc[j] = 0.0f;
    const float *ub = u + (int64_t)ch.y * r + j0;
#pragma unroll 4
    for (int k = 0; k < ch.z; k++) {
        const float xv = (float)x[(int64_t)perm[ch.y + k] * ldx + ic];
        const float *uk = ub + (int64_t)k * r;
#pragma unroll
        for (int j = 0; j < GRAD_RANKS; j++) acc[j] = fmaf(uk[min(j, nj - 1)], xv, acc[j]);
    }
    if (i >= cols) return;
    float *o = part + ((int64_t)blockIdx.x * r + j0) * cols + i;
#pragma unroll
    for (int j = 0; j < GRAD_RANKS; j++)
        if (j < nj) o[(int64_t)j * cols] = acc[j];
}

// out[a][j][i] (or, turned, out[a][i][j]) = the sum of the adapter's chunks in their order
template <class S>
__global__ __launch_bounds__(WG) void adapter_join_kernel(const float *__restrict__ part, const int32_t *__restrict__ chunk0, int r, int cols,
                                                          int turned, S *__restrict__ out)
{
    const int a = blockIdx.y;
    const int64_t t = (int64_t)blockIdx.x * WG + threadIdx.x;
    if (t >= (int64_t)r * cols) return;
    int j, i;
    if (turned) { i = (int)(t / r); j = (int)(t - (int64_t)i * r); }
    else { j = (int)(t / cols); i = (int)(t - (int64_t)j * cols); }
    float x = 0.0f;
    for (int c = chunk0[a]; c < chunk0[a + 1]; c++) x += part[((int64_t)c * r + j) * cols + i];
    out[(int64_t)a * r * cols + t] = (S)x;
}

template <class S>
static int adapter_grads(const ProjectArgs &g, const SortView &sv, const float *u, const float *v, float *part, hipStream_t s)
{
    const rairs_projection_t &p = g.p;
    const unsigned chunks = (unsigned)max_units(g.n, p.n_adapters, CHUNK_ROWS), rz = (unsigned)((p.rank + GRAD_RANKS - 1) / GRAD_RANKS);
    const int32_t *nch = sv.chunk0 + p.n_adapters;
    for (int side = 0; side < 2; side++) {
        const int cols = side ? p.d_out : p.d_in;
        hipLaunchKernelGGL(adapter_grad_kernel<S>, dim3(chunks, (unsigned)((cols + WG - 1) / WG), rz), dim3(WG), 0, s, (const S *)(side ? g.dy : g.x),
                           side ? g.lddy : g.ldx, sv.perm, side ? u : v, p.rank, cols, sv.chunks, nch, part);
        hipLaunchKernelGGL(adapter_join_kernel<S>, dim3((unsigned)(((int64_t)p.rank * cols + WG - 1) / WG), (unsigned)p.n_adapters), dim3(WG), 0, s,
                           part, sv.chunk0, p.rank, cols, side, (S *)(side ? g.db : g.da));
        RAIRS_HIP(hipGetLastError());
    }
    return RAIRS_OK;
}

template <class S>
static int transpose_launch(const void *src, int rows, int cols, int batches, void *dst, hipStream_t s)
{
    hipLaunchKernelGGL(transpose_kernel<S>, dim3((unsigned)((rows + 31) / 32), (unsigned)((cols + 31) / 32), (unsigned)batches), dim3(WG), 0, s,
                       (const S *)src, rows, cols, (S *)dst);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

int rairs_run_project_backward(const ProjectArgs &g, void *ws, size_t *bytes, hipStream_t s)
{
    const rairs_projection_t &p = g.p;
    const int np = dtype_pieces(p.dtype), na = p.n_adapters;
    const bool adapters = na > 0;
    const int64_t opad = pad_to(p.d_out, ROWPROD_K);
    Carve w(ws);
    __bf16 *yroom = w.take<__bf16>(pack_room(p.dtype, g.n, p.d_out)), *wt = w.take<__bf16>((int64_t)p.d_in * opad * np);
    SortView sv = {};
    SideBySide side = {};
    __bf16 *vp = nullptr, *ap = nullptr, *zero = nullptr;
    float *u = nullptr, *v = nullptr, *part = nullptr;
    char *bt = nullptr;
    if (adapters) {
        sv = sort_carve(w, g.adapter, g.n, na);
        side = side_by_side(3, np, p.rank);
        vp = w.take<__bf16>(g.n * side.kpad);
        ap = w.take<__bf16>((int64_t)na * p.d_in * side.kpad);
        zero = w.take<__bf16>(side.kpad);
        u = w.take<float>(g.n * p.rank);
        v = w.take<float>(g.n * p.rank);
        bt = w.take<char>((int64_t)na * p.rank * p.d_out * dtype_width(p.dtype));
        part = w.take<float>(max_units(g.n, na, CHUNK_ROWS) * p.rank * (p.d_in > p.d_out ? p.d_in : p.d_out));
    }
    if (bytes) *bytes = w.used;
    if (!ws) return RAIRS_OK;

    const bool use = adapters && g.adapter && g.n > 0;
    const bool bf = p.dtype == RAIRS_BF16;
    int rc = RAIRS_OK;
    if (use) {
        if ((rc = sort_launch(sv, s))) return rc;
        const int64_t units = max_units(g.n, na, UNIT_ROWS);
        rc = bf ? transpose_launch<__bf16>(p.B, p.d_out, p.rank, na, bt, s) : transpose_launch<float>(p.B, p.d_out, p.rank, na, bt, s);
        if (rc) return rc;
        ShrinkArgs sa = {g.dy, bt, g.lddy, p.d_out, p.rank, p.scale, sv.perm, sv.units, sv.unit0 + na, v, g.dx ? vp : nullptr, side};
        const bool vec = row_vec(g.dy, g.lddy, p.dtype) && row_vec(bt, p.d_out, p.dtype);
        if ((rc = bf ? shrink_launch<__bf16>(sa, units, vec, s) : shrink_launch<float>(sa, units, vec, s))) return rc;
        if (g.da) {
            ShrinkArgs su = {g.x, p.A, g.ldx, p.d_in, p.rank, p.scale, sv.perm, sv.units, sv.unit0 + na, u, nullptr, side};
            const bool xvec = row_vec(g.x, g.ldx, p.dtype) && row_vec(p.A, p.d_in, p.dtype);
            if ((rc = bf ? shrink_launch<__bf16>(su, units, xvec, s) : shrink_launch<float>(su, units, xvec, s))) return rc;
            if ((rc = bf ? adapter_grads<__bf16>(g, sv, u, v, part, s) : adapter_grads<float>(g, sv, u, v, part, s))) return rc;
        }
    } else if (g.da && adapters) {
        if ((rc = rairs_launch_clear_rows(g.da, na, (int64_t)p.rank * p.d_in, (int64_t)p.rank * p.d_in, p.dtype, s))) return rc;
        if ((rc = rairs_launch_clear_rows(g.db, na, (int64_t)p.rank * p.d_out, (int64_t)p.rank * p.d_out, p.dtype, s))) return rc;
    }
    if (!g.dx || g.n == 0) return RAIRS_OK;
    RowProd rp = {};
    rowprod_pieces(rp, np, np);
    rp.ksteps = (int)(opad / ROWPROD_K);
    if ((rc = rairs_launch_pack_cols(p.W, p.dtype, p.d_in, p.d_out, p.d_in, nullptr, ORDER_SAME, wt, opad, s))) return rc;
    rp.P = RowOperand{wt, opad, p.d_in * opad, p.d_in, nullptr, nullptr};
    if ((rc = rairs_operand(g.dy, p.dtype, g.lddy, g.n, p.d_out, use ? sv.perm : nullptr, yroom, rp.Q, s))) return rc;
    if (use) {
        if ((rc = pack_side_launch(p.A, p.dtype, (int64_t)p.rank * p.d_in, 1, p.d_in, p.d_in, na, side, ap, zero, s))) return rc;
        rp.ad = AdapterPart{vp, ap, zero, sv.of_row, sv.first + 1, side.kpad};
    }
    StoreEpi e = {g.dx, g.lddx, 0, p.d_in, g.n, use ? sv.perm : nullptr, bf, 0};
    return use ? rowprod_launch_any<true>(rp, e, s) : rowprod_launch_any(rp, e, s);
}
