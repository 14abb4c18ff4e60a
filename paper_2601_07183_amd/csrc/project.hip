// A shared projection with low-rank adapters of many tenants in one batch: y = W x + s_a B_a (A_a x).
//
// Rows are put in order of their adapter (a counting sort on the device; nothing is read back), so
// that an adapter's rows lie together: u = s_a A_a x is then one small product per run of up to 32
// rows, and in the large product a tile adds the terms of the few adapters that its rows have, as
// further steps of the same sum in the same registers, with u zero in the rows of the others.  (Zero times
// an infinity is not zero: what is not finite in an adapter goes in as zero, and is added to the adapter's own
// rows when they are written.)  u enters that product as three bf16 pieces.
//
// fp32 products of few tiles take the rows as they are and the fp32 instruction, u and B with them (10,000 x 1024 to
// 128: 43 us, by pieces 46 and 20 for making them; with 250 adapters of rank 16 51 us, as the tiles' adapters are
// further steps).  A few rows go
// another way altogether: no sort, the rows of W and x straight from memory into the matrix instruction's
// registers, and a row's own B times u on the vector units behind it.
#include <algorithm>

#include "fewrows.h"
#include "query_ops.h"
#include "rowpack.h"

#define SORT_ROWS 1024              // rows per workgroup of the sort
#define UNIT_ROWS 32                // rows of one adapter that one workgroup multiplies by A
#define CHUNK_ROWS 256              // rows of one adapter in one partial sum of its gradient
#define FEW_ROWS 256                // up to here every row takes its own way through its adapter's A

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

// Adapters that have rows, numbered in their order, where a batch may have far fewer than there are: what is laid out of
// adapters is laid out of these alone.
struct UsedView {
    const int32_t *adapter;         // [n]
    int64_t n;
    int na, most;                   // adapters; how many may have rows
    int32_t *number;                // [n] of the row's adapter, -1: none
    int32_t *orig, *of;             // [most] adapter of a number (the first one's for numbers that none has), [na] number of an adapter or -1
};
__global__ __launch_bounds__(1024) void used_kernel(UsedView v)
{
    __shared__ uint32_t bits[RAIRS_MAX_ADAPTERS / 32];
    __shared__ int32_t before[RAIRS_MAX_ADAPTERS / 32 + 1];
    const int tid = threadIdx.x, words = (v.na + 31) / 32;
    for (int w = tid; w < words; w += 1024) bits[w] = 0;
    __syncthreads();
    for (int64_t i = tid; i < v.n; i += 1024) {
        const int a = v.adapter[i];
        if (a >= 0 && a < v.na) atomicOr(&bits[a >> 5], 1u << (a & 31));
    }
    __syncthreads();
    if (tid == 0) {
        int s = 0;
        for (int w = 0; w < words; w++) {
            before[w] = s;
            s += __popc(bits[w]);
        }
        before[words] = s;
    }
    __syncthreads();
    const auto number = [&](int a) { return (bits[a >> 5] >> (a & 31)) & 1u ? before[a >> 5] + __popc(bits[a >> 5] & ((1u << (a & 31)) - 1u)) : -1; };
    for (int a = tid; a < v.na; a += 1024) {
        const int k = number(a);
        v.of[a] = k;
        if (k >= 0) v.orig[k] = a;
    }
    for (int k = before[words] + tid; k < v.most; k += 1024) v.orig[k] = 0;
    for (int64_t i = tid; i < v.n; i += 1024) {
        const int a = v.adapter[i];
        v.number[i] = a >= 0 && a < v.na ? number(a) : -1;
    }
}

// A launch more (6 us) against what is not laid out: 32 MB of it take as long.
static bool numbers_used(const rairs_projection_t &p, int64_t n, int64_t bytes_each) { return p.n_adapters > n && (p.n_adapters - n) * bytes_each > 32ll << 20; }
static UsedView used_carve(Carve &w, const rairs_projection_t &p, const int32_t *adapter, int64_t n)
{
    return UsedView{adapter, n, p.n_adapters, (int)n, w.take<int32_t>(n), w.take<int32_t>(n), w.take<int32_t>(p.n_adapters)};
}
static int used_launch(const UsedView &v, hipStream_t s)
{
    hipLaunchKernelGGL(used_kernel, dim3(1), dim3(1024), 0, s, v);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}
// (orig: null where adapters are their own numbers)
static __device__ __forceinline__ int64_t orig_of(const int32_t *orig, int64_t a) { return orig ? orig[a] : a; }

// lanes of the wave with the same key (below 2^bits, bits <= 13); key < 0: none
static __device__ __forceinline__ unsigned long long same_key(int key, int bits)
{
    const unsigned long long any = __ballot(key >= 0);
    uint32_t lo = (uint32_t)any, hi = (uint32_t)(any >> 32);
#pragma unroll
    for (int b = 0; b < 13; b++) {
        if (b < bits) {                                               // uniform
            const int mine = (int)((uint32_t)key << (31 - b)) >> 31;  // all bits or none
            const unsigned long long set = __ballot(mine);
            lo &= ~(mine ^ (uint32_t)set);
            hi &= ~(mine ^ (uint32_t)(set >> 32));
        }
    }
    return (unsigned long long)hi << 32 | lo;
}

__global__ __launch_bounds__(SORT_ROWS) void sort_count_kernel(SortView v)
{
    const int64_t i = (int64_t)blockIdx.x * SORT_ROWS + threadIdx.x;
    const int key = i < v.n ? sort_key(v, i) : -1;
    const unsigned long long m = same_key(key, 32 - __clz(v.na));
    if (key >= 0 && (threadIdx.x & 63) == (unsigned)__ffsll((long long)m) - 1)     // one addition per key and wave
        atomicAdd(&v.cnt[key * v.nb + blockIdx.x], (int)__popcll(m));
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

// The whole sort by one workgroup, for a batch whose keys fit LDS: every wave counts a run of the rows, 64 at
// a time, then places them behind the runs before it (in the batch's order, as above).
#define SORT_ONE_ROWS 16384
#define SORT_ONE_KEYS 1024
static __device__ void sort_one(const SortView &v, int32_t *sort_lds)
{
    __shared__ int32_t sums[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, keys = v.na + 1, bits = 32 - __clz(v.na);
    int32_t *cnt = sort_lds;                                          // [16][keys]
    const int n = (int)v.n;
    uint16_t *key_of = (uint16_t *)(sort_lds + 16 * keys), *rank_of = key_of + (n + 1) / 2 * 2;    // [n] both; a rank is the row's among its wave's
    const int per = ((n + 15) / 16 + 63) / 64 * 64;                   // rows per wave
#pragma unroll 8
    for (int i = tid; i < n; i += 1024) key_of[i] = (uint16_t)sort_key(v, i);
    for (int i = tid; i < 16 * keys; i += 1024) cnt[i] = 0;
    __syncthreads();
    int32_t *mine = cnt + wave * keys;
    for (int i0 = wave * per; i0 < min((wave + 1) * per, n); i0 += 64) {
        const int key = i0 + lane < n ? key_of[i0 + lane] : -1;
        const unsigned long long m = same_key(key, bits);
        const int base = key >= 0 ? mine[key] : 0;
        wave_lds_sync();
        if (key >= 0) {
            rank_of[i0 + lane] = (uint16_t)(base + __popcll(m & ((1ull << lane) - 1ull)));
            if (lane == __ffsll((long long)m) - 1) mine[key] = base + __popcll(m);
        }
        wave_lds_sync();
    }
    __syncthreads();
    // a thread per key: its rows, then exclusive sums over the keys of rows, units and chunks
    int rows = 0;
    if (tid < keys)
        for (int w = 0; w < 16; w++) rows += cnt[w * keys + tid];
    const auto scan = [&](int x) {
        const int incl = (int)wave_incl_sum_u32((uint32_t)x);
        __syncthreads();
        if (lane == 63) sums[wave] = incl;
        __syncthreads();
        int before = 0;
        for (int w = 0; w < wave; w++) before += sums[w];
        return before + incl - x;
    };
    const int first = scan(rows), real = tid < v.na ? rows : 0;
    const int unit0 = scan((real + UNIT_ROWS - 1) / UNIT_ROWS), chunk0 = scan((real + CHUNK_ROWS - 1) / CHUNK_ROWS);
    if (tid < keys) {
        v.first[tid] = first;
        v.unit0[tid] = unit0;
        v.chunk0[tid] = chunk0;
        int at = first;
        for (int w = 0; w < 16; w++) {
            const int c = cnt[w * keys + tid];
            cnt[w * keys + tid] = at;
            at += c;
        }
        if (tid < v.na) {
            for (int i = 0; i < rows; i += UNIT_ROWS) v.units[unit0 + i / UNIT_ROWS] = make_int4(tid, first + i, min(UNIT_ROWS, rows - i), 0);
            for (int i = 0; i < rows; i += CHUNK_ROWS) v.chunks[chunk0 + i / CHUNK_ROWS] = make_int4(tid, first + i, min(CHUNK_ROWS, rows - i), 0);
        }
    }
    if (tid == 0) v.first[v.na + 1] = n;
    __syncthreads();
    // (the order goes through LDS and out in runs: written from here, every lane's line would be an access)
    constexpr int EACH = SORT_ONE_ROWS / 1024;
    int pos[EACH];
#pragma unroll
    for (int u = 0; u < EACH; u++) {
        const int i = tid + u * 1024;
        pos[u] = i < n ? cnt[i / per * keys + key_of[i]] + rank_of[i] : 0;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < EACH; u++)
        if (tid + u * 1024 < n) rank_of[pos[u]] = (uint16_t)(tid + u * 1024);
    __syncthreads();
    for (int i = tid; i < n; i += 1024) {
        const int r = rank_of[i], key = key_of[r];
        v.perm[i] = r;
        v.of_row[i] = key < v.na ? key : -1;
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

static bool sorts_in_one(const SortView &v) { return v.n <= SORT_ONE_ROWS && v.na < SORT_ONE_KEYS; }
#define SORT_ONE_LDS (16 * SORT_ONE_KEYS * 4 + SORT_ONE_ROWS * 4)
static size_t sort_one_lds(const SortView &v) { return (size_t)16 * (v.na + 1) * 4 + (size_t)((v.n + 1) / 2) * 8; }

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

// ---- u = s_a A_a x for runs of rows of one adapter ---------------------------------------------------

// u (rows) and B or A (columns) as operands of the large product.  bf16: u's three pieces side by side, the smallest
// first, against three times B.  fp32: threes like the rows, or (F32) values for the fp32 instruction.
enum { SIDE_BF16, SIDE_THREES, SIDE_F32 };
struct Side {
    int mode, r, kpad;              // kpad: units of two bytes
};

static Side side_of(int mode, int r)
{
    return Side{mode, r, (int)(mode == SIDE_BF16 ? pad_to(3 * r, ROWPROD_K) : mode == SIDE_THREES ? 3 * pad_to(r, 32) : 2 * pad_to(r, 32))};
}

// place k of a row of u (ROWS) or of B, whose values are at(j)
template <bool ROWS, class F>
static __device__ __forceinline__ __bf16 side_piece(const Side &side, int k, const F &at)
{
    const bool threes = side.mode == SIDE_THREES;
    const int j = threes ? k / 96 * 32 + k % 32 : k % side.r, piece = threes ? k % 96 / 32 : ROWS ? 2 - k / side.r : 0;
    if (threes ? j >= side.r : k >= 3 * side.r) return (__bf16)0.0f;
    __bf16 pc[3];
    split_pieces<3>(at(j), pc);
    return piece == 0 ? pc[0] : piece == 1 ? pc[1] : pc[2];
}

// what the packing of an adapter's columns found: word i says whether its workgroup i met a value that is not finite
struct SideFlags {
    uint32_t *found, *bad;          // [side_blocks]; [adapters] the same by adapter (of its own and its neighbours' values)
    int64_t rows;                   // columns per adapter; 0: not wanted
};
static int64_t side_blocks(const Side &side, int64_t rows) { return (pad_to(rows, 64) * (side.kpad / 8) + 1023) / 1024; }

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
    Side side;
    SideFlags flags;
    const int32_t *orig, *aorig;    // of the scale, of a
};

// A workgroup per unit; its NW waves share the sum, which is joined in LDS.  Bound by the loads: a lane's 16 bytes lie in a
// row of their own, which costs a cache access each (10,000 x 1024 fp32, 250 adapters of rank 16: 19 us, half of it
// accesses; 8,191 x 4096 bf16, 7 of rank 64: 41 us).
template <class S, int RT, int NW, bool VEC>
__global__ __launch_bounds__(64 * NW) void shrink_kernel(ShrinkArgs one, ShrinkArgs two)
{
    const ShrinkArgs &a = blockIdx.y ? two : one;
    __shared__ float part[NW - 1][UNIT_ROWS][16 * RT + 1];    // [wave][row][rank]
    if ((int)blockIdx.x >= *a.nunits) return;
    const int4 unit = a.units[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const S *qrow[2];
    const S *prow[RT];
    v4f acc[RT][2];
    float nrm[RT];
    const int64_t ad = orig_of(a.aorig, unit.x);
#pragma unroll
    for (int j = 0; j < 2; j++) qrow[j] = (const S *)a.x + (int64_t)a.perm[unit.y + min(16 * j + (lane & 15), unit.z - 1)] * a.ldx;
#pragma unroll
    for (int i = 0; i < RT; i++) {
        const int j = min(16 * i + (lane & 15), a.r - 1);
        prow[i] = (const S *)a.a + (ad * a.r + j) * a.d;
        acc[i][0] = acc[i][1] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
    }
    int bad = 0;
    if (a.flags.rows) {
        const int64_t per = 64 * (a.side.kpad / 8), lo = unit.x * a.flags.rows / 64 * per / 1024, hi = (((unit.x + 1) * a.flags.rows - 1) / 64 + 1) * per - 1;
        for (int64_t b = lo + threadIdx.x; b <= hi / 1024; b += 64 * NW) bad |= a.flags.found[b];
    }
    const int steps = (a.d + 4 * FewLoad<S>::CH - 1) / (4 * FewLoad<S>::CH);
    few_dot<S, S, RT, 2, VEC, false>(prow, qrow, steps * wave / NW, steps * (wave + 1) / NW, a.d, lane, acc, nrm);
    if (wave)
#pragma unroll
        for (int i = 0; i < RT; i++)
#pragma unroll
            for (int j = 0; j < 2; j++)
#pragma unroll
                for (int e = 0; e < 4; e++) part[wave - 1][16 * j + (lane & 15)][16 * i + 4 * (lane >> 4) + e] = acc[i][j][e];
    __syncthreads();
    if (wave == 0) {
        const float sc = a.scale ? a.scale[orig_of(a.orig, unit.x)] : 1.0f;
#pragma unroll
        for (int i = 0; i < RT; i++)
#pragma unroll
            for (int j = 0; j < 2; j++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    float *p = &part[0][16 * j + (lane & 15)][16 * i + 4 * (lane >> 4) + e];
                    constexpr int W = UNIT_ROWS * (16 * RT + 1);
                    float x = acc[i][j][e];
#pragma unroll
                    for (int w = 0; w < NW - 1; w++) x += p[w * W];
                    *p = x * sc;
                }
    }
    bad = __syncthreads_or(bad);
    if (a.flags.rows && threadIdx.x == 0) a.flags.bad[unit.x] = bad;  // (all of the adapter's units write the same)
    if (a.u)
        for (int t = threadIdx.x; t < unit.z * a.r; t += 64 * NW) {
            const int i = t / a.r, j = t - i * a.r;
            a.u[(int64_t)(unit.y + i) * a.r + j] = part[0][i][j];
        }
    if (!a.up) return;
    if (a.side.mode == SIDE_F32) {
        const int k = a.side.kpad / 2;
        for (int t = threadIdx.x; t < unit.z * k; t += 64 * NW) {
            const int i = t / k, j = t - i * k;
            ((float *)a.up)[(int64_t)(unit.y + i) * k + j] = j < a.r ? part[0][i][j] : 0.0f;
        }
        return;
    }
    for (int t = threadIdx.x; t < unit.z * a.side.kpad; t += 64 * NW) {
        const int i = t / a.side.kpad, k = t - i * a.side.kpad;
        a.up[(int64_t)(unit.y + i) * a.side.kpad + k] = side_piece<true>(a.side, k, [&](int j) { return part[0][i][j]; });
    }
}

template <class S>
static int shrink_launch(const ShrinkArgs &a, const ShrinkArgs *two, int64_t units, bool vec, hipStream_t s)
{
    const dim3 grid((unsigned)units, two ? 2 : 1);
    const ShrinkArgs &b = two ? *two : a;
    // (four waves where eight would not have the registers)
#define RAIRS_SHRINK(RT_, NW_)                                                                            \
    if (vec) hipLaunchKernelGGL((shrink_kernel<S, RT_, NW_, true>), grid, dim3(64 * NW_), 0, s, a, b);       \
    else hipLaunchKernelGGL((shrink_kernel<S, RT_, NW_, false>), grid, dim3(64 * NW_), 0, s, a, b)
    if (a.r <= 16) { RAIRS_SHRINK(1, 8); }
    else if (a.r <= 32) { RAIRS_SHRINK(2, 8); }
    else if (a.r <= 64) { RAIRS_SHRINK(4, 4); }
    else { RAIRS_SHRINK(8, 4); }
#undef RAIRS_SHRINK
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

// ---- what is laid out before the products ---------------------------------------------------------------

// row a * rows + o of dst: src[a * batch + o * so + j * sj], j < r, as the side wants it; and the row of zeros
struct SideJob {
    const void *src;
    int64_t batch, so, sj, rows, total;
    Side side;
    __bf16 *dst, *zero;
    uint32_t *found;
    const int32_t *orig;            // of row block a; null: a
};

template <class S>
static __device__ __forceinline__ void pack_side(const SideJob &j, int64_t block)
{
    const Side &side = j.side;
    if (block == 0)
        for (int k = threadIdx.x; k < side.kpad; k += 1024) j.zero[k] = (__bf16)0.0f;
    // a thread per eight values; the rows of a group of 64 first, so that a transposed source is read along its rows
    const int eights = side.kpad / 8;
    const int64_t id = block * 1024 + threadIdx.x, t = id / (64 * eights) * 64 + (id & 63);
    int odd = 0;
    if (t < j.total) {
        const int k0 = (int)(id / 64 % eights) * 8;
        const int64_t a = t / j.rows, o = t - a * j.rows;
        const S *p = (const S *)j.src + orig_of(j.orig, a) * j.batch + o * j.so;
        const auto at = [&](int w) {
            const float x = (float)p[w * j.sj];
            const bool finite = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
            odd |= !finite;
            return finite ? x : 0.0f;
        };
        if (side.mode == SIDE_F32) {
            v4f x;
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = k0 / 2 + e < side.r ? at(k0 / 2 + e) : 0.0f;
            *(v4f *)(j.dst + t * side.kpad + k0) = x;
        } else {
            v8bf x;
#pragma unroll
            for (int e = 0; e < 8; e++) x[e] = side_piece<false>(side, k0 + e, at);
            *(v8bf *)(j.dst + t * side.kpad + k0) = x;
        }
    }
    odd = __syncthreads_or(odd);
    if (threadIdx.x == 0) j.found[block] = odd;
}

// dst[b][c][r] = src[orig b][r][c], 32 x 32 values
template <class S>
static __device__ __forceinline__ void transpose_tile(S (&tile)[32][33], const S *__restrict__ src, int rows, int cols, S *__restrict__ dst,
                                                      int64_t block, const int32_t *__restrict__ orig)
{
    const int rt = (rows + 31) / 32, ct = (cols + 31) / 32;
    const int64_t b = block / (rt * ct), batch = b * rows * cols, from = orig_of(orig, b) * rows * cols;
    const int in = (int)(block % (rt * ct)), r0 = in % rt * 32, c0 = in / rt * 32, x = threadIdx.x & 31, y = threadIdx.x >> 5;
    if (r0 + y < rows && c0 + x < cols) tile[y][x] = src[from + (int64_t)(r0 + y) * cols + c0 + x];
    __syncthreads();
    if (c0 + y < cols && r0 + x < rows) dst[batch + (int64_t)(c0 + y) * rows + r0 + x] = tile[x][y];
}

// The sort, which is one workgroup's, and beside it what does not wait for it: the adapters' B (or A) as pieces, W
// turned, B turned.  One launch after the other they took 20 us more (2,999 rows, 1024 x 960, 32 adapters).
#define PREP_MOST (1 << 20)
struct PrepArgs {
    SortView sort;
    int sorts;                      // workgroups: 0 or 1
    unsigned side_blocks, cols_blocks, turn_blocks;
    int64_t side_from, turn_from;   // where this launch goes on: of either at most PREP_MOST at a time, as a grid has less than 2^32 threads
    PackJobs rows;                  // W (forward) and the batch, in the batch's order
    SideJob side;
    const void *w, *b;              // [d_out][d_in], [na][d_out][r]
    const int32_t *orig;            // of b's, null: as they are
    int d_in, d_out, r, vec;
    __bf16 *wt;
    int64_t opad;
    PackLayout wto;
    void *bt;
};

template <class S, int NP>
__global__ __launch_bounds__(1024) void prep_kernel(PrepArgs a)
{
    extern __shared__ __align__(16) char prep_lds[];
    int64_t block = blockIdx.x;
    if (block < a.sorts) {
        sort_one(a.sort, (int32_t *)prep_lds);
        return;
    }
    block -= a.sorts;
    if (block < a.side_blocks) {
        pack_side<S>(a.side, block + a.side_from);
        return;
    }
    block -= a.side_blocks;
    if (block < a.cols_blocks) {
        const int half = threadIdx.x >> 9;
        const int64_t rt = a.opad / 64, ct = (a.d_in + 63) / 64, t = block * 2 + half;
        PackCols<S, NP> *sh = (PackCols<S, NP> *)prep_lds;
        pack_cols_tile<S, NP, 512>(sh[half], threadIdx.x & 511, t < rt * ct, (const S *)a.w, a.d_in, a.d_out, a.d_in, ORDER_SAME, a.vec, a.wt, a.opad,
                                   a.wto, t % rt * 64, t / rt * 64, [](int64_t) { return true; });
        return;
    }
    block -= a.cols_blocks;
    for (int i = 0; i < a.rows.n; i++) {
        if (block < a.rows.job[i].blocks) {
            pack_rows_job<S, NP, 1024>(a.rows.job[i], block);
            return;
        }
        block -= a.rows.job[i].blocks;
    }
    transpose_tile<S>(*(S(*)[32][33])prep_lds, (const S *)a.b, a.d_out, a.r, (S *)a.bt, block + a.turn_from, a.orig);
}

// The batch as an operand, to be taken through a permutation that is not known yet: laid out beside the sort, where 32-bit
// offsets reach all of its rows then; false: it is laid out after it.
static bool batch_operand(const void *x, int dtype, int64_t ld, int64_t n, int64_t cols, const int32_t *perm, __bf16 *room, RowOperand &out, PackJobs &jobs)
{
    PackJobs mine = {};
    rairs_operand_job(x, dtype, ld, n, cols, dtype == RAIRS_F32, room, out, mine);
    if (n * out.ld >= (1ll << 31)) return false;
    if (mine.n) jobs.job[jobs.n++] = mine.job[0];
    out.perm = perm;
    return true;
}

static int prep_launch(PrepArgs &a, int dtype, hipStream_t s)
{
    int rc = RAIRS_OK;
    size_t lds = 0;
    if (a.sort.n) {
        a.sorts = sorts_in_one(a.sort);
        if (a.sorts) lds = sort_one_lds(a.sort);
        else if ((rc = sort_launch(a.sort, s))) return rc;
    }
    int64_t side_work = 0, turn_work = 0;
    if (a.side.dst) side_work = side_blocks(a.side.side, a.side.total);
    if (a.wt) {
        a.cols_blocks = (unsigned)((a.opad / 64 * ((a.d_in + 63) / 64) + 1) / 2);
        lds = std::max(lds, dtype == RAIRS_F32 ? 2 * sizeof(PackCols<float, 3>) : 2 * sizeof(PackCols<__bf16, 1>));
        a.vec = is_vec(a.w, a.d_in, dtype_width(dtype));
    }
    if (a.bt) {
        turn_work = (int64_t)((a.d_out + 31) / 32 * ((a.r + 31) / 32)) * a.sort.na;
        lds = std::max(lds, sizeof(float) * 32 * 33);
    }
    for (int i = 0; i < a.rows.n; i++) {
        PackJob &j = a.rows.job[i];
        j.blocks = (unsigned)std::min<int64_t>((j.rows * (j.pad / 8) + 1023) / 1024, 2048);
        j.vec = is_vec(j.src, j.ld, dtype_width(dtype));
    }
    if (dtype == RAIRS_F32) RAIRS_HIP(hipFuncSetAttribute((const void *)prep_kernel<float, 3>, hipFuncAttributeMaxDynamicSharedMemorySize, SORT_ONE_LDS));   // (the same for every call)
    else RAIRS_HIP(hipFuncSetAttribute((const void *)prep_kernel<__bf16, 1>, hipFuncAttributeMaxDynamicSharedMemorySize, SORT_ONE_LDS));
    for (;;) {
        a.side_blocks = (unsigned)std::min<int64_t>(side_work - a.side_from, PREP_MOST);
        a.turn_blocks = (unsigned)std::min<int64_t>(turn_work - a.turn_from, PREP_MOST);
        unsigned blocks = a.sorts + a.side_blocks + a.cols_blocks + a.turn_blocks;
        for (int i = 0; i < a.rows.n; i++) blocks += a.rows.job[i].blocks;
        if (!blocks) return RAIRS_OK;
        if (dtype == RAIRS_F32) hipLaunchKernelGGL((prep_kernel<float, 3>), dim3(blocks), dim3(1024), lds, s, a);
        else hipLaunchKernelGGL((prep_kernel<__bf16, 1>), dim3(blocks), dim3(1024), lds, s, a);
        RAIRS_HIP(hipGetLastError());
        // (what is left of the most adapters' values)
        a.sorts = 0;
        a.cols_blocks = 0;
        a.rows.n = 0;
        a.side_from += a.side_blocks;
        a.turn_from += a.turn_blocks;
    }
}

// ---- a few rows ----------------------------------------------------------------------------------------

struct FewProjectArgs {
    const void *x, *w, *a, *b;
    int64_t ldx, ldy, n;
    int d_in, d_out, r, na;
    const int32_t *adapter;         // null: none
    const float *scale;
    float *u;                       // [n][r]; null: a workgroup makes its rows' own (up to 16 rows)
    int avec;
    void *y;
    int bf16_out;
};

// u[row][j] of adapter ad by a wave, in every lane
template <class S>
static __device__ __forceinline__ float few_u(const FewProjectArgs &a, int64_t row, int ad, int j, int lane)
{
    constexpr int CH = FewLoad<S>::CH;
    const S *x = (const S *)a.x + row * a.ldx, *w = (const S *)a.a + ((int64_t)ad * a.r + j) * a.d_in;
    float s = 0.0f;
    for (int k = lane * CH; k < a.d_in; k += 64 * CH) {
        const FewFrag<S, CH> f = a.avec ? few_load<S, CH, true>(x, k, a.d_in) : few_load<S, CH, false>(x, k, a.d_in);
        const FewFrag<S, CH> g = a.avec ? few_load<S, CH, true>(w, k, a.d_in) : few_load<S, CH, false>(w, k, a.d_in);
#pragma unroll
        for (int e = 0; e < CH; e++) s = fmaf((float)f.e[e], (float)g.e[e], s);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    return a.scale ? s * a.scale[ad] : s;
}

// u: a wave per row and rank
template <class S>
__global__ __launch_bounds__(WG) void few_shrink_kernel(FewProjectArgs a)
{
    const int lane = threadIdx.x & 63, j = blockIdx.y * (WG / 64) + (threadIdx.x >> 6);
    const int64_t row = blockIdx.x;
    const int ad = a.adapter[row];
    if (j >= a.r || ad < 0 || ad >= a.na) return;
    const float s = few_u<S>(a, row, ad, j, lane);
    if (lane == 0) a.u[row * a.r + j] = s;
}

// (1 row, 768 to 128, rank 8: 8.5 us in one launch, 5.4 and 3.8 in two; 100 rows, 1024 to 960, rank 16: 4.3 and 8.7 us:
// the latency of a row's loads, a chain of about four round trips.)
// 16 PT columns of y for 64 rows per workgroup: its waves share the sum over d_in, then each finishes one tile of 16
// rows.  The low-rank part is a row's own: its u against the columns' rows of its adapter's B, on the vector units.
template <class S, int PT, int QT, bool VEC, bool BVEC>
__global__ __launch_bounds__(WG) void few_project_kernel(FewProjectArgs a)
{
    __shared__ v4f part[4][PT][QT][64];
    __shared__ float own_u[QT == 1 ? 16 : 1][QT == 1 ? RAIRS_MAX_RANK : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // workgroups go round robin over the eight XCDs: the ones that read the same rows (of x, or of W if there are
    // fewer rows of x) one after the other on one of them, whose L2 cache has them after the first
    const int pt = (a.d_out + 16 * PT - 1) / (16 * PT), qt = (int)((a.n + 16 * QT - 1) / (16 * QT)), total = pt * qt, per = (total + 7) / 8;
    const int id = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
    if ((int)(blockIdx.x / 8) >= per || id >= total) return;
    const bool rows_first = a.n < a.d_out;
    const int p0 = (rows_first ? id / qt : id % pt) * 16 * PT;
    const int64_t q0 = (int64_t)(rows_first ? id % qt : id / pt) * 16 * QT;
    const S *prow[PT];
    const S *qrow[QT];
    v4f acc[PT][QT];
    float nrm[PT];
#pragma unroll
    for (int i = 0; i < PT; i++) prow[i] = (const S *)a.w + (int64_t)min(p0 + 16 * i + (lane & 15), a.d_out - 1) * a.d_in;
#pragma unroll
    for (int j = 0; j < QT; j++) {
        const int64_t q = min(q0 + 16 * j + (lane & 15), a.n - 1);
        qrow[j] = (const S *)a.x + q * a.ldx;
#pragma unroll
        for (int i = 0; i < PT; i++) acc[i][j] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int steps = (a.d_in + 4 * FewLoad<S>::CH - 1) / (4 * FewLoad<S>::CH);
    few_dot<S, S, PT, QT, VEC, false>(prow, qrow, steps * wave / 4, steps * (wave + 1) / 4, a.d_in, lane, acc, nrm);
#pragma unroll
    for (int i = 0; i < PT; i++)
#pragma unroll
        for (int j = 0; j < QT; j++) part[wave][i][j][lane] = acc[i][j];
    if constexpr (QT == 1)
        if (a.adapter && !a.u)
            for (int t = wave; t < (int)a.n * a.r; t += 4) {
                const int row = t / a.r, j = t - row * a.r, ad = a.adapter[row];
                if (ad < 0 || ad >= a.na) continue;
                const float x = few_u<S>(a, row, ad, j, lane);
                if (lane == 0) own_u[row][j] = x;
            }
    __syncthreads();
    if (wave >= QT) return;
    const int64_t q = q0 + 16 * wave + (lane & 15);
    if (q >= a.n) return;
    const int ad = a.adapter ? a.adapter[q] : -1;
    const bool own = ad >= 0 && ad < a.na;
    constexpr int CH = FewLoad<S>::CH;
#pragma unroll
    for (int i = 0; i < PT; i++) {
        v4f y = (part[0][i][wave][lane] + part[1][i][wave][lane]) + (part[2][i][wave][lane] + part[3][i][wave][lane]);
        const int o0 = p0 + 16 * i + 4 * (lane >> 4);
        if (own) {
            const float *u = QT == 1 && !a.u ? own_u[q & 15] : a.u + q * a.r;
            const S *b = (const S *)a.b + (int64_t)ad * a.d_out * a.r;
            v4f z = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int j = 0; j < a.r; j += CH) {
                FewFrag<S, CH> f[4];
                FewFrag<float, CH> uv;                                // (BVEC: the rank is a multiple of CH)
                if constexpr (BVEC) uv = few_load<float, CH, true>(u, j, a.r);
#pragma unroll
                for (int e = 0; e < 4; e++) f[e] = few_load<S, CH, BVEC>(b + (int64_t)min(o0 + e, a.d_out - 1) * a.r, j, a.r);
#pragma unroll
                for (int w = 0; w < CH; w++) {
                    const float uj = BVEC ? uv.e[w] : j + w < a.r ? u[j + w] : 0.0f;
#pragma unroll
                    for (int e = 0; e < 4; e++) z[e] = fmaf((float)f[e].e[w], uj, z[e]);
                }
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
}

static bool row_vec(const void *p, int64_t ld, int dtype) { return (uintptr_t)p % 16 == 0 && ld * dtype_width(dtype) % 16 == 0; }

template <class S, int PT, int QT>
static void few_project_launch(const FewProjectArgs &a, bool vec, bool bvec, hipStream_t s)
{
    const int64_t total = (a.d_out + 16 * PT - 1) / (16 * PT) * ((a.n + 16 * QT - 1) / (16 * QT));
    const dim3 grid((unsigned)(pad_to(total, 8)));
    if (vec && bvec) hipLaunchKernelGGL((few_project_kernel<S, PT, QT, true, true>), grid, dim3(WG), 0, s, a);
    else if (vec) hipLaunchKernelGGL((few_project_kernel<S, PT, QT, true, false>), grid, dim3(WG), 0, s, a);
    else hipLaunchKernelGGL((few_project_kernel<S, PT, QT, false, false>), grid, dim3(WG), 0, s, a);
}

template <class S>
static int few_project(const FewProjectArgs &a, int dtype, hipStream_t s)
{
    const bool vec = row_vec(a.x, a.ldx, dtype) && row_vec(a.w, a.d_in, dtype), bvec = a.adapter && row_vec(a.b, a.r, dtype);
    // two tiles of columns where that leaves two workgroups for every CU
    if (a.n <= 16) few_project_launch<S, 1, 1>(a, vec, bvec, s);
    else if (a.n <= 32) few_project_launch<S, 1, 2>(a, vec, bvec, s);
    else if ((int64_t)((a.d_out + 31) / 32) * ((a.n + 63) / 64) < 512) few_project_launch<S, 1, 4>(a, vec, bvec, s);
    else few_project_launch<S, 2, 4>(a, vec, bvec, s);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

template <class S>
static int few_shrink(const FewProjectArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL(few_shrink_kernel<S>, dim3((unsigned)a.n, (unsigned)((a.r + 3) / 4)), dim3(WG), 0, s, a);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

// ---- forward -------------------------------------------------------------------------------------------

// Stores a tile and adds to its rows what their adapters' values that are not finite make of u (seldom).
template <class S>
struct AdapterEpi : StoreEpi {
    const int32_t *of_row;
    const uint32_t *bad;
    const S *src;                   // as in SideJob
    int64_t batch, so, sj;
    const __bf16 *u;
    Side side;
    const int32_t *orig;
    template <class T>
    struct State : StoreEpi::State<T> {
        uint32_t odd;               // of this lane's rows
    };
    template <class T>
    __device__ __forceinline__ void begin(State<T> &st, int64_t q0, int lane) const
    {
        StoreEpi::begin<T>(st, q0, lane);
        st.odd = 0;
#pragma unroll
        for (int j = 0; j < T::QT; j++) {
            const int64_t q = q0 + 16 * j + (lane & 15);
            const int ad = q < nq ? of_row[q] : -1;
            if (ad >= 0 && bad[ad]) st.odd |= 1u << j;
        }
    }
    __device__ __forceinline__ float u_at(int64_t q, int j) const
    {
        const __bf16 *p = u + q * side.kpad;
        if (side.mode == SIDE_F32) return ((const float *)p)[j];
        if (side.mode == SIDE_THREES) p += j / 32 * 96 + j % 32;
        else p += j;
        const int step = side.mode == SIDE_THREES ? 32 : side.r;
        return ((float)p[0] + (float)p[step]) + (float)p[2 * step];
    }
    template <class T>
    __device__ __forceinline__ void end(State<T> &st, int run, int wp, int64_t q0, int lane) const
    {
        if (!__any(st.odd)) return;
#pragma unroll 1
        for (int j = 0; j < T::QT; j++) {
            if (!((st.odd >> j) & 1u)) continue;
            const int64_t q = q0 + 16 * j + (lane & 15), row = perm ? perm[q] : q;
            const S *b = src + orig_of(orig, of_row[q]) * batch;
#pragma unroll 1
            for (int i = 0; i < 4 * T::PT; i++) {
                // (a run is one tile; the lane that stored a value adds to it)
                const int64_t p = (int64_t)run * T::BP + wp * (16 * T::PT) + 16 * (i / 4) + 4 * (lane >> 4) + i % 4;
                if (p >= np) continue;
                float x = 0.0f;
                bool any = false;
#pragma unroll 1
                for (int k = 0; k < side.r; k++) {
                    const float v = (float)b[p * so + k * sj];
                    if ((__float_as_uint(v) & 0x7F800000u) != 0x7F800000u) continue;
                    x = fmaf(v, u_at(q, k), x);
                    any = true;
                }
                if (!any) continue;
                if (bf16_out) ((__bf16 *)out)[row * ld + p] = (__bf16)((float)((__bf16 *)out)[row * ld + p] + x);
                else ((float *)out)[row * ld + p] += x;
            }
        }
    }
};

static int large_product(RowProd &rp, const StoreEpi &e, bool bf, bool f32, const SideJob *job, const __bf16 *u, const uint32_t *bad, hipStream_t s)
{
    if (!job) {
        if (f32) return rowprod_launch<TileS, ROW_F32>(rp, e, s);
        return bf ? rowprod_launch_any(rp, e, s) : rowprod_launch_any<ROW_THREES>(rp, e, s);
    }
    if (bf) {
        const AdapterEpi<__bf16> ae = {e, rp.ad.of_row, bad, (const __bf16 *)job->src, job->batch, job->so, job->sj, u, job->side, job->orig};
        return rowprod_launch_any<ROW_ADAPT>(rp, ae, s);
    }
    const AdapterEpi<float> ae = {e, rp.ad.of_row, bad, (const float *)job->src, job->batch, job->so, job->sj, u, job->side, job->orig};
    return f32 ? rowprod_launch<TileS, ROW_F32 | ROW_ADAPT>(rp, ae, s) : rowprod_launch_any<ROW_THREES | ROW_ADAPT>(rp, ae, s);
}

// Rows straight from memory: up to 64 of them, or 256 where what the workgroups read of W and x (a lane's 16 bytes are a
// cache access each: about 10 TB/s) takes less than the launches of the other way, 20 us, or with adapters
// 40: a tile runs over all that its rows have.  This way / the other, us, rank 16: 64 x 4096 x 4096 bf16 23 / 23 and
// with 32 adapters 30 / 86; 256 x 1024 x 1024 bf16 15 / 17 and 20 / 37; 128 x 2048 x 2048 fp32 27 / 46 and with 100 36 / 139.
static bool few_rows(const rairs_projection_t &p, int64_t n)
{
    const double read = (double)((n + 63) / 64) * ((p.d_out + 31) / 32) * 96.0 * p.d_in * dtype_width(p.dtype);
    return n <= 64 || (n <= FEW_ROWS && read < (p.n_adapters ? 400e6 : 200e6));
}

int rairs_run_project(const ProjectArgs &g, void *ws, size_t *bytes, hipStream_t s)
{
    const rairs_projection_t &p = g.p;
    const bool adapters = p.n_adapters > 0, bf = p.dtype == RAIRS_BF16;
    Carve w(ws);
    int rc = RAIRS_OK;
    if (few_rows(p, g.n)) {
        FewProjectArgs a = {};
        // (every workgroup for itself where that reads no more than 128 KB: less than a launch)
        const bool own = g.n <= 16 && g.n * p.rank * p.d_in * dtype_width(p.dtype) <= 128 * 1024;
        a.u = adapters && !own ? w.take<float>(g.n * p.rank) : nullptr;
        if (bytes) *bytes = w.used;
        if (!ws) return RAIRS_OK;
        a.x = g.x; a.w = p.W; a.a = p.A; a.b = p.B;
        a.ldx = g.ldx; a.ldy = g.ldy; a.n = g.n;
        a.d_in = p.d_in; a.d_out = p.d_out; a.r = p.rank; a.na = p.n_adapters;
        a.adapter = adapters ? g.adapter : nullptr;
        a.scale = p.scale; a.y = g.y; a.bf16_out = g.ytype == RAIRS_BF16;
        a.avec = row_vec(g.x, g.ldx, p.dtype) && row_vec(p.A, p.d_in, p.dtype);
        if (a.adapter && !own && (rc = bf ? few_shrink<__bf16>(a, s) : few_shrink<float>(a, s))) return rc;
        return bf ? few_project<__bf16>(a, p.dtype, s) : few_project<float>(a, p.dtype, s);
    }
    const int np = dtype_pieces(p.dtype);
    __bf16 *xroom = w.take<__bf16>(pack_room(p.dtype, g.n, p.d_in)), *wroom = w.take<__bf16>(pack_room(p.dtype, p.d_out, p.d_in));
    SortView sv = {};
    UsedView used = {};
    int na = p.n_adapters;          // or how many of them are laid out
    Side side = {};
    SideFlags flags = {};
    __bf16 *up = nullptr, *bp = nullptr, *zero = nullptr;
    // fp32 rows that lie right, and too few of them for large tiles: as they are
    const bool f32 = rowprod_size(p.d_out, g.n) == 0 && f32_lies_right(p.W, p.dtype, p.d_in, p.d_in) &&
                     f32_lies_right(g.x, p.dtype, g.ldx, p.d_in) && g.n * g.ldx < (1ll << 30);
    if (adapters) {
        side = side_of(bf ? SIDE_BF16 : f32 ? SIDE_F32 : SIDE_THREES, p.rank);
        // (the size does not depend on where the rows lie)
        const int room = bf ? side.kpad : side_of(SIDE_THREES, p.rank).kpad;
        if (numbers_used(p, g.n, 2ll * p.d_out * room)) {
            used = used_carve(w, p, g.adapter, g.n);
            na = used.most;
        }
        sv = sort_carve(w, used.na ? used.number : g.adapter, g.n, na);
        up = w.take<__bf16>(g.n * room);
        bp = w.take<__bf16>((int64_t)na * p.d_out * room);
        zero = w.take<__bf16>(room);
        flags.found = w.take<uint32_t>(side_blocks(Side{0, 0, room}, (int64_t)na * p.d_out));
        flags.bad = w.take<uint32_t>(na);
        flags.rows = p.d_out;
    }
    if (bytes) *bytes = w.used;
    if (!ws) return RAIRS_OK;

    const bool use = adapters && g.adapter;
    RowProd rp = {};
    const SideJob job = {p.B, (int64_t)p.d_out * p.rank, p.rank, 1, p.d_out, (int64_t)na * p.d_out, side, bp, zero, flags.found, used.orig};
    PackJobs jobs = {};
    bool late = false;
    if (!f32) {
        rairs_operand_job(p.W, p.dtype, p.d_in, p.d_out, p.d_in, !bf, wroom, rp.P, jobs);
        late = !batch_operand(g.x, p.dtype, g.ldx, g.n, p.d_in, use ? sv.perm : nullptr, xroom, rp.Q, jobs);
    }
    if (use) {
        if (used.na && (rc = used_launch(used, s))) return rc;
        PrepArgs pa = {};
        pa.sort = sv;
        pa.side = job;
        pa.rows = jobs;
        if ((rc = prep_launch(pa, p.dtype, s))) return rc;
    }
    if (f32) {
        rowprod_pieces(rp, 1, 1);
        rp.ksteps = p.d_in / (ROWPROD_K / 2);
        rp.P = f32_operand(p.W, p.d_in, p.d_out);
        rp.Q = f32_operand(g.x, g.ldx, g.n);
        rp.Q.perm = use ? sv.perm : nullptr;
    } else {
        rowprod_sums(rp, np, np, pad_to(p.d_in, bf ? ROWPROD_K : 32));
        if (!use && (rc = rairs_launch_pack(jobs, s))) return rc;
        if (late && (rc = rairs_operand(g.x, p.dtype, g.ldx, g.n, p.d_in, use ? sv.perm : nullptr, !bf, xroom, rp.Q, s))) return rc;
    }
    if (use) {
        ShrinkArgs sa = {g.x, p.A, g.ldx, p.d_in, p.rank, p.scale, sv.perm, sv.units, sv.unit0 + na, nullptr, up, side, flags, used.orig, used.orig};
        const int64_t units = max_units(g.n, na, UNIT_ROWS);
        const bool vec = row_vec(g.x, g.ldx, p.dtype) && row_vec(p.A, p.d_in, p.dtype);
        if ((rc = bf ? shrink_launch<__bf16>(sa, nullptr, units, vec, s) : shrink_launch<float>(sa, nullptr, units, vec, s))) return rc;
        rp.ad = AdapterPart{up, bp, zero, sv.of_row, sv.first + 1, side.kpad};
    }
    StoreEpi e = {g.y, g.ldy, 0, p.d_out, g.n, use ? sv.perm : nullptr, g.ytype == RAIRS_BF16, 0};
    return large_product(rp, e, bf, f32, use ? &job : nullptr, up, flags.bad, s);
}

// ---- backward ------------------------------------------------------------------------------------------

// Partial sums of an adapter's gradient over a chunk of its rows: sum_rows x[row][i] u[row][j], by the fp32
// matrix instruction (16 x 16 x 4), whose operands are rows as they lie: a lane takes 16 bytes of one of four
// rows, its values go into as many products (product t has columns CH c + t), and one rank of u.  Rows are
// rank-bound small change next to the projection; the fp32 rate is enough and nothing is rounded.  The
// workgroup's waves take every fourth four of rows and are joined in LDS.  (8,191 rows, 2048 + 2048 columns, rank 32: 45 us
// for both sides, 17 of them the instruction's; 2,999 rows, 1024 + 960, rank 8: 10 us.)
// part[chunk][j][i], or turned [chunk][i][j].
struct AdapterGradArgs {            // of A: x and v; of B (turned): dy and u
    const void *x[2];
    int64_t ldx[2];
    const float *u[2];
    int cols[2];
    float *part[2];
    void *out[2];
    const int32_t *perm, *chunk0;
    const int4 *chunks;
    int r, na;
    const int32_t *of;              // number of an adapter, -1: it has no rows; null: its own
};

template <class S, int RT, bool VEC>
__global__ __launch_bounds__(WG) void adapter_grad_kernel(AdapterGradArgs a)
{
    const int r = a.r, rts = (r + 16 * RT - 1) / (16 * RT), turned = (int)blockIdx.z / rts, cols = a.cols[turned];
    const S *__restrict__ x = (const S *)a.x[turned];
    const float *__restrict__ u = a.u[turned];
    const int64_t ldx = a.ldx[turned];
    const int32_t *__restrict__ perm = a.perm;
    if ((int)blockIdx.y * 16 * FewLoad<S>::CH >= cols) return;
    constexpr int CH = FewLoad<S>::CH;
    __shared__ v4f sums[3][CH * RT][64];
    if ((int)blockIdx.x >= a.chunk0[a.na]) return;
    const int4 ch = a.chunks[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, h = lane >> 4;
    const int i0 = (blockIdx.y * 16 + c) * CH, j0 = ((int)blockIdx.z - turned * rts) * 16 * RT;
    v4f acc[CH][RT];
#pragma unroll
    for (int t = 0; t < CH; t++)
#pragma unroll
        for (int j = 0; j < RT; j++) acc[t][j] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int AHEAD = 4;                                          // fours of rows on the way
    for (int k0 = wave * 4; k0 < ch.z; k0 += 16 * AHEAD) {
        FewFrag<S, CH> f[AHEAD];
        float v[AHEAD][RT];
        int64_t row[AHEAD];
#pragma unroll
        for (int w = 0; w < AHEAD; w++) row[w] = perm[ch.y + min(k0 + 16 * w + h, ch.z - 1)];
#pragma unroll
        for (int w = 0; w < AHEAD; w++) {
            const int k = min(k0 + 16 * w + h, ch.z - 1);
            f[w] = few_load<S, CH, VEC>(x + row[w] * ldx, i0, cols);
#pragma unroll
            for (int j = 0; j < RT; j++) v[w][j] = u[(int64_t)(ch.y + k) * r + min(j0 + 16 * j + c, r - 1)];
        }
#pragma unroll
        for (int w = 0; w < AHEAD; w++) {
            const bool in = k0 + 16 * w + h < ch.z;
#pragma unroll
            for (int t = 0; t < CH; t++)
#pragma unroll
                for (int j = 0; j < RT; j++)
                    acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? (float)f[w].e[t] : 0.0f, in ? v[w][j] : 0.0f, acc[t][j], 0, 0, 0);
        }
    }
    if (wave)
#pragma unroll
        for (int t = 0; t < CH; t++)
#pragma unroll
            for (int j = 0; j < RT; j++) sums[wave - 1][t * RT + j][lane] = acc[t][j];
    __syncthreads();
    if (wave) return;
    float *o = a.part[turned] + (int64_t)blockIdx.x * r * cols;
#pragma unroll
    for (int t = 0; t < CH; t++)
#pragma unroll
        for (int j = 0; j < RT; j++) {
            const v4f y = (acc[t][j] + sums[0][t * RT + j][lane]) + (sums[1][t * RT + j][lane] + sums[2][t * RT + j][lane]);
            const int rank = j0 + 16 * j + c;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int i = (blockIdx.y * 16 + 4 * h + e) * CH + t;
                if (rank < r && i < cols) o[turned ? (int64_t)i * r + rank : (int64_t)rank * cols + i] = y[e];
            }
        }
}

// an adapter's gradient: its chunks' sums in their order (both lie alike)
template <class S>
__global__ __launch_bounds__(WG) void adapter_join_kernel(AdapterGradArgs g)
{
    const int a = blockIdx.y;
    const int64_t size = (int64_t)g.r * g.cols[blockIdx.z], t = (int64_t)blockIdx.x * WG + threadIdx.x;
    if (t >= size) return;
    const float *part = g.part[blockIdx.z];
    float x = 0.0f;
    const int k = g.of ? g.of[a] : a;
    if (k >= 0)
        for (int c = g.chunk0[k]; c < g.chunk0[k + 1]; c++) x += part[c * size + t];
    ((S *)g.out[blockIdx.z])[a * size + t] = (S)x;
}

template <class S>
static int adapter_grads(const ProjectArgs &g, const SortView &sv, const int32_t *of, const float *u, const float *v, float *apart, float *bpart, hipStream_t s)
{
    const rairs_projection_t &p = g.p;
    const unsigned chunks = (unsigned)max_units(g.n, sv.na, CHUNK_ROWS);
    const int rt = p.rank <= 16 ? 1 : 2, most = std::max(p.d_in, p.d_out);
    const AdapterGradArgs a = {{g.x, g.dy}, {g.ldx, g.lddy}, {v, u}, {p.d_in, p.d_out}, {apart, bpart}, {g.da, g.db}, sv.perm, sv.chunk0, sv.chunks,
                               p.rank, sv.na, of};
    const dim3 grid(chunks, (unsigned)((most + 16 * FewLoad<S>::CH - 1) / (16 * FewLoad<S>::CH)), 2 * (unsigned)((p.rank + 16 * rt - 1) / (16 * rt)));
    const bool vec = row_vec(g.x, g.ldx, p.dtype) && row_vec(g.dy, g.lddy, p.dtype);
    if (rt == 1 && vec) hipLaunchKernelGGL((adapter_grad_kernel<S, 1, true>), grid, dim3(WG), 0, s, a);
    else if (rt == 1) hipLaunchKernelGGL((adapter_grad_kernel<S, 1, false>), grid, dim3(WG), 0, s, a);
    else if (vec) hipLaunchKernelGGL((adapter_grad_kernel<S, 2, true>), grid, dim3(WG), 0, s, a);
    else hipLaunchKernelGGL((adapter_grad_kernel<S, 2, false>), grid, dim3(WG), 0, s, a);
    hipLaunchKernelGGL(adapter_join_kernel<S>, dim3((unsigned)(((int64_t)p.rank * most + WG - 1) / WG), (unsigned)p.n_adapters, 2), dim3(WG), 0, s, a);
    RAIRS_HIP(hipGetLastError());
    return RAIRS_OK;
}

int rairs_run_project_backward(const ProjectArgs &g, void *ws, size_t *bytes, hipStream_t s)
{
    const rairs_projection_t &p = g.p;
    const int np = dtype_pieces(p.dtype);
    const bool adapters = p.n_adapters > 0, bf = p.dtype == RAIRS_BF16;
    UsedView used = {};
    int na = p.n_adapters;          // or how many of them are laid out
    const int64_t opad = pad_to(p.d_out, ROWPROD_K);
    Carve w(ws);
    __bf16 *yroom = w.take<__bf16>(pack_room(p.dtype, g.n, p.d_out)), *wt = w.take<__bf16>((int64_t)p.d_in * opad * np);
    SortView sv = {};
    Side side = {};
    SideFlags flags = {};
    __bf16 *vp = nullptr, *ap = nullptr, *zero = nullptr;
    float *u = nullptr, *v = nullptr, *apart = nullptr, *bpart = nullptr;
    char *bt = nullptr;
    if (adapters) {
        side = side_of(bf ? SIDE_BF16 : SIDE_THREES, p.rank);
        // (A as pieces, B turned)
        if (g.n > 0 && numbers_used(p, g.n, 2ll * p.d_in * side.kpad + (int64_t)p.d_out * p.rank * dtype_width(p.dtype))) {
            used = used_carve(w, p, g.adapter, g.n);
            na = used.most;
        }
        sv = sort_carve(w, used.na ? used.number : g.adapter, g.n, na);
        vp = w.take<__bf16>(g.n * side.kpad);
        ap = w.take<__bf16>((int64_t)na * p.d_in * side.kpad);
        zero = w.take<__bf16>(side.kpad);
        flags.found = w.take<uint32_t>(side_blocks(side, (int64_t)na * p.d_in));
        flags.bad = w.take<uint32_t>(na);
        flags.rows = g.dx ? p.d_in : 0;
        u = w.take<float>(g.n * p.rank);
        v = w.take<float>(g.n * p.rank);
        bt = w.take<char>((int64_t)na * p.rank * p.d_out * dtype_width(p.dtype));
        apart = w.take<float>(max_units(g.n, na, CHUNK_ROWS) * p.rank * p.d_in);
        bpart = w.take<float>(max_units(g.n, na, CHUNK_ROWS) * p.rank * p.d_out);
    }
    if (bytes) *bytes = w.used;
    if (!ws) return RAIRS_OK;

    const bool use = adapters && g.adapter && g.n > 0;
    const PackLayout wto = pack_layout(p.d_in, opad, !bf);
    int rc = RAIRS_OK;
    const SideJob job = {p.A, (int64_t)p.rank * p.d_in, 1, p.d_in, p.d_in, (int64_t)na * p.d_in, side, ap, zero, flags.found, used.orig};
    RowProd rp = {};
    PackJobs jobs = {};
    bool late = false;
    if (g.dx && g.n > 0) late = !batch_operand(g.dy, p.dtype, g.lddy, g.n, p.d_out, use ? sv.perm : nullptr, yroom, rp.Q, jobs);
    if (use) {
        if (used.na && (rc = used_launch(used, s))) return rc;
        PrepArgs pa = {};
        pa.sort = sv;
        pa.rows = jobs;
        pa.b = p.B; pa.bt = bt; pa.orig = used.orig;
        pa.w = p.W; pa.d_in = p.d_in; pa.d_out = p.d_out; pa.r = p.rank; pa.opad = opad; pa.wto = wto;
        if (g.dx) {
            pa.wt = wt;
            pa.side = job;
        }
        if ((rc = prep_launch(pa, p.dtype, s))) return rc;
        const int64_t units = max_units(g.n, na, UNIT_ROWS);
        const ShrinkArgs sa = {g.dy, bt, g.lddy, p.d_out, p.rank, p.scale, sv.perm, sv.units, sv.unit0 + na, v, g.dx ? vp : nullptr, side, flags, used.orig, nullptr};
        const ShrinkArgs su = {g.x, p.A, g.ldx, p.d_in, p.rank, p.scale, sv.perm, sv.units, sv.unit0 + na, u, nullptr, side, {}, used.orig, used.orig};
        const bool vec = row_vec(g.dy, g.lddy, p.dtype) && row_vec(bt, p.d_out, p.dtype) &&
                         (!g.da || (row_vec(g.x, g.ldx, p.dtype) && row_vec(p.A, p.d_in, p.dtype)));
        if ((rc = bf ? shrink_launch<__bf16>(sa, g.da ? &su : nullptr, units, vec, s) : shrink_launch<float>(sa, g.da ? &su : nullptr, units, vec, s)))
            return rc;
        if (g.da && (rc = bf ? adapter_grads<__bf16>(g, sv, used.of, u, v, apart, bpart, s) : adapter_grads<float>(g, sv, used.of, u, v, apart, bpart, s))) return rc;
    } else if (g.da && adapters) {
        if ((rc = rairs_launch_clear_rows(g.da, p.n_adapters, (int64_t)p.rank * p.d_in, (int64_t)p.rank * p.d_in, p.dtype, s))) return rc;
        if ((rc = rairs_launch_clear_rows(g.db, p.n_adapters, (int64_t)p.rank * p.d_out, (int64_t)p.rank * p.d_out, p.dtype, s))) return rc;
    }
    if (!g.dx || g.n == 0) return RAIRS_OK;
    rowprod_sums(rp, np, np, bf ? opad : pad_to(p.d_out, 32));        // (as far as the batch's rows are laid out)
    if (!use && (rc = rairs_launch_pack(jobs, s))) return rc;
    if (!use && (rc = rairs_launch_pack_cols(p.W, p.dtype, p.d_in, p.d_out, p.d_in, nullptr, ORDER_SAME, wt, opad, wto, s))) return rc;
    rp.P = RowOperand{wt, wto.ld, 0, p.d_in, nullptr, nullptr};
    if (late && (rc = rairs_operand(g.dy, p.dtype, g.lddy, g.n, p.d_out, use ? sv.perm : nullptr, !bf, yroom, rp.Q, s))) return rc;
    if (use) {
        rp.ad = AdapterPart{vp, ap, zero, sv.of_row, sv.first + 1, side.kpad};
    }
    StoreEpi e = {g.dx, g.lddx, 0, p.d_in, g.n, use ? sv.perm : nullptr, bf, 0};
    return large_product(rp, e, bf, false, use ? &job : nullptr, vp, flags.bad, s);
}
