// Mean over the rows of each sequence, forward and backward: e_i = (1 / n_i) sum x_j, 0 for an empty sequence; dx_j = de_i / n_i.
// Sums in 32 bits; the embedding stays in 32 bits because it is encoded next.  Bound by reading x, or by writing dx.
#pragma once
#include "enc_common.h"

struct PoolArgs {
    const void *x;
    float *e;
    float *part; // [slots][width]: the sums of the tiles
    int64_t x_row;
    Spans s;
    int width;
    int tile; // rows of a tile, or 0: a work-group per sequence
};
struct PoolGradArgs {
    const float *de;
    void *dx;
    int64_t dx_row;
    Spans s;
    int width, fill;
    int tile; // rows of a tile
};

// 256 sequences of 555 rows of 768 on average, bf16: 38 us (5.8 TB/s), and 4 us to join; 32 of 68 rows 6 us: the sequence's numbers, then one or two trips.
// grid (sequences or tile slots, column blocks).  A thread has one vector of columns and every RG-th row; CL = threads along the columns.
template <class T, int VEC, int THREADS> __global__ __launch_bounds__(THREADS) void k_pool(PoolArgs a, int CL)
{
    __shared__ float join[THREADS * VEC];
    const int RG = THREADS / CL, cl = threadIdx.x % CL, rg = threadIdx.x / CL;
    const int own = (blockIdx.y * CL + cl) * VEC; // the thread's columns begin here, its vector earlier where it would reach over the row's end
    const int col = a.width < VEC ? own : min(own, a.width - VEC);
    int lo, hi, n;
    if (a.tile) {
        const TileRows t = tile_rows(a.s, a.s, blockIdx.x, a.tile);
        lo = max(t.first, t.begin), hi = min(t.top, t.end), n = 1;
        if (lo >= hi) return; // k_pool_join does not ask for it
    } else {
        lo = span_begin(a.s, blockIdx.x), hi = span_end(a.s, blockIdx.x), n = max(hi - lo, 1);
    }
    float s[VEC];
#pragma unroll
    for (int e = 0; e < VEC; e++) s[e] = 0.f;
    // No more than it takes to give each eight rows, which cost one trip to memory: fewer shares are to be joined then.
    const int groups = min(RG, max((hi - lo + 7) / 8, 1));
    if (rg < groups && own < a.width) {
        const T *x = (const T *)a.x + (lo + rg) * a.x_row;
        const int64_t step = groups * a.x_row;
        int left = (hi - lo - rg + groups - 1) / groups; // rows of this thread
        if (a.width >= VEC)
            for (; left > 0; left -= 8) {
                Vec<T, VEC> v[8];
#pragma unroll
                for (int u = 0; u < 8; u++) { // the last row again where there are fewer
                    v[u] = load_once<T, VEC>(x + col);
                    if (u + 1 < left) x += step;
                }
                __builtin_amdgcn_sched_barrier(0); // eight rows are under way before the first one is waited for
#pragma unroll
                for (int u = 0; u < 8; u++)
#pragma unroll
                    for (int e = 0; e < VEC; e++) s[e] += u < left ? (float)v[u][e] : 0.f;
            }
        else
            for (; left > 0; left--, x += step) {
                const Vec<T, VEC> v = load_vec<T, VEC>(x, col, a.width);
#pragma unroll
                for (int e = 0; e < VEC; e++) s[e] += (float)v[e];
            }
    }
    // the shares of the upper half of the groups that are left go to the lower half
    for (int half = 1 << (31 - __clz(2 * groups - 1)) >> 1; half >= 1; half >>= 1) {
        if (rg >= half && rg < 2 * half)
#pragma unroll
            for (int e = 0; e < VEC; e++) join[e * THREADS + threadIdx.x] = s[e];
        __syncthreads();
        if (rg < half && rg + half < groups)
#pragma unroll
            for (int e = 0; e < VEC; e++) s[e] += join[e * THREADS + threadIdx.x + half * CL];
    }
    if (rg != 0) return;
    float *out = (a.tile ? a.part : a.e) + (size_t)blockIdx.x * a.width;
    const float f = 1.f / (float)n;
#pragma unroll
    for (int e = 0; e < VEC; e++)
        if (col + e >= own && col + e < a.width) out[col + e] = s[e] * f;
}

// grid (sequences, columns * SHARES / 256), SHARES threads to a column: the tiles of a sequence are those of the slots tile_slot(c, i) .. that reach into it.
// Shares pay where sequences have many tiles: one sequence of 8192 rows in 128 of them 11 us with one share, 4 with eight; 256 sequences of 555 in 8 4 us, 7.
#define POOL_SHARED_TILES 16 // per sequence, from which on there are eight shares
template <int SHARES> __global__ __launch_bounds__(256) void k_pool_join(PoolArgs a)
{
    constexpr int COLS = 256 / SHARES;
    __shared__ float join[256];
    const int col = blockIdx.y * COLS + threadIdx.x % COLS, share = threadIdx.x / COLS, i = blockIdx.x;
    const int begin = span_begin(a.s, i), end = span_end(a.s, i), c = i ? begin : 0, top = i + 1 < a.s.count ? span_begin(a.s, i + 1) : a.s.rows;
    const int stop = min(end, top); // a tile ends at the next sequence's begin
    const int64_t slot = tile_slot(c, i, a.tile);
    float s = 0.f;
    if (stop > begin && col < a.width) {
        const int first = (begin - c) / a.tile, last = (stop - 1 - c) / a.tile;
#pragma unroll 4
        for (int k = first + share; k <= last; k += SHARES) s += a.part[(size_t)(slot + k) * a.width + col];
    }
    if constexpr (SHARES > 1) {
        join[threadIdx.x] = s;
        __syncthreads();
        if (share) return;
#pragma unroll
        for (int k = 1; k < SHARES; k++) s += join[COLS * k + threadIdx.x];
    }
    if (col < a.width) a.e[(size_t)i * a.width + col] = end > begin ? s / (float)(end - begin) : 0.f;
}

// 256 sequences of 555 rows of 768 on average, bf16: 35 us (6.3 TB/s).
// grid (tile slots, column blocks): the rows of one tile get the sequence's row, rows of no sequence zeros if `fill`.
template <class T, int VEC> __global__ __launch_bounds__(256) void k_pool_grad(PoolGradArgs a, int CL)
{
    const TileRows t = tile_rows(a.s, a.s, blockIdx.x, a.tile);
    if (t.first >= t.top) return;
    const int RG = 256 / CL, cl = threadIdx.x % CL, rg = threadIdx.x / CL;
    const int col = (blockIdx.y * CL + cl) * VEC, n = t.end - t.begin;
    if (rg >= RG || col >= a.width) return;
    const float nf = (float)max(n, 1);
    const Vec<float, VEC> de = load_vec<float, VEC>(a.de + (size_t)t.seq * a.width, col, a.width);
    Vec<T, VEC> v, zero = {};
#pragma unroll
    for (int e = 0; e < VEC; e++) v[e] = (T)(de[e] / nf);
    for (int j = t.first + rg; j < t.top; j += RG) {
        const bool in = j >= t.begin && j < t.end;
        if (in || a.fill) store_vec<T, VEC>(in ? v : zero, (T *)a.dx + j * a.dx_row, col, a.width);
    }
}
