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

// grid (sequences or tile slots, column blocks).  A thread has one vector of columns and every RG-th row; CL = threads along the columns.
template <class T, int VEC, int THREADS> __global__ __launch_bounds__(THREADS) void k_pool(PoolArgs a, int CL)
{
    __shared__ float join[THREADS * VEC];
    const int RG = THREADS / CL, cl = threadIdx.x % CL, rg = threadIdx.x / CL;
    const int col = (blockIdx.y * CL + cl) * VEC;
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
    if (rg < RG && col < a.width) {
        const T *x = (const T *)a.x + (lo + rg) * a.x_row;
        const int64_t step = RG * a.x_row;
        int left = (hi - lo - rg + RG - 1) / RG; // rows of this thread
        if (col + VEC <= a.width)
            for (; left >= 8; left -= 8) {
                Vec<T, VEC> v[8];
#pragma unroll
                for (int u = 0; u < 8; u++, x += step) v[u] = load_once<T, VEC>(x + col);
                __builtin_amdgcn_sched_barrier(0); // eight rows are under way before the first one is waited for
#pragma unroll
                for (int u = 0; u < 8; u++)
#pragma unroll
                    for (int e = 0; e < VEC; e++) s[e] += (float)v[u][e];
            }
        for (; left > 0; left--, x += step) {
            const Vec<T, VEC> v = load_vec<T, VEC>(x, col, a.width);
#pragma unroll
            for (int e = 0; e < VEC; e++) s[e] += (float)v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; e++) join[e * THREADS + threadIdx.x] = s[e];
    __syncthreads();
    if (rg != 0) return;
    float *out = (a.tile ? a.part : a.e) + (size_t)blockIdx.x * a.width;
    const float f = 1.f / (float)n;
#pragma unroll
    for (int e = 0; e < VEC; e++) {
        for (int k = 1; k < RG; k++) s[e] += join[e * THREADS + k * CL + cl];
        if (col + e < a.width) out[col + e] = s[e] * f;
    }
}

// grid (sequences, columns / 256): the tiles of a sequence are those of the slots tile_slot(c, i) .. that reach into it.
static __global__ __launch_bounds__(256) void k_pool_join(PoolArgs a)
{
    const int col = blockIdx.y * 256 + threadIdx.x, i = blockIdx.x;
    if (col >= a.width) return;
    const int begin = span_begin(a.s, i), end = span_end(a.s, i), c = i ? begin : 0, top = i + 1 < a.s.count ? span_begin(a.s, i + 1) : a.s.rows;
    const int stop = min(end, top); // a tile ends at the next sequence's begin
    const int64_t slot = tile_slot(c, i, a.tile);
    float s = 0.f;
    if (stop > begin) {
        const int first = (begin - c) / a.tile, last = (stop - 1 - c) / a.tile;
#pragma unroll 4
        for (int k = first; k <= last; k++) s += a.part[(size_t)(slot + k) * a.width + col];
    }
    a.e[(size_t)i * a.width + col] = end > begin ? s / (float)(end - begin) : 0.f;
}

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
