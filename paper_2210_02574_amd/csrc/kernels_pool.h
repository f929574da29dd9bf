// Mean over the rows of each sequence, forward and backward: e_i = (1 / n_i) sum x_j, 0 for an empty sequence; dx_j = de_i / n_i.
// Sums in 32 bits; the embedding stays in 32 bits because it is encoded next.  Bound by reading x, or by writing dx.
#pragma once
#include "enc_common.h"

struct PoolArgs {
    const void *x;
    float *e;
    float *part; // [count][splits][width] sums, where a sequence is cut
    int64_t x_row;
    Spans s;
    int width, splits;
};
struct PoolGradArgs {
    const float *de;
    void *dx;
    int64_t dx_row;
    Spans s;
    int width, fill;
};

// grid (sequences, column blocks, splits).  A thread has one vector of columns and every RG-th row; CL = threads along the columns.
#define POOL_THREADS 1024
template <class T, int VEC> __global__ __launch_bounds__(POOL_THREADS) void k_pool(PoolArgs a, int CL)
{
    __shared__ float join[POOL_THREADS * VEC];
    const int RG = POOL_THREADS / CL, cl = threadIdx.x % CL, rg = threadIdx.x / CL;
    const int col = (blockIdx.y * CL + cl) * VEC, i = blockIdx.x;
    const int begin = span_begin(a.s, i), end = span_end(a.s, i), n = max(end - begin, 0);
    const int per = (n + a.splits - 1) / a.splits, lo = begin + min(n, (int)blockIdx.z * per), hi = min(lo + per, begin + n);
    float s[VEC];
#pragma unroll
    for (int e = 0; e < VEC; e++) s[e] = 0.f;
    if (rg < RG && col < a.width) {
        const T *x = (const T *)a.x + col;
        int j = lo + rg;
        for (; j + 3 * RG < hi; j += 4 * RG) { // four rows in flight
            Vec<T, VEC> v[4];
#pragma unroll
            for (int u = 0; u < 4; u++) v[u] = *(const Vec<T, VEC> *)(x + (j + u * RG) * a.x_row);
#pragma unroll
            for (int u = 0; u < 4; u++)
#pragma unroll
                for (int e = 0; e < VEC; e++) s[e] += (float)v[u][e];
        }
        for (; j < hi; j += RG) {
            const Vec<T, VEC> v = *(const Vec<T, VEC> *)(x + j * a.x_row);
#pragma unroll
            for (int e = 0; e < VEC; e++) s[e] += (float)v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; e++) join[e * POOL_THREADS + threadIdx.x] = s[e];
    __syncthreads();
    if (rg != 0 || col >= a.width) return;
    const float f = a.splits > 1 ? 1.f : n > 0 ? 1.f / (float)n : 0.f;
    float *out = a.splits > 1 ? a.part + ((size_t)i * a.splits + blockIdx.z) * a.width : a.e + (size_t)i * a.width;
#pragma unroll
    for (int e = 0; e < VEC; e++) {
        for (int k = 1; k < RG; k++) s[e] += join[e * POOL_THREADS + k * CL + cl];
        out[col + e] = s[e] * f;
    }
}

// grid (sequences, columns / 256)
static __global__ __launch_bounds__(256) void k_pool_join(PoolArgs a)
{
    const int col = blockIdx.y * 256 + threadIdx.x, i = blockIdx.x;
    if (col >= a.width) return;
    const int n = span_end(a.s, i) - span_begin(a.s, i);
    float s = 0.f;
    for (int k = 0; k < a.splits; k++) s += a.part[((size_t)i * a.splits + k) * a.width + col];
    a.e[(size_t)i * a.width + col] = n > 0 ? s / (float)n : 0.f;
}

// grid (tile slots, column blocks): the rows of one tile get the sequence's row, rows of no sequence zeros if `fill`.
#define POOL_TILE 32
template <class T, int VEC> __global__ __launch_bounds__(256) void k_pool_grad(PoolGradArgs a, int CL)
{
    const TileRows t = tile_rows(a.s, blockIdx.x, POOL_TILE);
    if (t.first >= t.top) return;
    const int RG = 256 / CL, cl = threadIdx.x % CL, rg = threadIdx.x / CL;
    const int col = (blockIdx.y * CL + cl) * VEC, n = t.end - t.begin;
    if (rg >= RG || col >= a.width) return;
    Vec<T, VEC> v, zero;
    const float nf = (float)max(n, 1);
#pragma unroll
    for (int e = 0; e < VEC; e++) {
        v[e] = (T)(a.de[(size_t)t.seq * a.width + col + e] / nf);
        zero[e] = (T)0.f;
    }
    for (int j = t.first + rg; j < t.top; j += RG) {
        const bool in = j >= t.begin && j < t.end;
        if (in || a.fill) *(Vec<T, VEC> *)((T *)a.dx + j * a.dx_row + col) = in ? v : zero;
    }
}
