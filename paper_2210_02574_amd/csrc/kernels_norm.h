// Layer norm over rows of token states, forward and backward.
//
//   s = x + r (rounded to the type, where there is a residual r; else s = x), m = mean(s), rstd = (mean((s - m)^2) + eps)^-1/2,
//   xh = (s - m) rstd, y = xh w + b.
//   With g = dy w:  ds = rstd (g - mean(g) - xh mean(g xh)) + ds', dw = sum over rows of dy xh, db = sum over rows of dy.
//
// A row stays in the registers of its TPR threads, NC vectors of VEC elements each, so that it is read once: the variance is a second
// pass over registers, which has no cancellation of large means.  All sums are in 32 bits.  Both directions are bound by memory.
#pragma once
#include "enc_common.h"

struct NormArgs {
    const void *x, *r, *w, *b;
    void *y, *s;
    float *mean, *rstd;
    int64_t x_row, r_row, y_row, s_row; // row strides, in elements
    int rows, width, first; // rows, of them the first one of this launch
    float eps;
};
struct NormGradArgs {
    const void *dy, *s, *w, *add;
    void *ds;
    const float *mean, *rstd;
    float *part; // [gridDim.x][2][width]: every work-group's share of dw and db
    int64_t dy_row, s_row, add_row, ds_row;
    int rows, width;
};

// Sum over the TPR threads of a row, the same in each.  Rows of several waves go through LDS; `red` has room for one word per wave and is
// written again only behind a barrier.
template <int TPR> __device__ __forceinline__ float row_sum(float v, float *red)
{
    if constexpr (TPR <= 64) return lanes_sum<TPR>(v);
    v = lanes_sum<64>(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < TPR / 64; k++) t += red[k];
    __syncthreads();
    return t;
}

// The vector c of a thread.  Every load is a whole vector and none is behind a branch, so that all loads of a row are under way together: a vector that
// would reach over the row's end (ODD: widths that VEC does not divide) begins earlier and repeats elements of its neighbour, which it does
// not count (count(e) false) and stores with the same values; a thread behind the row's end reads the last vector and counts nothing.
// A width below VEC (SMALL) is one thread's, element by element.
enum { WIDTH_EVEN, WIDTH_ODD, WIDTH_SMALL };
template <int VEC, int WIDTH> struct Cols {
    int at, first, width;
    bool in;
    __device__ __forceinline__ Cols(int col, int width) : at(WIDTH == WIDTH_SMALL ? col : min(col, width - VEC)), first(col - at), width(width), in(col < width) {}
    __device__ __forceinline__ bool count(int e) const
    {
        return in && (WIDTH == WIDTH_EVEN || (WIDTH == WIDTH_ODD ? e >= first : at + e < width));
    }
    template <class T> __device__ __forceinline__ Vec<T, VEC> load(const T *row) const
    {
        if constexpr (WIDTH == WIDTH_SMALL) return load_vec<T, VEC>(row, at, width);
        return *(const typename UnalignedVec<T, VEC>::type *)(row + at);
    }
    template <class T> __device__ __forceinline__ void store(Vec<T, VEC> x, T *row) const
    {
        if constexpr (WIDTH == WIDTH_SMALL)
            store_vec<T, VEC>(x, row, at, width);
        else if (in)
            *(typename UnalignedVec<T, VEC>::type *)(row + at) = x;
    }
};

// Bound by memory: 65536 x 768 in bf16 with a residual 73 us (5.5 TB/s), 4999 x 1021 in 32 bits 8.8 us (4.7 TB/s, half of it from caches); 23 rows 4.2 us, two
// trips to memory.
template <class T, class TW, int VEC, int TPR, int NC, int WIDTH>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_layer_norm(NormArgs a)
{
    constexpr int THREADS = TPR > 256 ? TPR : 256;
    __shared__ float red[THREADS / 64];
    const int t = threadIdx.x % TPR, row = a.first + blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR;
    const bool live = row < a.rows; // a row's lanes are live or not together; all of them take part in the sums, on the last row
    const int64_t r = min(row, a.rows - 1);
    Vec<T, VEC> x[NC], res[NC];
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
        x[c] = k.load((const T *)a.x + r * a.x_row);
        if (a.r) res[c] = k.load((const T *)a.r + r * a.r_row);
    }
    __builtin_amdgcn_sched_barrier(0);
    float v[NC][VEC];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
        if (a.r) {
#pragma unroll
            for (int e = 0; e < VEC; e++) x[c][e] = (T)((float)x[c][e] + (float)res[c][e]);
            if (live) k.store(x[c], (T *)a.s + r * a.s_row);
        }
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            v[c][e] = (float)x[c][e];
            sum += k.count(e) ? v[c][e] : 0.f;
        }
    }
    const float inv_w = 1.f / (float)a.width;
    const float mean = row_sum<TPR>(sum, red) * inv_w;
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            const float d = k.count(e) ? v[c][e] - mean : 0.f;
            sq += d * d;
        }
    }
    const float rstd = rsqrtf(row_sum<TPR>(sq, red) * inv_w + a.eps);
    if (!live) return;
    if (t == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
        const Vec<TW, VEC> w = k.load((const TW *)a.w), b = k.load((const TW *)a.b); // (asked for ahead of the sums they cost a wave: 16384 x 768 16 us, 19)
        Vec<T, VEC> y;
#pragma unroll
        for (int e = 0; e < VEC; e++) y[e] = (T)((v[c][e] - mean) * rstd * (float)w[e] + (float)b[e]);
        k.store(y, (T *)a.y + r * a.y_row);
    }
}

// 2 work-groups per CU: their partial rows cost little to sum and their registers (about 180 for 768 columns) leave room for no third (16384 x 768 bf16: 18 us;
// 256 work-groups 22, 768 of them 22; asking for the next row ahead of this one's sums changed nothing).
// Work-group g takes the rows g, g + gridDim.x, .. (times the rows of a work-group), keeps its columns' shares of dw and db in registers, joins those of its
// rows in LDS and writes one partial row each; k_norm_weight_grad sums the partial rows.  No atomics: a run repeats bit for bit.
template <class T, class TW, int VEC, int TPR, int NC, int WIDTH>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_layer_norm_grad(NormGradArgs a)
{
    constexpr int THREADS = TPR > 256 ? TPR : 256, RPW = THREADS / TPR;
    __shared__ float red[THREADS / 64];
    __shared__ float join[RPW > 1 ? (RPW - 1) * TPR * VEC * 2 : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    float dw[NC][VEC], db[NC][VEC];
    Vec<TW, VEC> w[NC];
#pragma unroll
    for (int c = 0; c < NC; c++) {
        w[c] = Cols<VEC, WIDTH>((c * TPR + t) * VEC, a.width).load((const TW *)a.w);
#pragma unroll
        for (int e = 0; e < VEC; e++) dw[c][e] = db[c][e] = 0.f;
    }
    const float inv_w = 1.f / (float)a.width;
    for (int row0 = blockIdx.x * RPW; row0 < a.rows; row0 += gridDim.x * RPW) {
        Vec<T, VEC> d[NC], s[NC], add[NC];
        const int64_t r = min(row0 + sub, a.rows - 1);
        const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
        for (int c = 0; c < NC; c++) {
            const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
            d[c] = k.load((const T *)a.dy + r * a.dy_row);
            s[c] = k.load((const T *)a.s + r * a.s_row);
            if (a.add) add[c] = k.load((const T *)a.add + r * a.add_row);
        }
        __builtin_amdgcn_sched_barrier(0);
        const int row = row0 + sub;
        const bool live = row < a.rows;
        float c1 = 0.f, c2 = 0.f;
#pragma unroll
        for (int c = 0; c < NC; c++) {
            const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                const float dy = live && k.count(e) ? (float)d[c][e] : 0.f, g = dy * (float)w[c][e], xh = ((float)s[c][e] - mean) * rstd;
                c1 += g;
                if (!live || !k.count(e)) continue; // (a product with an infinity of no account would not be zero)
                c2 += g * xh;
                dw[c][e] += dy * xh;
                db[c][e] += dy;
            }
        }
        c1 = row_sum<TPR>(c1, red) * inv_w;
        c2 = row_sum<TPR>(c2, red) * inv_w;
        if (!live) continue; // rows of one wave or more: all of its threads; the barriers are behind
#pragma unroll
        for (int c = 0; c < NC; c++) {
            const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
            Vec<T, VEC> o;
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                float u = rstd * ((float)d[c][e] * (float)w[c][e] - c1 - ((float)s[c][e] - mean) * rstd * c2);
                if (a.add) u += (float)add[c][e];
                o[e] = (T)u;
            }
            k.store(o, (T *)a.ds + row * a.ds_row);
        }
    }
    float *part = a.part + (size_t)blockIdx.x * 2 * a.width;
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
        if constexpr (RPW > 1) {
            __syncthreads();
            if (sub > 0)
#pragma unroll
                for (int e = 0; e < VEC; e++) {
                    join[((sub - 1) * 2 * VEC + e) * TPR + t] = dw[c][e];
                    join[((sub - 1) * 2 * VEC + VEC + e) * TPR + t] = db[c][e];
                }
            __syncthreads();
        }
        if (sub == 0)
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                if (!k.count(e)) continue;
                float u = dw[c][e], v = db[c][e];
                if constexpr (RPW > 1)
#pragma unroll
                    for (int i = 0; i < RPW - 1; i++) {
                        u += join[(i * 2 * VEC + e) * TPR + t];
                        v += join[(i * 2 * VEC + VEC + e) * TPR + t];
                    }
                part[k.at + e] = u;
                part[a.width + k.at + e] = v;
            }
    }
}

// dw and db from the partial rows (512 x 768: 4 us, a launch and one trip): 16 columns per work-group, 16 threads to a column, blockIdx.y = 0: dw, 1: db.
template <class TW> __global__ __launch_bounds__(256) void k_norm_weight_grad(const float *__restrict__ part, int parts, int width, TW *dw, TW *db)
{
    __shared__ float red[256];
    const int c = threadIdx.x & 15, k0 = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    const float *p = part + (size_t)blockIdx.y * width + col;
    float s = 0.f;
    if (col < width)
#pragma unroll 8
        for (int k = k0; k < parts; k += 16) s += p[(size_t)k * 2 * width];
    red[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x >= 16 || col >= width) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; k++) s += red[k * 16 + c];
    (blockIdx.y ? db : dw)[col] = (TW)s;
}
