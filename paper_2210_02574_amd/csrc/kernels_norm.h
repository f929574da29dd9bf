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
    int rows, width;
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

template <class T, class TW, int VEC, int TPR, int NC>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_layer_norm(NormArgs a)
{
    constexpr int THREADS = TPR > 256 ? TPR : 256;
    __shared__ float red[THREADS / 64];
    const int t = threadIdx.x % TPR, row = blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR;
    const bool live = row < a.rows; // a row's lanes are live or not together; all of them take part in the sums
    float v[NC][VEC];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const int col = (c * TPR + t) * VEC;
        Vec<T, VEC> x = {};
        if (live && col < a.width) {
            x = load_vec<T, VEC>((const T *)a.x + row * a.x_row, col, a.width);
            if (a.r) {
                const Vec<T, VEC> r = load_vec<T, VEC>((const T *)a.r + row * a.r_row, col, a.width);
#pragma unroll
                for (int e = 0; e < VEC; e++) x[e] = (T)((float)x[e] + (float)r[e]);
                store_vec<T, VEC>(x, (T *)a.s + row * a.s_row, col, a.width);
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            v[c][e] = (float)x[e];
            sum += v[c][e];
        }
    }
    const float inv_w = 1.f / (float)a.width;
    const float mean = row_sum<TPR>(sum, red) * inv_w;
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const int col = (c * TPR + t) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            const float d = col + e < a.width ? v[c][e] - mean : 0.f;
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
        const int col = (c * TPR + t) * VEC;
        if (col >= a.width) continue;
        const Vec<TW, VEC> w = load_vec<TW, VEC>((const TW *)a.w, col, a.width), b = load_vec<TW, VEC>((const TW *)a.b, col, a.width);
        Vec<T, VEC> y;
#pragma unroll
        for (int e = 0; e < VEC; e++) y[e] = (T)((v[c][e] - mean) * rstd * (float)w[e] + (float)b[e]);
        store_vec<T, VEC>(y, (T *)a.y + row * a.y_row, col, a.width);
    }
}

// Work-group g takes the rows g, g + gridDim.x, .. (times the rows of a work-group), keeps its columns' shares of dw and db in registers, joins those of its
// rows in LDS and writes one partial row each; k_norm_weight_grad sums the partial rows.  No atomics: a run repeats bit for bit.
template <class T, class TW, int VEC, int TPR, int NC>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_layer_norm_grad(NormGradArgs a)
{
    constexpr int THREADS = TPR > 256 ? TPR : 256, RPW = THREADS / TPR;
    __shared__ float red[THREADS / 64];
    __shared__ float join[RPW > 1 ? (RPW - 1) * TPR * VEC * 2 : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    float w[NC][VEC], dw[NC][VEC], db[NC][VEC];
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const int col = (c * TPR + t) * VEC;
        const Vec<TW, VEC> u = load_vec<TW, VEC>((const TW *)a.w, col, a.width);
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            w[c][e] = (float)u[e];
            dw[c][e] = db[c][e] = 0.f;
        }
    }
    const float inv_w = 1.f / (float)a.width;
    for (int row0 = blockIdx.x * RPW; row0 < a.rows; row0 += gridDim.x * RPW) {
        const int row = row0 + sub;
        const bool live = row < a.rows;
        const float mean = live ? a.mean[row] : 0.f, rstd = live ? a.rstd[row] : 0.f;
        float g[NC][VEC], xh[NC][VEC];
        float c1 = 0.f, c2 = 0.f;
#pragma unroll
        for (int c = 0; c < NC; c++) {
            const int col = (c * TPR + t) * VEC;
            Vec<T, VEC> d = {}, s = {};
            if (live && col < a.width) {
                d = load_vec<T, VEC>((const T *)a.dy + row * a.dy_row, col, a.width);
                s = load_vec<T, VEC>((const T *)a.s + row * a.s_row, col, a.width);
            }
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                const float dy = (float)d[e];
                xh[c][e] = col + e < a.width ? ((float)s[e] - mean) * rstd : 0.f;
                g[c][e] = dy * w[c][e];
                c1 += g[c][e];
                c2 += g[c][e] * xh[c][e];
                dw[c][e] += dy * xh[c][e];
                db[c][e] += dy;
            }
        }
        c1 = row_sum<TPR>(c1, red) * inv_w;
        c2 = row_sum<TPR>(c2, red) * inv_w;
        if (!live) continue; // rows of one wave or more: all of its threads; the barriers are behind
#pragma unroll
        for (int c = 0; c < NC; c++) {
            const int col = (c * TPR + t) * VEC;
            if (col >= a.width) continue;
            Vec<T, VEC> o, add = {};
            if (a.add) add = load_vec<T, VEC>((const T *)a.add + row * a.add_row, col, a.width);
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                float v = rstd * (g[c][e] - c1 - xh[c][e] * c2);
                if (a.add) v += (float)add[e];
                o[e] = (T)v;
            }
            store_vec<T, VEC>(o, (T *)a.ds + row * a.ds_row, col, a.width);
        }
    }
    float *part = a.part + (size_t)blockIdx.x * 2 * a.width;
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const int col = (c * TPR + t) * VEC;
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
                if (col + e >= a.width) break;
                float u = dw[c][e], v = db[c][e];
                if constexpr (RPW > 1)
#pragma unroll
                    for (int k = 0; k < RPW - 1; k++) {
                        u += join[(k * 2 * VEC + e) * TPR + t];
                        v += join[(k * 2 * VEC + VEC + e) * TPR + t];
                    }
                part[col + e] = u;
                part[a.width + col + e] = v;
            }
    }
}

// dw and db from the partial rows: 16 columns per work-group, 16 threads to a column, blockIdx.y = 0: dw, 1: db.
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
