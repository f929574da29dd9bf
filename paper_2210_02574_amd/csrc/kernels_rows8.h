// Root-mean-square norm over rows of token states, forward and backward, and rows in 8 bits.
//
//   s = x + r (rounded to the type, where there is a residual r; else s = x), rstd = (mean(s^2) + eps)^-1/2, y = s rstd w.
//   With g = dy w:  ds = rstd (g - s rstd^2 mean(g s)) + ds', dw = sum over rows of dy s rstd.
//   A row f in 8 bits: t = max |f|, integers rint(127 f / t), scale t / 127.  Of y it takes f = s w alone, as rstd is common to the row: scale t rstd / 127.
//
// As in layer norm a row stays in the registers of its TPR threads and is read once; sums are in 32 bits.  All of it is bound by memory.
#pragma once
#include "kernels_norm.h"

// How results are written that fill whole lines, each by one wave.  KEEP: as lines that stay in L2 until the kernel's end.  THROUGH: to the last-level cache as they come, where all of
// them fit in the L2s, and would leave them only at the end.  PAST: to memory, where what the call moves does not fit in the last-level cache.
enum { KEEP, THROUGH, PAST };
template <class T, int VEC, int WIDTH> __device__ __forceinline__ void write_vec(const Cols<VEC, WIDTH> &k, const Vec<T, VEC> v, void *to, int64_t row, int how)
{
    if constexpr (WIDTH == WIDTH_EVEN) {
        if (how == THROUGH) {
            typedef int Words __attribute__((ext_vector_type(sizeof(v) / 4)));
            const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc(to, 0, 0x7fffffff, 0x00027000);
            const int at = (int)(row + k.at) * (int)sizeof(T);
            if (!k.in) return;
            if constexpr (sizeof(v) == 16)
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(Words, v), all, at, 0, 1 << 4); // scope: the device
            else if constexpr (sizeof(v) == 8)
                __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(Words, v), all, at, 0, 1 << 4);
            else
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(int, v), all, at, 0, 1 << 4);
            return;
        }
        if (how == PAST) {
            asm volatile(""); // (or this store and the other become one that keeps its lines)
            if (k.in) __builtin_nontemporal_store(v, (Vec<T, VEC> *)((T *)to + row + k.at));
            asm volatile("");
            return;
        }
    }
    k.store(v, (T *)to + row);
}

struct RmsArgs {
    const void *x, *r, *w;
    void *y, *s;  // y: the rows' type, or 8-bit integers
    float *out;   // [rows]: rstd, or the scales
    int64_t x_row, r_row, y_row, s_row; // row strides, in elements
    int rows, width, first; // rows, of them the first one of this launch
    int how;                // y is written; s past the caches too, or kept
    float eps;
};
struct RmsGradArgs {
    const void *dy, *s, *w, *add;
    void *ds;
    const float *rstd;
    float *part; // [gridDim.x][width]: every work-group's share of dw
    void *dw;    // for a lone work-group, which has all of it
    int64_t dy_row, s_row, add_row, ds_row;
    int rows, width, how;
};

// The sum of v and the largest m over the TPR threads of a row, the same in each; red: two words per wave.
template <int TPR> __device__ __forceinline__ void row_sum_max(float &v, unsigned &m, float *red)
{
    constexpr int LANES = TPR < 64 ? TPR : 64;
#pragma unroll
    for (int s = LANES / 2; s > 0; s >>= 1) {
        v += __shfl_xor(v, s, 64);
        m = max(m, (unsigned)__shfl_xor((int)m, s, 64));
    }
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) {
            red[2 * (threadIdx.x >> 6)] = v;
            red[2 * (threadIdx.x >> 6) + 1] = __uint_as_float(m);
        }
        __syncthreads();
        v = 0.f, m = 0;
#pragma unroll
        for (int k = 0; k < TPR / 64; k++) {
            v += red[2 * k];
            m = max(m, __float_as_uint(red[2 * k + 1]));
        }
    }
}

// x Phi(x) = max(x, 0) - z Phi(-z) with z = |x|, and Phi(-z) = t 2^(q(t) - z^2 log2(e) / 2), t = 1 / (1 + c z): q is a fit of degree 8 to the function that this leaves, within
// 2e-7 of it for z <= 14 (1.35e-7 of Phi), so that the lower tail is as exact, relatively, as the exponential: 1 + erf would lose it.  Half of the 2^-20 (1 + x^2 / 8) that is
// granted is used from -13 on; below, 2^(..) becomes subnormal, which the instruction makes zero.
__device__ __forceinline__ float gelu(float x)
{
    const float z = fabsf(x), t = __builtin_amdgcn_rcpf(fmaf(z, 0.28f, 1.f));
    float q = -0.31165364384651184f;
    q = fmaf(q, t, 1.4158542156219482f);
    q = fmaf(q, t, -2.3475422859191895f);
    q = fmaf(q, t, 1.6794201135635376f);
    q = fmaf(q, t, -0.780142068862915f);
    q = fmaf(q, t, 0.49303320050239563f);
    q = fmaf(q, t, 0.5668017268180847f);
    q = fmaf(q, t, 1.4466335773468018f);
    q = fmaf(q, t, -3.162405014038086f);
    q = fmaf(x * x, -0.72134752044448170f, q);
    return fmaf(-z, t * __builtin_amdgcn_exp2f(q), fmaxf(x, 0.f));
}

// The row's numbers for its integers, from the bits of max |f| (largest as an integer: a NaN is above an infinity is above all others).
struct Eight {
    float t, c; // the maximum, and 127 / t
    float top;  // the maximum times a power of two that brings it into [1/2, 1), and that power
    int exp;
    bool bad;   // not finite
    bool plain; // far from the ends of the range: c neither overflows nor loses bits
    __device__ __forceinline__ explicit Eight(unsigned bits)
    {
        bad = bits >= 0x7f800000u;
        t = __uint_as_float(bits);
        const float one = bad || !bits ? 1.f : t;
        exp = -__builtin_amdgcn_frexp_expf(one);
        top = __builtin_amdgcn_frexp_mantf(one);
        c = __builtin_amdgcn_ldexpf(127.f / top, exp);
        plain = exp > -100 && exp < 100;
    }
    __device__ __forceinline__ float scale(float rstd) const { return bad ? __builtin_nanf("") : t == 0.f ? 0.f : t * rstd / 127.f; }
    // 127 f / t to the nearest integer, in the low byte of the result: the sum with 1.5 2^23 rounds to whole numbers, ties to the even one.
    static constexpr float MAGIC = 12582912.f;
    __device__ __forceinline__ unsigned near(float f) const { return __float_as_uint(fmaf(f, c, MAGIC)); }
    // How far the quotient is from that integer.
    __device__ __forceinline__ float far(float f) const { return fabsf(fmaf(f, c, MAGIC - fmaf(f, c, MAGIC))); }
    // The same integer at the ends of the range, and where the quotient, off by up to 2^-17 as c is rounded, may lie on the other side of a border, or on it: the rest 127 f - n t
    // decides, with no rounding that could change its sign for 16-bit rows and weights.
    __device__ __forceinline__ unsigned exact(float f) const
    {
        const float p = __builtin_amdgcn_ldexpf(f, exp), m = fmaf(p, 127.f / top, MAGIC), n = m - MAGIC;
        const float h = 127.f * p, rest = 2.f * (fmaf(-n, top, h) + fmaf(127.f, p, -h));
        const unsigned i = __float_as_uint(m), odd = i & 1;
        return i + (rest > top || (rest == top && odd) ? 1u : 0u) - (rest < -top || (rest == -top && odd) ? 1u : 0u);
    }
};
// VEC values of a row in 8 bits.  EXACT: the nearest integers; else, of values that are themselves off by a few 2^-22, the nearest to quotients off by 2^-17.
template <int VEC, bool EXACT> __device__ __forceinline__ Vec<int8_t, VEC> eight_vec(const float (&f)[VEC], const Eight &q)
{
    unsigned b[VEC];
    float far = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; e++) {
        b[e] = q.near(f[e]);
        if constexpr (EXACT) far = fmaxf(far, q.far(f[e]));
    }
    if (!q.plain || !(far < 0.49999f))
#pragma unroll
        for (int e = 0; e < VEC; e++) b[e] = q.exact(f[e]);
    unsigned w[VEC / 4];
#pragma unroll
    for (int i = 0; i < VEC / 4; i++) {
        const unsigned lo = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x0c0c0400u);
        w[i] = q.bad ? 0u : lo | hi << 16;
    }
    Vec<int8_t, VEC> v;
    __builtin_memcpy(&v, w, VEC);
    return v;
}

// Bound by memory, reads being faster than a copy: 65536 x 768 in bf16 with a residual 58 us (6.9 TB/s, a part of it from the last-level cache; three sets of inputs in turn 71 us,
// 5.7 TB/s), 4999 x 1021 in 32 bits 8.2 us (5.0 TB/s); in 8 bits 16384 x 768 in bf16 with a residual 15.6 us (5.6 TB/s), 23 rows 3.5 us, two trips to memory.
template <class T, class TW, int VEC, int TPR, int NC, int WIDTH, bool EIGHT> __device__ __forceinline__ void rms_norm_rows(const RmsArgs &a)
{
    constexpr int THREADS = TPR > 256 ? TPR : 256;
    __shared__ float red[THREADS / 32];
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
    float sq = 0.f;
    unsigned top = 0;
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
        Vec<TW, VEC> w;
        if constexpr (EIGHT) w = k.load((const TW *)a.w);
        if (a.r) {
#pragma unroll
            for (int e = 0; e < VEC; e++) x[c][e] = (T)((float)x[c][e] + (float)res[c][e]);
            if (live) write_vec<T>(k, x[c], a.s, r * a.s_row, a.how == PAST ? PAST : KEEP);
        }
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            v[c][e] = (float)x[c][e];
            sq += k.count(e) ? v[c][e] * v[c][e] : 0.f;
            if constexpr (EIGHT) {
                v[c][e] *= (float)w[e];
                top = max(top, __float_as_uint(v[c][e]) & 0x7fffffffu); // (elements that are a neighbour's as well, or zeros behind the end, do no harm)
            }
        }
    }
    const float inv_w = 1.f / (float)a.width;
    if constexpr (EIGHT) {
        row_sum_max<TPR>(sq, top, red);
        if (!live) return;
        const Eight q(top);
        const float rstd = rsqrtf(sq * inv_w + a.eps);
        if (t == 0) a.out[row] = q.scale(rstd);
#pragma unroll
        for (int c = 0; c < NC; c++) write_vec<int8_t>(Cols<VEC, WIDTH>((c * TPR + t) * VEC, a.width), eight_vec<VEC, true>(v[c], q), a.y, r * a.y_row, a.how);
    } else {
        const float rstd = rsqrtf(row_sum<TPR>(sq, red) * inv_w + a.eps);
        if (!live) return;
        if (t == 0) a.out[row] = rstd;
#pragma unroll
        for (int c = 0; c < NC; c++) {
            const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
            const Vec<TW, VEC> w = k.load((const TW *)a.w);
            Vec<T, VEC> y;
#pragma unroll
            for (int e = 0; e < VEC; e++) y[e] = (T)(v[c][e] * rstd * (float)w[e]);
            write_vec<T>(k, y, a.y, r * a.y_row, a.how);
        }
    }
}

template <class T, class TW, int VEC, int TPR, int NC, int WIDTH>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_rms_norm(RmsArgs a)
{
    rms_norm_rows<T, TW, VEC, TPR, NC, WIDTH, false>(a);
}
template <class T, class TW, int VEC, int TPR, int NC, int WIDTH>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_rms_norm8(RmsArgs a)
{
    rms_norm_rows<T, TW, VEC, TPR, NC, WIDTH, true>(a);
}

// A work-group takes every gridDim.x-th group of RPW rows, holds its share of dw in registers and writes it as a partial row; k_rms_weight_grad sums those, unless there is but one.
// How many work-groups there are: rms_parts.  No atomics: a run repeats bit for bit.
// Bound by memory: 16384 x 768 in bf16 with ds' 17 us (5.9 TB/s), 65536 x 768 with the sum of dw 65 us (6.2 TB/s), 4999 x 1021 in 32 bits 13.9 us (4.4 TB/s).
template <class T, class TW, int VEC, int TPR, int NC, int WIDTH>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_rms_norm_grad(RmsGradArgs a)
{
    constexpr int THREADS = TPR > 256 ? TPR : 256, RPW = THREADS / TPR;
    __shared__ float red[THREADS / 64];
    __shared__ float join[RPW > 1 ? (RPW - 1) * TPR * VEC : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    float dw[NC][VEC];
    Vec<TW, VEC> w[NC];
#pragma unroll
    for (int c = 0; c < NC; c++) {
        w[c] = Cols<VEC, WIDTH>((c * TPR + t) * VEC, a.width).load((const TW *)a.w);
#pragma unroll
        for (int e = 0; e < VEC; e++) dw[c][e] = 0.f;
    }
    const float inv_w = 1.f / (float)a.width;
    for (int row0 = blockIdx.x * RPW; row0 < a.rows; row0 += gridDim.x * RPW) {
        Vec<T, VEC> d[NC], s[NC], add[NC];
        const int64_t r = min(row0 + sub, a.rows - 1);
        const float rstd = a.rstd[r];
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
        float c2 = 0.f;
#pragma unroll
        for (int c = 0; c < NC; c++) {
            const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                if (!live || !k.count(e)) continue; // (a product with an infinity of no account would not be zero)
                const float dy = (float)d[c][e], xh = (float)s[c][e] * rstd;
                c2 += dy * (float)w[c][e] * xh;
                dw[c][e] += dy * xh;
            }
        }
        c2 = row_sum<TPR>(c2, red) * inv_w;
        if (!live) continue; // rows of one wave or more: all of its threads; the barriers are behind
#pragma unroll
        for (int c = 0; c < NC; c++) {
            const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
            Vec<T, VEC> o;
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                float u = rstd * ((float)d[c][e] * (float)w[c][e] - (float)s[c][e] * rstd * c2);
                if (a.add) u += (float)add[c][e];
                o[e] = (T)u;
            }
            write_vec<T>(k, o, a.ds, row * a.ds_row, a.how == PAST ? PAST : KEEP);
        }
    }
    float *part = a.part + (size_t)blockIdx.x * a.width;
#pragma unroll
    for (int c = 0; c < NC; c++) {
        const Cols<VEC, WIDTH> k((c * TPR + t) * VEC, a.width);
        if constexpr (RPW > 1) {
            __syncthreads();
            if (sub > 0)
#pragma unroll
                for (int e = 0; e < VEC; e++) join[((sub - 1) * VEC + e) * TPR + t] = dw[c][e];
            __syncthreads();
        }
        if (sub == 0)
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                if (!k.count(e)) continue;
                float u = dw[c][e];
                if constexpr (RPW > 1)
#pragma unroll
                    for (int i = 0; i < RPW - 1; i++) u += join[(i * VEC + e) * TPR + t];
                if (gridDim.x == 1)
                    ((TW *)a.dw)[k.at + e] = (TW)u;
                else
                    part[k.at + e] = u;
            }
    }
}

// dw from the partial rows: 16 columns per work-group, 16 threads to a column.  Bound by the trips to memory that follow the other kernel's end: 512 x 768 3.8 to 4.6 us, and as
// much with 64 threads to a column.
template <class TW> __global__ __launch_bounds__(256) void k_rms_weight_grad(const float *__restrict__ part, int parts, int width, TW *dw)
{
    __shared__ float red[256];
    const int c = threadIdx.x & 15, k0 = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    const float *p = part + col;
    float s = 0.f;
    if (col < width)
#pragma unroll 8
        for (int k = k0; k < parts; k += 16) s += p[(size_t)k * width];
    red[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x >= 16 || col >= width) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; k++) s += red[k * 16 + c];
    dw[col] = (TW)s;
}

struct Rows8Args {
    const void *x;
    int8_t *y;
    float *scale;
    int64_t x_row, y_row;
    int rows, width, first, how;
};
// Gaussian error units are bound by vector instructions, some 30 to a number: 16384 x 2048 in bf16 26 us (3.9 TB/s); rows as they are by memory, or by two trips to it: 3001 x 1000
// in fp16 5.8 us.
template <class T, int VEC, int TPR, int NC, int WIDTH, bool GELU>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_quantize8(Rows8Args a)
{
    constexpr int THREADS = TPR > 256 ? TPR : 256;
    __shared__ float red[THREADS / 32];
    const int t = threadIdx.x % TPR, row = a.first + blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR;
    const bool live = row < a.rows;
    const int64_t r = min(row, a.rows - 1);
    Vec<T, VEC> x[NC];
#pragma unroll
    for (int c = 0; c < NC; c++) x[c] = Cols<VEC, WIDTH>((c * TPR + t) * VEC, a.width).load((const T *)a.x + r * a.x_row);
    __builtin_amdgcn_sched_barrier(0);
    float v[NC][VEC], none = 0.f;
    unsigned top = 0;
#pragma unroll
    for (int c = 0; c < NC; c++)
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            v[c][e] = (float)x[c][e];
            if constexpr (GELU) v[c][e] = gelu(v[c][e]);
            // (elements that are a neighbour's as well, or zeros behind the row's end, do no harm)
            top = max(top, __float_as_uint(v[c][e]) & 0x7fffffffu);
        }
    row_sum_max<TPR>(none, top, red);
    if (!live) return;
    const Eight q(top);
    if (t == 0) a.scale[row] = q.scale(1.f);
#pragma unroll
    for (int c = 0; c < NC; c++) write_vec<int8_t>(Cols<VEC, WIDTH>((c * TPR + t) * VEC, a.width), eight_vec<VEC, !GELU>(v[c], q), a.y, r * a.y_row, a.how);
}
