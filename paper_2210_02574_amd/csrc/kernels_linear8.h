// Product of 8-bit rows and 8-bit weights, both dense along the sum: o[m][n] = (sum over k of x[m][k] w[n][k]) x_scale[m] w_scale[n] + bias[n].
//
// Sums are exact in 32-bit integers.  A sum over 32 (or 64) numbers is one matrix instruction, whose operands are 16 bytes of a row for each lane: bytes of x and w
// that a lane holds side by side are multiplied, so any order along k serves as long as both use it.
// Weights are operand A, rows of x operand B: a lane then holds neighbouring channels of one row, which it can write together.
#pragma once
#include "enc_common.h"

typedef Vec<int, 4> i32x4;
typedef Vec<int, 16> i32x16;

struct Linear8Args {
    const int8_t *x, *w;
    const float *x_scale, *w_scale;
    const void *bias; // of 32 bits (bias32) or of the result's type, or null
    void *o;
    int64_t x_row, w_row, o_row; // row strides, in elements
    int rows, width, channels;
    int tiles_m, tiles_n;
    int bias32;
};

// Results of one row, N neighbouring channels from n on.
template <class T, int N> __device__ __forceinline__ Vec<T, N> linear8_results(const Linear8Args &a, const int (&sum)[N], float xs, int n)
{
    Vec<T, N> y;
    Vec<float, N> ws = {}, b = {};
    if (n + N <= a.channels) {
        ws = *(const typename UnalignedVec<float, N>::type *)(a.w_scale + n);
        if (a.bias && a.bias32) b = *(const typename UnalignedVec<float, N>::type *)((const float *)a.bias + n);
        if (a.bias && !a.bias32) {
            const Vec<T, N> t = *(const typename UnalignedVec<T, N>::type *)((const T *)a.bias + n);
#pragma unroll
            for (int e = 0; e < N; e++) b[e] = (float)t[e];
        }
    } else
#pragma unroll
        for (int e = 0; e < N; e++)
            if (n + e < a.channels) {
                ws[e] = a.w_scale[n + e];
                if (a.bias) b[e] = a.bias32 ? ((const float *)a.bias)[n + e] : (float)((const T *)a.bias)[n + e];
            }
#pragma unroll
    for (int e = 0; e < N; e++) {
        float f = (float)sum[e] * xs * ws[e];
        if (a.bias) f += b[e];
        y[e] = (T)f;
    }
    return y;
}

// 16 bytes for each lane from `at` of a buffer (zeros behind its end) to LDS, lane i's at to + 16 i, with no register in between.
// (Not in the template itself: the host's pass knows no such size and would drop the instance.)
__device__ __forceinline__ void fetch_lds(__amdgpu_buffer_rsrc_t from, unsigned at, int8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, at, 0, 0, 0);
}

#define LINEAR8_K 128 // numbers of a row that a stage holds

// Tiles of 64 MB rows by 64 NB channels, 2 x 2 waves with MB x NB blocks of 32 x 32 each.  A stage is 128 bytes of every row of both, written to LDS by
// the loads themselves, chunk c of row r at c ^ (r / 2 mod 8): the 16 rows that a 16-byte read of LDS takes at a time then lie in 16 different places.  There are two stages; the loads of one
// are under way for the whole of the other.  Per stage one barrier, ahead of its last products: behind it the next stage's first operands are read while those run.
template <class T, int MB, int NB> __global__ __launch_bounds__(256) void k_linear8(Linear8Args a)
{
    constexpr int BM = 64 * MB, BN = 64 * NB, STAGE = (BM + BN) * LINEAR8_K;
    constexpr int OUT_PITCH = 32 * NB * (int)sizeof(T) + 16; // of a row of results in LDS, bytes
    constexpr int OUT_BYTES = 4 * 32 * OUT_PITCH, LDS = 2 * STAGE > OUT_BYTES ? 2 * STAGE : OUT_BYTES;
    __shared__ __attribute__((aligned(1024))) int8_t lds[LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;

    // Each of the eight dies takes a run of tiles that follow one another, in bands of eight tiles of rows, so that they share operands in its L2.
    const int tiles = a.tiles_m * a.tiles_n, per = tiles / 8, extra = tiles % 8, die = blockIdx.x % 8, at = blockIdx.x / 8;
    const int id = die * per + min(die, extra) + at;
    constexpr int BAND = 8;
    const int band = id / (BAND * a.tiles_n), first = band * BAND, high = min(BAND, a.tiles_m - first), in = id - band * BAND * a.tiles_n;
    const int m0 = (first + in % high) * BM, n0 = in / high * BN;

    const int steps = (a.width + LINEAR8_K - 1) / LINEAR8_K;
    const int whole = (a.width + 15) / 16 * 16; // bytes of a row that may be read
    const int rows_m = min(BM, a.rows - m0), rows_n = min(BN, a.channels - n0);
    const int8_t *const xb = a.x + m0 * a.x_row, *const wb = a.w + n0 * a.w_row;
    const int bytes_m = (rows_m - 1) * (int)a.x_row + whole, bytes_n = (rows_n - 1) * (int)a.w_row + whole; // below 2^31, as strides are below 2^23
    // One load of a wave brings eight rows; wave v takes every fourth eight of them.
    constexpr int LM = BM / 32, LN = BN / 32;
    unsigned at_m[LM], at_n[LN];
#pragma unroll
    for (int i = 0; i < LM; i++) {
        const int row = 8 * (4 * i + wave) + lane / 8, c = (lane % 8) ^ (row >> 1 & 7);
        at_m[i] = (unsigned)row * (unsigned)a.x_row + 16 * c;
    }
#pragma unroll
    for (int i = 0; i < LN; i++) {
        const int row = 8 * (4 * i + wave) + lane / 8, c = (lane % 8) ^ (row >> 1 & 7);
        at_n[i] = (unsigned)row * (unsigned)a.w_row + 16 * c;
    }
    const auto fetch = [&](int step, int8_t *stage) {
        const int k = step * LINEAR8_K; // below the width
        const __amdgpu_buffer_rsrc_t rm = __builtin_amdgcn_make_buffer_rsrc((void *)(xb + k), 0, bytes_m - k, 0x00027000);
        const __amdgpu_buffer_rsrc_t rn = __builtin_amdgcn_make_buffer_rsrc((void *)(wb + k), 0, bytes_n - k, 0x00027000);
#pragma unroll
        for (int i = 0; i < LM; i++)
            fetch_lds(rm, at_m[i], stage + (4 * i + wave) * 1024);
#pragma unroll
        for (int i = 0; i < LN; i++)
            fetch_lds(rn, at_n[i], stage + BM * LINEAR8_K + (4 * i + wave) * 1024);
    };
    // Behind the end of the sum: weights of a stage's numbers from `left` on become zeros, so that what x's rows have there does not count.
    const auto cut = [&](int8_t *stage, int left) {
        for (int row = threadIdx.x; row < BN; row += 256) {
            int8_t *const r = stage + BM * LINEAR8_K + row * LINEAR8_K;
            for (int c = left / 16; c < 8; c++) {
                int8_t *const p = r + 16 * (c ^ (row >> 1 & 7));
                for (int b = max(left - 16 * c, 0); b < 16; b++) p[b] = 0;
            }
        }
        __syncthreads();
    };

    // Loads that write to LDS are waited for by hand: the barrier's own wait does not cover them.
    const auto arrive = [&] {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    i32x16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NB; j++) acc[i][j] = i32x16{};
    i32x4 fx[2][MB], fw[2][NB];
    // operands of the numbers 32 kk .. of a stage: lane's row l mod 32 of each block, 16 numbers
    const auto read = [&](const int8_t *stage, int kk, int to) {
        const int row = lane % 32, c = (2 * kk + lane / 32) ^ (row >> 1 & 7);
#pragma unroll
        for (int i = 0; i < MB; i++) fx[to][i] = *(const i32x4 *)(stage + (32 * (MB * wm + i) + row) * LINEAR8_K + 16 * c);
#pragma unroll
        for (int j = 0; j < NB; j++) fw[to][j] = *(const i32x4 *)(stage + (BM + 32 * (NB * wn + j) + row) * LINEAR8_K + 16 * c);
    };

    fetch(0, lds);
    if (steps > 1) fetch(1, lds + STAGE);
    arrive();
    if (steps == 1 && a.width % LINEAR8_K) cut(lds, a.width);
    read(lds, 0, 0);
    for (int t = 0; t < steps; t++) {
        int8_t *const here = lds + (t & 1) * STAGE, *const next = lds + (~t & 1) * STAGE;
#pragma unroll
        for (int kk = 0; kk < 4; kk++) {
            if (kk < 3)
                read(here, kk + 1, (kk + 1) & 1);
            else {
                arrive(); // the next stage is there, and nobody reads this one any more
                if (t + 1 < steps) {
                    if (t + 2 == steps && a.width % LINEAR8_K) cut(next, a.width - (t + 1) * LINEAR8_K);
                    read(next, 0, 0);
                }
                if (t + 2 < steps) fetch(t + 2, here);
            }
#pragma unroll
            for (int i = 0; i < MB; i++)
#pragma unroll
                for (int j = 0; j < NB; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[kk & 1][j], fx[kk & 1][i], acc[i][j], 0, 0, 0);
        }
    }

    // Results: a lane has channels 8 g + 4 (l / 32) .. of row l mod 32 of a block.  32 rows at a time go through a part of LDS that is the wave's own and leave it as whole rows.
    int8_t *const own = lds + wave * 32 * OUT_PITCH;
    constexpr int VEC = 16 / (int)sizeof(T), CHUNKS = 32 * NB / VEC; // a row's 16-byte pieces
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MB; i++) {
        const int m = m0 + 32 * (MB * wm + i), row = lane % 32;
        const float xs = a.x_scale[min(m + row, a.rows - 1)];
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const int col = 32 * j + 8 * g + 4 * (lane / 32);
                int sum[4];
#pragma unroll
                for (int e = 0; e < 4; e++) sum[e] = acc[i][j][4 * g + e];
                *(Vec<T, 4> *)(own + row * OUT_PITCH + col * (int)sizeof(T)) = linear8_results<T, 4>(a, sum, xs, n0 + 32 * NB * wn + col);
            }
        __builtin_amdgcn_wave_barrier();
        for (int p = lane; p < 32 * CHUNKS; p += 64) {
            const int r = p / CHUNKS, c = p % CHUNKS, n = n0 + 32 * NB * wn + c * VEC;
            const Vec<T, VEC> y = *(const Vec<T, VEC> *)(own + r * OUT_PITCH + 16 * c);
            if (m + r < a.rows) store_vec<T, VEC>(y, (T *)a.o + (m + r) * a.o_row, n, a.channels);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Few rows: 16 channels and 16 MB rows to a work-group, whose waves share the sum; operands come from memory straight into registers, each once, and the waves' sums are
// joined in LDS.
template <class T, int MB> __global__ __launch_bounds__(1024) void k_linear8_few(Linear8Args a)
{
    __shared__ i32x4 join[16][MB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MB;
    const int row = lane % 16, part = lane / 16 * 16;
    const int8_t *const w = a.w + (int64_t)min(n0 + row, a.channels - 1) * a.w_row;
    const int8_t *x[MB];
#pragma unroll
    for (int i = 0; i < MB; i++) x[i] = a.x + (int64_t)min(m0 + 16 * i + row, a.rows - 1) * a.x_row;
    i32x4 acc[MB];
#pragma unroll
    for (int i = 0; i < MB; i++) acc[i] = i32x4{};
    const int last = (a.width - 1) / 16 * 16; // the last piece of a row
    constexpr int U = 4;
    for (int k0 = wave * 64; k0 < a.width; k0 += waves * 64 * U) {
        i32x4 fw[U], fx[U][MB];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int k = min(k0 + u * waves * 64 + part, last); // behind the end the last piece again, which does not count
            fw[u] = *(const i32x4 *)(w + k);
#pragma unroll
            for (int i = 0; i < MB; i++) fx[u][i] = *(const i32x4 *)(x[i] + k);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int left = a.width - (k0 + u * waves * 64 + part); // numbers of the piece that count
            if (left < 16)
#pragma unroll
                for (int e = 0; e < 4; e++) fw[u][e] &= left >= 4 * e + 4 ? -1 : left <= 4 * e ? 0 : (int)((1u << 8 * (left - 4 * e)) - 1);
#pragma unroll
            for (int i = 0; i < MB; i++) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fx[u][i], acc[i], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < MB; i++) join[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < MB; i += waves) {
        i32x4 s = join[0][i][lane];
        for (int k = 1; k < waves; k++) s += join[k][i][lane];
        // a lane has channels 4 (l / 16) .. of row l mod 16
        const int m = m0 + 16 * i + row, n = n0 + lane / 16 * 4;
        if (m >= a.rows) continue;
        const int sum[4] = {s[0], s[1], s[2], s[3]};
        store_vec<T, 4>(linear8_results<T, 4>(a, sum, a.x_scale[m], n), (T *)a.o + m * a.o_row, n, a.channels);
    }
}
