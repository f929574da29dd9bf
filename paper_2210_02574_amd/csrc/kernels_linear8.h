// Product of 8-bit rows and 8-bit weights, both dense along the sum: o[m][n] = (sum over k of x[m][k] w[n][k]) x_scale[m] w_scale[n] + bias[n].
//
// Sums are exact in 32-bit integers.  A matrix instruction multiplies blocks of 32 x 32 numbers, whose operands are 16 bytes of a row for each lane: bytes of x and w
// that lanes hold in the same places are multiplied, so any order along k serves as long as both use it.
// Weights are operand A, rows of x operand B: a lane then holds four neighbouring channels of one row, which it can write together.
#pragma once
#include "enc_common.h"
#include <type_traits>

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

// 16 bytes for each lane from `at` of a buffer (zeros behind its end) to LDS, lane i's at to + 16 i, with no register in between.
// (Not in the template itself: the host's pass knows no such size and would drop the instance.)
__device__ __forceinline__ void fetch_lds(__amdgpu_buffer_rsrc_t from, unsigned at, int8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, at, 0, 0, 0);
}

// 16 bytes of each lane to `at` of a buffer, written to memory at once and past the last-level cache
__device__ __forceinline__ void store_through(i32x4 v, __amdgpu_buffer_rsrc_t to, int at)
{
    typedef int Words __attribute__((ext_vector_type(4)));
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(Words, v), to, at, 0, 2 | 1 << 4); // non-temporal; scope: the device
}

#define LINEAR8_K 128 // numbers of a row that a stage holds
// Chunk c of 16 bytes of row r lies at c ^ (r / 2 mod 8) of the row's 128 bytes in LDS: the 16 rows that a 16-byte read takes at a time then lie in 16 different places.
__device__ __forceinline__ int linear8_twist(int row) { return row >> 1 & 7; }

// A result: s x_scale w_scale + b.  From 2^64 on x_scale (FAR: where there may be such rows) comes last: a sum times it may leave 32 bits where the result does not,
// while one times w_scale then leaves them only where the result does.  Sums are below 2^31.
__device__ __forceinline__ bool linear8_far(float xs) { return fabsf(xs) >= 0x1p64f; }
template <bool FAR> __device__ __forceinline__ float linear8_scaled(int s, float xs, float ws, float b)
{
    const bool last = FAR && linear8_far(xs);
    return fmaf((float)s * (last ? ws : xs), last ? xs : ws, b);
}
// Four of them in their type.  Each is rounded to 32 bits first: in some places of some variants one instruction would round to fp16 alone, and a row's results hang on the rows beside it.
template <class T> __device__ __forceinline__ Vec<T, 4> linear8_typed(f32x4 y)
{
    if constexpr (std::is_same<T, f16>::value) asm("" : "+v"(y));
    Vec<T, 4> o;
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] = (T)y[e];
    return o;
}

// The tile of a work-group.  Each of the eight dies takes a run of tiles that follow one another, in bands of eight tiles of rows, so that they share operands in its L2.
__device__ __forceinline__ void linear8_tile(const Linear8Args &a, int &m, int &n)
{
    const int tiles = a.tiles_m * a.tiles_n, per = tiles / 8, extra = tiles % 8, die = blockIdx.x % 8;
    const int id = die * per + min(die, extra) + blockIdx.x / 8;
    constexpr int BAND = 8;
    const int band = id / (BAND * a.tiles_n), first = band * BAND, high = min(BAND, a.tiles_m - first), in = id - band * BAND * a.tiles_n;
    m = first + in % high, n = in / high;
}

// Tiles of 32 MB WM rows by 32 NB WN channels, WM x WN waves with MB x NB blocks of 32 x 32 each; G such groups of waves share the sum, each taking every G-th
// stage.  A stage is 128 bytes of every row of both, written to LDS by the loads themselves.  A group has two: the loads of one are under way for the whole of the other.  Per
// stage one barrier, ahead of its last products: behind it the next stage's first operands are read while those run.
// Large products are bound by the power limit: 16384 x 4096 x 4096 231 us (2380 TOPS, matrix instructions in 0.64 of the cycles), 180 us where all numbers are zero.  Short sums are
// bound by LDS, by a tile's first loads and by its results, which tiles of 128 cover with a second work-group on the CU: 16384 x 768 x 2304 in bf16 41 us, with tiles of 192 40
// (18 of them the rate of memory), 16384 x 2048 x 768 27 us.  What gained nothing: three or four stages, of 64 or 128 numbers; work-groups that go on to another tile, its first loads
// under way; blocks of 4 x 4 to a wave, or of 2 x 2 in tiles of 128, which read less of LDS with fewer waves; operands from memory to registers; wave priorities.
template <class T, int MB, int NB, int WM, int WN, int G, int OCC> __global__ __launch_bounds__(64 * WM * WN * G, OCC) void k_linear8(Linear8Args a)
{
    static_assert(G == 1 || (G == 4 && MB == 1 && NB == 1), "");
    constexpr int W = WM * WN, THREADS = 64 * W * G, BM = 32 * MB * WM, BN = 32 * NB * WN, STAGE = (BM + BN) * LINEAR8_K;
    constexpr int SIZE = (int)sizeof(T), VEC = 16 / SIZE;
    constexpr bool ALONE = G == 1 && 32 * NB * SIZE % 128 == 0; // a wave's results are whole lines, which it writes by itself
    constexpr int COLS = ALONE ? 32 * NB : BN, PITCH = COLS * SIZE + 16; // of a row of results in LDS, bytes
    constexpr int OUT = ALONE ? 32 * W * PITCH : G == 1 ? 32 * WM * PITCH : G * W * 4096 + BM * PITCH, LDS = G * 2 * STAGE > OUT ? G * 2 * STAGE : OUT;
    __shared__ __attribute__((aligned(1024))) int8_t lds[LDS];
    __shared__ __attribute__((aligned(16))) float sx[BM], sw[BN], sb[BN];
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = all % W, group = all / W, wm = wave % WM, wn = wave / WM;

    int tile_m, tile_n;
    linear8_tile(a, tile_m, tile_n);
    const int m0 = tile_m * BM, n0 = tile_n * BN;

    const int steps = (a.width + LINEAR8_K - 1) / LINEAR8_K, rounds = (steps + G - 1) / G, tail = a.width % LINEAR8_K;
    const int whole = (a.width + 15) / 16 * 16; // bytes of a row that may be read
    const int8_t *const xb = a.x + m0 * a.x_row, *const wb = a.w + n0 * a.w_row;
    const int bytes_m = (min(BM, a.rows - m0) - 1) * (int)a.x_row + whole, bytes_n = (min(BN, a.channels - n0) - 1) * (int)a.w_row + whole; // below 2^31: strides are below 2^23
    // One load of a wave brings eight rows.
    constexpr int LM = BM / 8 / W, LN = BN / 8 / W;
    static_assert(LM * 8 * W == BM && LN * 8 * W == BN, "");
    unsigned at_m[LM], at_n[LN];
#pragma unroll
    for (int i = 0; i < LM; i++) {
        const int row = 8 * (W * i + wave) + lane / 8;
        at_m[i] = (unsigned)row * (unsigned)a.x_row + 16 * (lane % 8 ^ linear8_twist(row));
    }
#pragma unroll
    for (int i = 0; i < LN; i++) {
        const int row = 8 * (W * i + wave) + lane / 8;
        at_n[i] = (unsigned)row * (unsigned)a.w_row + 16 * (lane % 8 ^ linear8_twist(row));
    }
    int8_t *const mine = lds + group * 2 * STAGE;
    const auto fetch = [&](int step, int8_t *stage) { // step < steps
        const int k = step * LINEAR8_K;
        const __amdgpu_buffer_rsrc_t rm = __builtin_amdgcn_make_buffer_rsrc((void *)(xb + k), 0, bytes_m - k, 0x00027000);
        const __amdgpu_buffer_rsrc_t rn = __builtin_amdgcn_make_buffer_rsrc((void *)(wb + k), 0, bytes_n - k, 0x00027000);
#pragma unroll
        for (int i = 0; i < LM; i++) fetch_lds(rm, at_m[i], stage + (W * i + wave) * 1024);
#pragma unroll
        for (int i = 0; i < LN; i++) fetch_lds(rn, at_n[i], stage + BM * LINEAR8_K + (W * i + wave) * 1024);
    };
    // Loads that write to LDS are waited for by hand: the barrier's own wait does not cover them.
    const auto arrive = [&] {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    // Behind the end of the sum: weights of its last stage from number `tail` on become zeros, so that what x's rows have there does not count.  All of a work-group
    // take part.
    const auto cut = [&](int8_t *stage) {
        for (int i = threadIdx.x; i < BN * 8; i += THREADS) {
            const int row = i / 8, left = tail - 16 * (i % 8); // numbers of this piece that count
            if (left >= 16) continue;
            i32x4 *const p = (i32x4 *)(stage + (BM + row) * LINEAR8_K + 16 * (i % 8 ^ linear8_twist(row)));
            i32x4 v = *p;
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] &= left >= 4 * e + 4 ? -1 : left <= 4 * e ? 0 : (int)((1u << 8 * (left - 4 * e)) - 1);
            *p = v;
        }
        __syncthreads();
    };
    const int last_round = (steps - 1) / G, last_group = (steps - 1) % G; // where the last stage is
    int8_t *const last_stage = lds + (last_group * 2 + (last_round & 1)) * STAGE;

    i32x16 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NB; j++) acc[i][j] = i32x16{};
    i32x4 fx[2][MB], fw[2][NB];
    // operands of the numbers 32 kk .. of a stage: lane's row l mod 32 of each block, 16 numbers
    const auto read = [&](const int8_t *stage, int kk, int to) {
        const int row = lane % 32, c = (2 * kk + lane / 32) ^ linear8_twist(row);
#pragma unroll
        for (int j = 0; j < NB; j++) fw[to][j] = *(const i32x4 *)(stage + (BM + 32 * (NB * wn + j) + row) * LINEAR8_K + 16 * c);
#pragma unroll
        for (int i = 0; i < MB; i++) fx[to][i] = *(const i32x4 *)(stage + (32 * (MB * wm + i) + row) * LINEAR8_K + 16 * c);
    };

    if (group < steps) fetch(group, mine);
    if (group + G < steps) fetch(group + G, mine + STAGE);
    for (int i = threadIdx.x; i < BM + BN; i += THREADS) {
        if (i < BM)
            sx[i] = a.x_scale[min(m0 + i, a.rows - 1)];
        else {
            const int n = min(n0 + i - BM, a.channels - 1);
            sw[i - BM] = a.w_scale[n];
            sb[i - BM] = !a.bias ? 0.f : a.bias32 ? ((const float *)a.bias)[n] : (float)((const T *)a.bias)[n];
        }
    }
    arrive();
    if (last_round == 0 && tail) cut(last_stage);
    read(mine, 0, 0);
    for (int t = 0; t < rounds; t++) {
        int8_t *const here = mine + (t & 1) * STAGE, *const next = mine + (~t & 1) * STAGE;
        const bool some = G == 1 || t * G + group < steps;
#pragma unroll
        for (int kk = 0; kk < 4; kk++) {
            if (kk < 3)
                read(here, kk + 1, (kk + 1) & 1);
            else {
                arrive(); // the next stage is there, and nobody reads this one any more
                if (t + 1 < rounds) {
                    if (t + 1 == last_round && tail) cut(last_stage);
                    read(next, 0, 0);
                }
                if ((t + 2) * G + group < steps) fetch((t + 2) * G + group, here);
            }
            if (some)
#pragma unroll
                for (int i = 0; i < MB; i++)
#pragma unroll
                    for (int j = 0; j < NB; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[kk & 1][j], fx[kk & 1][i], acc[i][j], 0, 0, 0);
        }
    }

    // Results: a lane has channels 8 g + 4 (l / 32) .. of row l mod 32 of a block.  They leave through LDS as whole pieces of rows, a wave's or the
    // tile's.  Where those are whole lines they are written
    // to memory as they come: the next kernel begins with another L2, and what is written early need not be when this one ends; and operands stay in the last-level cache
    // (16384 x 768 x 2304 in bf16 behind the norm, three sets of inputs in turn, 58 us, 71 with lines kept there; 16384 x 4096 x 4096 231, 256; four layers of an encoder on 32 sentences
    // of 512 1.06 ms, 1.09).  Parts of lines have to meet in L2 (16384 x 64 x 3000: 30 us, 54 without).
    const int64_t pitch = a.o_row * SIZE;
    const bool through = (((int64_t)a.o | pitch) & 127) == 0 && pitch < (1 << 23); // (offsets inside a tile have 32 bits)
    const __amdgpu_buffer_rsrc_t ro = __builtin_amdgcn_make_buffer_rsrc((int8_t *)a.o + m0 * pitch, 0, through ? min(BM, a.rows - m0) * (int)pitch : 0, 0x00027000);
    const int row = lane % 32, h = lane / 32;
    const auto scaled = [&](const i32x4 s, float xs, int col, auto far) {
        const f32x4 ws = *(const f32x4 *)(sw + col), b = *(const f32x4 *)(sb + col);
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; e++) y[e] = linear8_scaled<far>(s[e], xs, ws[e], b[e]);
        return linear8_typed<T>(y);
    };
    const auto store = [&](const Vec<T, VEC> y, int m, int n) { // row m of the tile
        if (m0 + m >= a.rows) return;
        if (n + VEC <= a.channels && through)
            store_through(__builtin_bit_cast(i32x4, y), ro, m * (int)pitch + n * SIZE);
        else
            store_vec<T, VEC>(y, (T *)((int8_t *)a.o + (m0 + m) * pitch), n, a.channels);
    };
    __syncthreads();
    constexpr int CHUNKS = COLS / VEC;
    if constexpr (G == 1) { // 32 rows of each wave at a time
        constexpr int SHARE = ALONE ? 64 : THREADS, PER = (ALONE ? 32 : 32 * WM) * CHUNKS / SHARE;
        static_assert(PER * SHARE == (ALONE ? 32 : 32 * WM) * CHUNKS, "");
        int8_t *const own = lds + (ALONE ? wave * 32 * PITCH : 0);
        const int me = ALONE ? lane : threadIdx.x, first_row = ALONE ? 0 : 32 * wm, first_col = ALONE ? COLS * wn : 0;
        const auto exchange = [] {
            if constexpr (ALONE) { // between the lanes of a wave
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            } else
                __syncthreads();
        };
#pragma unroll
        for (int i = 0; i < MB; i++) {
            if (i) exchange();
            const float xs = sx[32 * (MB * wm + i) + row];
            const auto put = [&](auto far) {
#pragma unroll
                for (int j = 0; j < NB; j++)
#pragma unroll
                    for (int g = 0; g < 4; g++) {
                        const int col = 32 * (NB * wn + j) + 8 * g + 4 * h;
                        const i32x4 s = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                        *(Vec<T, 4> *)(own + (first_row + row) * PITCH + (col - first_col) * SIZE) = scaled(s, xs, col, far);
                    }
            };
            if (__builtin_expect(__ballot(linear8_far(xs)) != 0, 0)) // (rather than a choice for each result)
                put(std::true_type{});
            else
                put(std::false_type{});
            exchange();
            Vec<T, VEC> y[PER];
#pragma unroll
            for (int p = 0; p < PER; p++) {
                const int at = p * SHARE + me;
                y[p] = *(const Vec<T, VEC> *)(own + at / CHUNKS * PITCH + 16 * (at % CHUNKS));
            }
#pragma unroll
            for (int p = 0; p < PER; p++) {
                const int at = p * SHARE + me, r = at / CHUNKS;
                store(y[p], ALONE ? 32 * (MB * wm + i) + r : 32 * (MB * (r / 32) + i) + r % 32, n0 + first_col + at % CHUNKS * VEC);
            }
        }
    } else { // each of the four groups joins a quarter of all groups' sums of each block
        i32x4 *const join = (i32x4 *)lds + wave * G * 256; // [group][quarter][lane]
#pragma unroll
        for (int g = 0; g < 4; g++) join[(group * 4 + g) * 64 + lane] = i32x4{acc[0][0][4 * g], acc[0][0][4 * g + 1], acc[0][0][4 * g + 2], acc[0][0][4 * g + 3]};
        __syncthreads();
        i32x4 s = {};
#pragma unroll
        for (int g = 0; g < G; g++) s += join[(g * 4 + group) * 64 + lane];
        int8_t *const out = lds + G * W * 4096;
        const int m = 32 * wm + row, col = 32 * wn + 8 * group + 4 * h;
        *(Vec<T, 4> *)(out + m * PITCH + col * SIZE) = scaled(s, sx[m], col, std::true_type{});
        __syncthreads();
        for (int p = threadIdx.x; p < BM * CHUNKS; p += THREADS)
            store(*(const Vec<T, VEC> *)(out + p / CHUNKS * PITCH + 16 * (p % CHUNKS)), p / CHUNKS, n0 + p % CHUNKS * VEC);
    }
}

// Few tiles: BLK rows by BLK channels, 16 or 32, and G waves that share the sum, each with two stages of its own, which it alone waits for: no barrier until the waves' sums are joined.
// What bounds it is how much the card has under way and, of short sums, a launch and two trips to memory: 32 x 8192 x 1024 4.5 us (7.8 where
// barriers keep eight waves together on tiles of 32), 23 x 768 x 768 3.0 us (3.6).
template <class T, int BLK, int G> __global__ __launch_bounds__(64 * G) void k_linear8_few(Linear8Args a)
{
    constexpr int ROWS = BLK * LINEAR8_K, STAGE = 2 * ROWS, LOADS = BLK / 8;       // bytes of a stage's rows of x, of all of it; loads that bring the former
    constexpr int KK = BLK == 32 ? 4 : 2, PARTS = 64 / BLK, QUARTERS = BLK * BLK / 256; // matrix instructions to a stage; lanes to a row; results of a lane, by fours
    __shared__ __attribute__((aligned(1024))) int8_t lds[G * 2 * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile_m, tile_n;
    linear8_tile(a, tile_m, tile_n);
    const int m0 = tile_m * BLK, n0 = tile_n * BLK;
    const int steps = (a.width + LINEAR8_K - 1) / LINEAR8_K, tail = a.width % LINEAR8_K, whole = (a.width + 15) / 16 * 16;
    const int8_t *const xb = a.x + m0 * a.x_row, *const wb = a.w + n0 * a.w_row;
    const int bytes_m = (min(BLK, a.rows - m0) - 1) * (int)a.x_row + whole, bytes_n = (min(BLK, a.channels - n0) - 1) * (int)a.w_row + whole;
    unsigned at_m[LOADS], at_n[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
        const int row = 8 * i + lane / 8, c = 16 * (lane % 8 ^ linear8_twist(row));
        at_m[i] = (unsigned)row * (unsigned)a.x_row + c;
        at_n[i] = (unsigned)row * (unsigned)a.w_row + c;
    }
    int8_t *const mine = lds + wave * 2 * STAGE;
    const auto fetch = [&](int step, int8_t *stage) { // step < steps
        const int k = step * LINEAR8_K;
        const __amdgpu_buffer_rsrc_t rm = __builtin_amdgcn_make_buffer_rsrc((void *)(xb + k), 0, bytes_m - k, 0x00027000);
        const __amdgpu_buffer_rsrc_t rn = __builtin_amdgcn_make_buffer_rsrc((void *)(wb + k), 0, bytes_n - k, 0x00027000);
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            fetch_lds(rm, at_m[i], stage + i * 1024);
            fetch_lds(rn, at_n[i], stage + ROWS + i * 1024);
        }
    };
    typedef typename std::conditional<BLK == 32, i32x16, i32x4>::type Sums;
    Sums acc = {};
    const int row = lane % BLK, part = lane / BLK;
    if (wave < steps) fetch(wave, mine);
    if (wave + G < steps) fetch(wave + G, mine + STAGE);
    for (int t = 0, step = wave; step < steps; t ^= 1, step += G) {
        int8_t *const stage = mine + t * STAGE;
        if (step + G < steps) // the next stage's loads may be under way
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        i32x4 fx[KK], fw[KK];
#pragma unroll
        for (int kk = 0; kk < KK; kk++) {
            const int at = row * LINEAR8_K + 16 * ((PARTS * kk + part) ^ linear8_twist(row));
            fx[kk] = *(const i32x4 *)(stage + at);
            fw[kk] = *(const i32x4 *)(stage + ROWS + at);
        }
        if (step + 1 == steps && tail) // numbers of weights behind the end of the sum
#pragma unroll
            for (int kk = 0; kk < KK; kk++) {
                const int left = tail - 16 * (PARTS * kk + part);
#pragma unroll
                for (int e = 0; e < 4; e++) fw[kk][e] &= left >= 4 * e + 4 ? -1 : left <= 4 * e ? 0 : (int)((1u << 8 * (left - 4 * e)) - 1);
            }
#pragma unroll
        for (int kk = 0; kk < KK; kk++) {
            if constexpr (BLK == 32)
                acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[kk], fx[kk], acc, 0, 0, 0);
            else
                acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[kk], fx[kk], acc, 0, 0, 0);
        }
        if (step + 2 * G < steps) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // this one has been read
            fetch(step + 2 * G, stage);
        }
    }
    __syncthreads();
    i32x4 *const join = (i32x4 *)lds; // [wave][quarter][lane]
#pragma unroll
    for (int p = 0; p < QUARTERS; p++) join[(wave * QUARTERS + p) * 64 + lane] = i32x4{acc[4 * p], acc[4 * p + 1], acc[4 * p + 2], acc[4 * p + 3]};
    __syncthreads();
    if (wave >= QUARTERS) return;
    i32x4 s = {};
#pragma unroll
    for (int g = 0; g < G; g++) s += join[(g * QUARTERS + wave) * 64 + lane];
    const int m = m0 + row, n = n0 + 8 * wave + 4 * part; // four channels of a row
    if (m >= a.rows) return;
    const float xs = a.x_scale[m];
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const int c = min(n + e, a.channels - 1);
        const float b = !a.bias ? 0.f : a.bias32 ? ((const float *)a.bias)[c] : (float)((const T *)a.bias)[c];
        y[e] = linear8_scaled<true>(s[e], xs, a.w_scale[c], b);
    }
    store_vec<T, 4>(linear8_typed<T>(y), (T *)a.o + m * a.o_row, n, a.channels);
}
