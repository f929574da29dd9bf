// Attention inside each sequence of a batch, forward and backward, by matrix instructions.
//
//   t_ij = scale q_i . k_j, u_ij = cap tanh(t_ij / cap) (no cap: t_ij), s_ij = u_ij - slope_h |pos_i - pos_j|
//   lse_i = log sum_j exp(s_ij), p_ij = exp(s_ij - lse_i), o_i = sum_j p_ij v_j; no keys: o_i = 0, lse_i = -inf
//   delta_i = do_i . o_i, dp_ij = do_i . v_j, ds_ij = p_ij (dp_ij - delta_i), dt_ij = ds_ij (1 - (u_ij / cap)^2) scale
//   dv_j = sum_i p_ij do_i, dk_j = sum_i dt_ij q_i, dq_i = sum_j dt_ij k_j (dv, dk: over the query heads that share the key head too)
//
// One layout carries all three kernels.  A 32 x 32 product C = A B leaves lane l with column l mod 32 and the rows 8 (r / 4) + 4 (l / 32) + r mod 4,
// r < 16.  The rows of a work-group's own tile (queries in the forward pass and for dq, keys for dk and dv) are the columns n, the rows that
// stream by are the rows m.  So a softmax statistic belongs to one lane and its partner 32 further on; and eight of a lane's values of C, rounded, are
// its operand B of the next product over those rows, whose order inside a block of 16 does not matter as long as A has the same one:
// slot (l / 32, e) holds row 4 (l / 32) + e for e < 4 and 8 + 4 (l / 32) + e - 4 above.  Nothing moves between lanes on the way.
// The operand A of that product is a transposed tile: 16-bit types read it from LDS with the transposing read, 32-bit ones word by word.
//
// Roundings: products take p and dt in the type of the inputs (16 bits: relative 2^-8 or 2^-11 of each term at most, as the inputs themselves have),
// everything else, sums and statistics included, is in 32 bits.  (dt is rounded before its factor scale.)  Rounding both the terms and the result leaves 1.4
// times the error of rounding the result alone.  delta takes o as it was rounded: its error has the size of that rounding, |do . o| 2^-8 or 2^-11 at most, and matters where
// o is not small beside the values' own spread: under a steep distance bias, which leaves few keys with a weight whatever the data are, dq and dk had 1.55 times the error of
// rounding the result alone.  With a bias it is therefore mended (k_attn_grad_q, which also says what it is otherwise), and for up to 32 keys of short sequences, which are at hand
// at once, delta is exact.
// fp16 has the bits for all of this but not the range: there factors are lifted by powers of two, weights by constants (attn_lift, GRAD_LIFT), ds by what
// k_attn_grad_size finds.
#pragma once
#include "enc_common.h"
#include <type_traits>

struct AttnArgs {
    const void *q, *k, *v, *o_in, *go; // o_in, go: the forward pass's o and the gradient that reaches it (backward)
    void *o, *dq, *dk, *dv;
    float *lse;         // [heads][rows_q], natural logarithm
    float *delta;       // [heads][rows_q]
    float *v_size, *go_size; // fp16, backward: [slots of keys or queries][kv_heads], k_attn_grad_size
    float *part_o;      // forward: [splits][heads][rows_q][dim]; dk and dv: [splits][2][kv_heads][rows_k][dim]
    float *part_lse;    // [splits][heads][rows_q]
    const float *slope; // [heads] or null
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, oi_row, oi_head, go_row, go_head; // strides, in elements
    int64_t dq_row, dq_head, dk_row, dk_head, dv_row, dv_head;
    Spans sq, sk;
    int heads, group, dim; // group: query heads that share a key head
    float scale, cap;
    int slots, splits, fill;
    int pack; // few queries: query heads of one key head that lie side by side in a tile, `group` or 1
    unsigned work; // work-groups that have something to do
    int slots_q, tile_q, slots_k, tile_k; // of the backward pass, in both of its kernels
};

template <class T> struct AttnType;
template <> struct AttnType<f16> {
    static __device__ __forceinline__ f32x16 mma(Vec<f16, 8> a, Vec<f16, 8> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct AttnType<bf16> {
    static __device__ __forceinline__ f32x16 mma(Vec<bf16, 8> a, Vec<bf16, 8> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct AttnType<float> {
    // slot (l / 32, e): eight products over two rows each
    static __device__ __forceinline__ f32x16 mma(Vec<float, 8> a, Vec<float, 8> b, f32x16 c)
    {
#pragma unroll
        for (int e = 0; e < 8; e++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

#define ATTN_THREADS 256
#define LOG2E 1.44269504088896340736f
#define LN2 0.69314718055994530942f

// The value of the other lane of the pair (l, l + 32), joined.
__device__ __forceinline__ float pair_max(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float pair_sum(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// Tiles in LDS, rows of DP elements in 16-byte chunks.  LDS has 64 banks of 4 bytes, 16 chunks, and takes 16 lanes of a 16-byte read at a time: one
// chunk of 16 rows; or 32 lanes of a transposing read: four neighbouring chunks of four rows.  Chunk c of row r is stored at c ^ twist(r), which gives
// both of them 16 different places.
template <class T, int DP> struct AttnTile {
    static constexpr int VEC = 16 / (int)sizeof(T); // elements of a chunk
    static constexpr int CHUNKS = DP / VEC;
    typedef Vec<T, VEC> Chunk;

    static __device__ __forceinline__ int twist(int row)
    {
        // Four neighbouring rows four chunks apart, as far as the row's length does not do that by itself; rows four apart in the chunks between.
        if constexpr (CHUNKS % 16 == 0) return (row & 3) << 2 | (row >> 2 & 3); // 256 bytes
        if constexpr (CHUNKS % 8 == 0) return (row << 1 & 4) | (row >> 1 & 2) | (row >> 3 & 1);
        return row >> 2 & 3; // 64 or 192
    }
    static __device__ __forceinline__ int place(int row, int chunk) { return (row * CHUNKS + (chunk ^ twist(row))) * VEC; }

    // ROWS rows by `NT` threads: from memory to registers, zeros for the rows from `end` on and the columns from dim on.  The reads go through a
    // buffer descriptor whose length is that of the rows that are there: behind it they return zeros, without a comparison or an address in
    // 64 bits per read (row strides are below 2^24 bytes).
    template <int ROWS, int NT> static constexpr int per() { return (ROWS * CHUNKS + NT - 1) / NT; }
    template <int ROWS, int NT> struct Reads {
        unsigned at[per<ROWS, NT>()]; // bytes from the first row
        __device__ __forceinline__ Reads(int64_t stride, int dim, int tid)
        {
#pragma unroll
            for (int i = 0; i < per<ROWS, NT>(); i++) {
                const int n = i * NT + tid, col = (n % CHUNKS) * VEC;
                at[i] = n < ROWS * CHUNKS && col < dim ? (unsigned)(n / CHUNKS * (int)stride + col) * (unsigned)sizeof(T) : 0xfffffff0u;
            }
        }
        __device__ __forceinline__ void load(Chunk (&c)[per<ROWS, NT>()], const T *base, int64_t stride, int first, int end, int dim) const
        {
            const int rows = min(max(end - first, 0), ROWS), bytes = rows ? ((rows - 1) * (int)stride + dim) * (int)sizeof(T) : 0;
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)(base + first * stride), 0, bytes, 0x00027000);
#pragma unroll
            for (int i = 0; i < per<ROWS, NT>(); i++) c[i] = __builtin_bit_cast(Chunk, __builtin_amdgcn_raw_buffer_load_b128(r, at[i], 0, 0));
        }
    };
    // .. and from registers to LDS
    template <int ROWS, int NT> static __device__ __forceinline__ void store(const Chunk (&c)[per<ROWS, NT>()], T *lds, int tid)
    {
#pragma unroll
        for (int i = 0; i < per<ROWS, NT>(); i++) {
            const int at = i * NT + tid;
            if (at < ROWS * CHUNKS) *(Chunk *)(lds + place(at / CHUNKS, at % CHUNKS)) = c[i];
        }
    }
    // operand A or B: lane's row `row0 + l mod 32` (row0: a multiple of 32), columns 16 kk + 8 (l / 32) ..
    static __device__ __forceinline__ Vec<T, 8> rows(const T *lds, int row0, int kk, int lane)
    {
        const int row = lane & 31, col = 16 * kk + 8 * (lane >> 5);
        const T *p = lds + row0 * DP;
        if constexpr (sizeof(T) == 4) {
            const f32x4 a = *(const f32x4 *)(p + place(row, col / VEC)), b = *(const f32x4 *)(p + place(row, col / VEC + 1));
            return Vec<T, 8>{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        } else
            return *(const Vec<T, 8> *)(p + place(row, col / VEC));
    }
    static __device__ __forceinline__ Vec<T, 8> eight(const T *p) // of memory
    {
        if constexpr (sizeof(T) == 4) {
            const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
            return Vec<T, 8>{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        } else
            return *(const Vec<T, 8> *)p;
    }
    // operand A of a transposed tile: lane's column 32 db + l mod 32, the rows row0 + .. (row0: a multiple of 16) in slot order
    static __device__ __forceinline__ Vec<T, 8> cols(const T *lds, int row0, int db, int lane)
    {
        const int h = lane >> 5;
        const T *p = lds + row0 * DP;
        if constexpr (sizeof(T) == 4) {
            const int col = 32 * db + (lane & 31);
            Vec<T, 8> x;
#pragma unroll
            for (int e = 0; e < 8; e++) x[e] = p[place(4 * h + (e & 3) + 8 * (e >> 2), col / VEC) + col % VEC];
            return x;
        } else {
            // 16 lanes read four rows of 16 elements, four lanes to a row; lane j of them gets element j of each row
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef short s8 __attribute__((ext_vector_type(8)));
            typedef __attribute__((address_space(3))) s4 *Ptr;
            const int j = lane & 15, col = 32 * db + (lane & 16) + (j & 3) * 4;
            const int row = 4 * h + (j >> 2);
            const s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(p + place(row, col / VEC) + col % VEC));
            const s4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(p + place(row + 8, col / VEC) + col % VEC));
            const s8 x = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            return __builtin_bit_cast(Vec<T, 8>, x);
        }
    }
    // the operand from memory: row `row` of base, or zeros
    static __device__ __forceinline__ Vec<T, 8> own(const T *base, int64_t stride, int row, bool in, int kk, int dim, int lane)
    {
        const int col = 16 * kk + 8 * (lane >> 5);
        Vec<T, 8> x = {};
        if (in && col < dim) x = eight(base + row * stride + col);
        return x;
    }
};

// eight of a lane's values of C as operand B
template <class T> __device__ __forceinline__ Vec<T, 8> round8(const f32x16 &c, int half)
{
    Vec<T, 8> x;
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = (T)c[8 * half + e];
    return x;
}

// a lane's column of C^T blocks, times f, as a row of memory
template <class T, int DB> __device__ __forceinline__ void store_row(const f32x16 (&c)[DB], float f, T *row, int dim, int lane)
{
    const int h = lane >> 5;
#pragma unroll
    for (int db = 0; db < DB; db++)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int col = 32 * db + 2 * r + 4 * h;
            Vec<T, 4> x;
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = (T)(c[db][r + e] * f);
            if (col < dim) *(Vec<T, 4> *)(row + col) = x;
        }
}

// Work-group -> (head, slot, split), neighbours on one of the eight dies' caches: work-groups go to the dies in turn, so die d is given
// the d-th eighth of the work, in which tiles of one head, which read the same keys, come one after the other.  (All heads of a tile one after the
// other instead: 2 sequences of 16384 4 % slower, 64 of up to 512 2 to 5 %.)
__device__ __forceinline__ bool attn_work(const AttnArgs &a, unsigned per_head, int &head, int &slot, int &split)
{
    const unsigned w = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    if (w >= a.work) return false;
    head = w / per_head;
    const unsigned r = w % per_head;
    split = r % a.splits;
    slot = r / a.splits;
    return true;
}

// Scores of 32 x 32 blocks, x = log2(e) s, from products c = q . k.  MODE: MODE_CAP, MODE_SLOPE, both or neither.  16-bit types take tanh(y) =
// 1 - 2 / (1 + e^2y) by the hardware's exponential and reciprocal: it is off by 2^-22 at most, but absolutely, so that a score is off by that times the
// cap, however small it is.  Up to caps of 64 that is 2^-16, a 32nd of what rounding its weight to fp16 costs (bf16: a 256th).  Above (MODE_EXACT),
// and in 32 bits, tanh is the library's, which keeps small values: a cap may be far above all scores.  3 sequences of 4000, 16 heads of 64 on 8 in fp16, biased,
// caps of 64 and 65: 375 us forward and 1106 backward, 446 and 1468; 32 of 300, 12 heads of 64: 32 and 96, 41 and 126.
enum { MODE_CAP = 1, MODE_SLOPE = 2, MODE_EXACT = 4 };
#define ATTN_FAST_CAP 64.f
template <class T, int MODE> constexpr bool attn_fast_tanh() { return sizeof(T) == 2 && (MODE & MODE_CAP) && !(MODE & MODE_EXACT); }
template <class T, int MODE> struct Scores {
    float in, out, slope; // of c before tanh, of tanh (or of c), of the distance
    float unit;           // of c: to score / cap

    __device__ __forceinline__ Scores(const AttnArgs &a, int head)
    {
        out = a.scale * LOG2E;
        if (MODE & MODE_CAP) {
            out = a.cap * LOG2E;
            unit = a.scale / a.cap;
            in = attn_fast_tanh<T, MODE>() ? unit * (2.f * LOG2E) : unit;
        }
        if (MODE & MODE_SLOPE) slope = a.slope[head] * LOG2E;
    }
    // what is left to multiply scores with: without a cap or a bias the exponential's fma does it
    __device__ __forceinline__ float rest() const { return MODE ? 1.f : out; }
    // pos: position of the lane's own row minus the one of row 0 of the block: the distance of row m is |pos - m|
    // lone: they are all that a row has.  lse in 32 bits is as exact as they are then (of two keys under a cap of 50 it was off by 2e-6 of itself; from 32 on errors
    // of the scores cancel), so tanh is the library's.
    __device__ __forceinline__ void operator()(f32x16 &c, float pos, int h, bool lone) const
    {
        if constexpr (MODE != 0) {
            const float p = pos - (float)(4 * h);
#pragma unroll
            for (int r = 0; r < 16; r++) {
                float x;
                if constexpr (MODE & MODE_CAP) {
                    if (attn_fast_tanh<T, MODE>() && !lone) {
                        const float g = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(c[r] * in));
                        x = fmaf(-2.f * out, g, out);
                    } else {
                        x = tanhf(c[r] * unit);
                        x *= out;
                    }
                } else
                    x = c[r] * out;
                if constexpr (MODE & MODE_SLOPE) x = fmaf(-slope, fabsf(p - (float)(8 * (r >> 2) + (r & 3))), x);
                c[r] = x;
            }
        }
    }
};

// ---- forward ---------------------------------------------------------------------------------------------------------

// The rows of a work-group's tile and the keys that it reads, the same for both kernels of the forward pass.
struct FwdRange {
    TileRows t;
    int kb, ke; // the sequence's keys
    int lo, hi; // those of this split
    int back;   // a query row's position among the keys, the first at 0, is its number plus this
    __device__ __forceinline__ FwdRange(const AttnArgs &a, const TileRows &t, int split, int tile) : t(t)
    {
        kb = t.other_begin, ke = t.other_end;
        back = (ke - kb) - t.end;
        if (t.first >= t.end || t.top <= t.begin) ke = kb; // a tile between sequences: nothing to sum
        const int tiles = (ke - kb + tile - 1) / tile, per = (tiles + a.splits - 1) / a.splits;
        lo = kb + min(split * per, tiles) * tile, hi = min(ke, kb + min((split + 1) * per, tiles) * tile);
    }
};

// Weights refer to the running maximum, which may be 8 behind: they are at most 2^8.  In fp16, whose numbers end at 2^-25, they are lifted by 2^7 more, as far as
// its 65504 allow, so that many small weights beside a large one still count: a weight is off by 2^-32 of the largest (not lifted, 60000 weights of 2^-25.2
// were zeros, 0.0016 of the sum).  It costs nothing: the lift is in what the exponent is taken less of.
template <class T> constexpr float attn_lift() { return std::is_same<T, f16>::value ? 7.f : 0.f; }

// A row's result: its sum of weights, the maximum that they refer to (in units of log2) and the weighted sum of values in o.
template <class T, int DB> __device__ __forceinline__ void fwd_store(const AttnArgs &a, const FwdRange &g, int head, int split, int row, float top, float sum, f32x16 (&o)[DB], int lane)
{
    const bool in = row >= g.t.begin && row < g.t.end;
    if (row >= g.t.top || (!in && !a.fill)) return;
    // a row without keys, and a row of no sequence: zeros
    const bool some = in && g.hi > g.lo;
    const float f = some ? 1.f / sum : 0.f, lse = some ? (top - attn_lift<T>() + __builtin_amdgcn_logf(sum)) * LN2 : -INFINITY;
    const int64_t at = (int64_t)head * a.sq.rows + row;
    if (a.splits > 1) {
        const int64_t part = (int64_t)split * a.heads * a.sq.rows + at;
        if (lane < 32) a.part_lse[part] = lse;
        if (some) store_row<float, DB>(o, f, a.part_o + part * a.dim, a.dim, lane);
        return;
    }
    if (lane < 32) a.lse[at] = lse;
    if (!some) // not 0 * o: the row may hold what a zero does not clear
#pragma unroll
        for (int db = 0; db < DB; db++) o[db] = f32x16{};
    store_row<T, DB>(o, f, (T *)a.o + head * a.o_head + row * a.o_row, a.dim, lane);
}

// scores of missing keys: rows of C from `left` on
__device__ __forceinline__ void mask_rows(f32x16 &s, int left, int h)
{
#pragma unroll
    for (int r = 0; r < 16; r++)
        if (8 * (r >> 2) + 4 * h + (r & 3) >= left) s[r] = -INFINITY;
}
__device__ __forceinline__ float col_max(const f32x16 &s)
{
    float m = s[0];
#pragma unroll
    for (int r = 1; r < 16; r++) m = fmaxf(m, s[r]);
    return pair_max(m);
}

// Many queries: four waves with 32 QB queries each, all of which read all keys.  A step takes 32 keys: the products of the next step's scores are
// independent of this step's exponentials, so that matrix and vector instructions of one wave overlap.  Tiles of BN keys pass through three LDS
// stages, which takes one barrier a tile: the stage that a wave overwrites is the one that every wave has left before the last barrier.
// 12 heads of 128 on 4 key heads, 16384 rows of bf16: 1.70 ms, 970 TF, 0.80 of what a library product of 8192^3 reaches on the card (1208); matrix instructions
// take 0.47 of the cycles, vector instructions 0.50, at the clock that the power limit leaves (1.7 to 1.9 GHz).  64 sequences of 277 rows on average, 12 heads of
// 64: 44 us: a work-group has 9 steps then, and spends a third of its time on its first loads and its store.
// Tried and not kept: no maximum per step, weights watched by their sums instead (heads of 32 1.1 times as fast, of 64 and 128 1.02, a steep distance bias 0.87);
// the weighted sum one step later, so that all of a step's products and exponentials are independent (85 registers more, 0.85); waves without rows
// skipping their products (full tiles 0.93).
template <class T, int DP, int QB> struct AttnFwd {
    // Two blocks of queries halve what is read of LDS for a product; heads above 64 then take the registers of one wave per SIMD, everything
    // else leaves room for two or three, and its stages for as many work-groups.
    static constexpr int BM = 128 * QB, BN = QB == 1 && DP * sizeof(T) > 128 ? 32 : 64, SUB = BN / 32;
    static constexpr int WAVES = sizeof(T) == 4 || (QB == 2 && DP > 64) ? 1 : 2;
    static constexpr int TILE = BN * DP; // elements
};
template <class T, int DP, int QB, int MODE> __global__ __launch_bounds__(ATTN_THREADS, (AttnFwd<T, DP, QB>::WAVES)) void k_attn(AttnArgs a)
{
    typedef AttnFwd<T, DP, QB> F;
    typedef AttnTile<T, DP> L;
    constexpr int BN = F::BN, SUB = F::SUB, KK = DP / 16, DB = DP / 32;
    __shared__ __attribute__((aligned(16))) T lds[3][2][F::TILE];

    int head, slot, split;
    if (!attn_work(a, a.slots * a.splits, head, slot, split)) return;
    const TileRows t = tile_rows(a.sq, a.sk, slot, F::BM);
    if (t.first >= t.top) return;
    const FwdRange g(a, t, split, BN);
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row0 = t.first + 32 * QB * wave + (lane & 31); // and 32 further on for each block

    const T *const q = (const T *)a.q + head * a.q_head;
    const T *const k = (const T *)a.k + (head / a.group) * a.k_head, *const v = (const T *)a.v + (head / a.group) * a.v_head;
    typename L::Chunk ck[L::template per<BN, ATTN_THREADS>()], cv[L::template per<BN, ATTN_THREADS>()];
    const typename L::template Reads<BN, ATTN_THREADS> reads_k(a.k_row, a.dim, tid), reads_v(a.v_row, a.dim, tid);
    const auto load = [&](int j) {
        reads_k.load(ck, k, a.k_row, j, g.hi, a.dim);
        reads_v.load(cv, v, a.v_row, j, g.hi, a.dim);
    };
    const auto store = [&](int stage) {
        L::template store<BN, ATTN_THREADS>(ck, lds[stage][0], tid);
        L::template store<BN, ATTN_THREADS>(cv, lds[stage][1], tid);
    };
    load(g.lo);
    Vec<T, 8> fq[QB][KK];
#pragma unroll
    for (int b = 0; b < QB; b++)
#pragma unroll
        for (int kk = 0; kk < KK; kk++) {
            const int row = row0 + 32 * b;
            fq[b][kk] = L::own(q, a.q_row, row, row < t.top && row >= t.begin && row < t.end, kk, a.dim, lane);
        }
    const Scores<T, MODE> scores(a, head);
    const float c2 = scores.rest(); // scores are kept times this below
    float top[QB], sum[QB], m[QB];  // the maximum that sums refer to (in units of log2), the lane's own sum, the maximum of the scores at hand
    f32x16 o[QB][DB], s[QB];
#pragma unroll
    for (int b = 0; b < QB; b++) {
        top[b] = -INFINITY, sum[b] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; db++) o[b][db] = f32x16{};
    }
    // operands of the 32 keys in rows `at` .. of a stage: keys, and values by halves
    Vec<T, 8> fk[KK], fv[2][DB];
    const auto read_keys = [&](const T *lk, int at) {
#pragma unroll
        for (int kk = 0; kk < KK; kk++) fk[kk] = L::rows(lk, at, kk, lane);
    };
    const auto read_values = [&](const T *lv, int at, int half) {
#pragma unroll
        for (int db = 0; db < DB; db++) fv[half][db] = L::cols(lv, at + 16 * half, db, lane);
    };
    const auto products = [&](f32x16 (&x)[QB]) {
#pragma unroll
        for (int b = 0; b < QB; b++) x[b] = f32x16{};
#pragma unroll
        for (int kk = 0; kk < KK; kk++)
#pragma unroll
            for (int b = 0; b < QB; b++) x[b] = AttnType<T>::mma(fk[kk], fq[b][kk], x[b]);
    };
    const auto finish = [&](f32x16 (&x)[QB], int j, auto lone) { // of the keys from j on
#pragma unroll
        for (int b = 0; b < QB; b++) scores(x[b], (float)(row0 + 32 * b + g.back - (j - g.kb)), h, lone);
    };
    // The maximum that the sums refer to moves only when it is left 8 behind (attn_lift): most steps skip the rescaling.
    const auto rescale = [&]() {
        bool far = false;
#pragma unroll
        for (int b = 0; b < QB; b++) far |= m[b] * c2 > top[b] + 8.f;
        if (!__any(far)) return;
#pragma unroll
        for (int b = 0; b < QB; b++) {
            const float now = fmaxf(m[b] * c2, top[b]);
            const float f = __builtin_amdgcn_exp2f(top[b] - (now == -INFINITY ? 0.f : now));
            top[b] = now;
            sum[b] *= f;
#pragma unroll
            for (int db = 0; db < DB; db++)
#pragma unroll
                for (int r = 0; r < 16; r++) o[b][db][r] *= f;
        }
    };
    Vec<T, 8> p[2][QB];
    const auto exponentials = [&](int half) {
#pragma unroll
        for (int b = 0; b < QB; b++) {
            const float ref = (top[b] == -INFINITY ? 0.f : top[b]) - attn_lift<T>();
            float eight = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[b][8 * half + e], c2, -ref));
                eight += x;
                p[half][b][e] = (T)x;
            }
            sum[b] += eight; // one by one, weights below 2^-25 of the sum would leave it as it is
        }
    };
    const auto weigh = [&](int half) {
#pragma unroll
        for (int db = 0; db < DB; db++)
#pragma unroll
            for (int b = 0; b < QB; b++) o[b][db] = AttnType<T>::mma(fv[half][db], p[half][b], o[b][db]);
    };

    if (g.hi > g.lo) {
        const int blocks = (g.hi - g.lo + 31) / 32;
        store(0);
        load(g.lo + BN);
        __syncthreads();
        read_keys(lds[0][0], 0);
        products(s);
        if (blocks > 1) {
            finish(s, g.lo, std::false_type{});
#pragma unroll
            for (int b = 0; b < QB; b++) m[b] = col_max(s[b]);
        } else
            finish(s, g.lo, std::true_type{});
        int stage = 0, i = 0;
        while (i + 1 < blocks) {
#pragma unroll
            for (int sub = 0; sub < SUB; sub++) {
                const int next = stage == 2 ? 0 : stage + 1;
                const bool last = sub == SUB - 1;
                if (last) { // the next step's keys are in the next tile
                    store(next);
                    load(g.lo + 32 * i + BN + 32);
                    __syncthreads();
                }
                // operands are asked for ahead of the products that take them: a lone wave waits for LDS otherwise
                read_keys(lds[last ? next : stage][0], last ? 0 : 32 * (sub + 1));
                read_values(lds[stage][1], 32 * sub, 0);
                read_values(lds[stage][1], 32 * sub, 1);
                rescale();
                f32x16 n[QB];
                products(n);
                exponentials(0);
                weigh(0);
                exponentials(1);
                weigh(1);
                finish(n, g.lo + 32 * (i + 1), std::false_type{});
#pragma unroll
                for (int b = 0; b < QB; b++) {
                    s[b] = n[b];
                    m[b] = col_max(s[b]);
                }
                i++;
                if (last) stage = next;
                if (i + 1 >= blocks) break;
            }
        }
        const int left = g.hi - g.lo - 32 * i; // the last 32 keys may be fewer
        read_values(lds[stage][1], 32 * (i % SUB), 0);
        read_values(lds[stage][1], 32 * (i % SUB), 1);
#pragma unroll
        for (int b = 0; b < QB; b++) {
            if (left < 32) mask_rows(s[b], left, h);
            m[b] = col_max(s[b]);
        }
        rescale();
        exponentials(0);
        weigh(0);
        exponentials(1);
        weigh(1);
    }
#pragma unroll
    for (int b = 0; b < QB; b++) fwd_store<T, DB>(a, g, head, split, row0 + 32 * b, top[b], pair_sum(sum[b]), o[b], lane);
}

// Few queries: NWQ of the four waves along the queries, 32 each, 4 / NWQ along the keys, whose shares are joined in LDS at the end: so that 32 queries
// still keep four waves busy.  With NWQ = 1 a tile may hold the a.pack query heads that share a key head, row r being query r / a.pack of head r % a.pack, so
// that keys are read once for all of them.  Bound by latency where there is little to read (23 rows in 32 bits 7.6 us: sequence numbers, rows, products, store),
// then by memory: 16 sequences of one query and 1152 keys, 12 heads of 64 in bf16 14.5 us (3.9 TB/s), 64 of them 40 (5.7).  (Two tiles under way instead of
// one: 5 % slower.)
template <class T, int DP, int NWQ> struct AttnFew {
    static constexpr int NWK = 4 / NWQ, BM = 32 * NWQ, BN = 32 * NWK;
    static constexpr int TILE = BN * DP; // elements of a tile
    static constexpr int JOIN = (NWK - 1) * NWQ * 64 * (DP / 2 + 2);      // floats
    static constexpr int LDS = 2 * TILE * (int)sizeof(T) > JOIN * 4 ? 2 * TILE * (int)sizeof(T) : JOIN * 4;
};
template <class T, int DP, int NWQ, int MODE> __global__ __launch_bounds__(ATTN_THREADS) void k_attn_few(AttnArgs a)
{
    typedef AttnFew<T, DP, NWQ> F;
    typedef AttnTile<T, DP> L;
    constexpr int NWK = F::NWK, BN = F::BN, KK = DP / 16, DB = DP / 32;
    __shared__ __attribute__((aligned(16))) char lds[F::LDS];
    T *const lk = (T *)lds, *const lv = lk + F::TILE;

    int first, slot, split; // first: key head of a packed tile, or query head
    if (!attn_work(a, a.slots * a.splits, first, slot, split)) return;
    const int pack = NWQ == 1 ? a.pack : 1;
    const TileRows t = tile_rows(a.sq, a.sk, slot, F::BM / pack);
    if (t.first >= t.top) return;
    const FwdRange g(a, t, split, BN);
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wq = wave % NWQ, wk = wave / NWQ;
    const int row = t.first + (32 * wq + (lane & 31)) / pack, head = first * pack + (lane & 31) % pack, kh = pack > 1 ? first : first / a.group;

    const T *const q = (const T *)a.q + head * a.q_head;
    const T *const k = (const T *)a.k + kh * a.k_head, *const v = (const T *)a.v + kh * a.v_head;
    typename L::Chunk ck[L::template per<BN, ATTN_THREADS>()], cv[L::template per<BN, ATTN_THREADS>()];
    const typename L::template Reads<BN, ATTN_THREADS> reads_k(a.k_row, a.dim, tid), reads_v(a.v_row, a.dim, tid);
    reads_k.load(ck, k, a.k_row, g.lo, g.hi, a.dim);
    reads_v.load(cv, v, a.v_row, g.lo, g.hi, a.dim);
    Vec<T, 8> fq[KK];
#pragma unroll
    for (int kk = 0; kk < KK; kk++) fq[kk] = L::own(q, a.q_row, row, row < t.top && row >= t.begin && row < t.end, kk, a.dim, lane);

    const Scores<T, MODE> scores(a, head);
    const float c2 = scores.rest();
    float top = -INFINITY, sum = 0.f;
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; db++) o[db] = f32x16{};

    for (int j0 = g.lo; j0 < g.hi; j0 += BN) {
        __syncthreads();
        L::template store<BN, ATTN_THREADS>(ck, lk, tid);
        L::template store<BN, ATTN_THREADS>(cv, lv, tid);
        __syncthreads();
        reads_k.load(ck, k, a.k_row, j0 + BN, g.hi, a.dim); // the next tile is under way meanwhile
        reads_v.load(cv, v, a.v_row, j0 + BN, g.hi, a.dim);
        const int j = j0 + 32 * wk; // the wave's keys of the tile
        if (j >= g.hi) continue;
        f32x16 s = {};
#pragma unroll
        for (int kk = 0; kk < KK; kk++) s = AttnType<T>::mma(L::rows(lk, 32 * wk, kk, lane), fq[kk], s);
        if (g.ke - g.kb <= 32)
            scores(s, (float)(row + g.back - (j - g.kb)), h, true);
        else
            scores(s, (float)(row + g.back - (j - g.kb)), h, false);
        if (g.hi - j < 32) mask_rows(s, g.hi - j, h);
        const float m = col_max(s) * c2;
        if (__any(m > top + 8.f)) { // as in k_attn
            const float now = fmaxf(m, top);
            const float f = __builtin_amdgcn_exp2f(top - (now == -INFINITY ? 0.f : now));
            top = now;
            sum *= f;
#pragma unroll
            for (int db = 0; db < DB; db++)
#pragma unroll
                for (int r = 0; r < 16; r++) o[db][r] *= f;
        }
        const float ref = (top == -INFINITY ? 0.f : top) - attn_lift<T>();
#pragma unroll
        for (int half = 0; half < 2; half++) {
            Vec<T, 8> p;
            float eight = 0.f; // as in k_attn
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[8 * half + e], c2, -ref));
                eight += x;
                p[e] = (T)x;
            }
            sum += eight;
#pragma unroll
            for (int db = 0; db < DB; db++) o[db] = AttnType<T>::mma(L::cols(lv, 32 * wk + 16 * half, db, lane), p, o[db]);
        }
    }
    sum = pair_sum(sum);

    // join the waves along the keys that had any: word i of all lanes side by side
    const int waves = min(NWK, (g.hi - g.lo + 31) >> 5);
    if (waves <= 1) {
        if (wk == 0) fwd_store<T, DB>(a, g, head, split, row, top, sum, o, lane);
        return;
    }
    float *const join = (float *)lds;
    __syncthreads();
    if (wk > 0) {
        float *p = join + ((wk - 1) * NWQ + wq) * 64 * (DP / 2 + 2) + lane;
        p[0] = top;
        p[64] = sum;
#pragma unroll
        for (int db = 0; db < DB; db++)
#pragma unroll
            for (int r = 0; r < 16; r++) p[(2 + db * 16 + r) * 64] = o[db][r];
    }
    __syncthreads();
    if (wk > 0) return;
    for (int w = 0; w < waves - 1; w++) {
        const float *p = join + (w * NWQ + wq) * 64 * (DP / 2 + 2) + lane;
        const float m = fmaxf(top, p[0]), ref = m == -INFINITY ? 0.f : m;
        const float f = __builtin_amdgcn_exp2f(top - ref), x = __builtin_amdgcn_exp2f(p[0] - ref);
        top = m;
        sum = sum * f + p[64] * x;
#pragma unroll
        for (int db = 0; db < DB; db++)
#pragma unroll
            for (int r = 0; r < 16; r++) o[db][r] = o[db][r] * f + p[(2 + db * 16 + r) * 64] * x;
    }
    fwd_store<T, DB>(a, g, head, split, row, top, sum, o, lane);
}

// Whether a row belongs to a sequence, sought by 64 lanes.
__device__ __forceinline__ bool row_in(const Spans &s, int row)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = s.count;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lo + lane * step;
        const unsigned long long m = __ballot(lane * step < n && span_begin(s, i) <= row);
        const int k = m ? 63 - __clzll(m) : 0;
        n = min(step, n - k * step);
        lo += k * step;
    }
    return row >= span_begin(s, lo) && row < span_end(s, lo);
}

// The splits of a row, 64 at most: weights w_s = exp(lse_s - max), o = sum w_s o_s / sum w_s.  A wave per row and head, blockIdx.x * 4 + wave over
// [heads][rows]; lane s has the weight of split s, and lane c the columns c and c + 64 of the sum, so that all reads of one kind are under way together (12 rows of
// 16 splits: 4 us; split after split 11).
#define ATTN_SPLITS 64
template <class T> __global__ __launch_bounds__(256) void k_attn_join(AttnArgs a)
{
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), all = (int64_t)a.heads * a.sq.rows;
    if (at >= all) return;
    const int lane = threadIdx.x & 63, head = at / a.sq.rows, row = at % a.sq.rows;
    const float l = lane < a.splits ? a.part_lse[lane * all + at] : -INFINITY;
    const bool in = row_in(a.sq, row); // the splits of other rows hold nothing
    if (!in && !a.fill) return;
    float o0 = 0.f, o1 = 0.f, lse = -INFINITY;
    if (in) {
        float top = l; // (a NaN among them comes back in the sum)
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, 64));
        const float w = l == -INFINITY ? 0.f : expf(l - top);
        const float sum = lanes_sum<64>(w);
        if (sum != 0.f) { // else no split had keys (NaN is not zero)
            const float *p = a.part_o + at * a.dim;
            const bool c0 = lane < a.dim, c1 = lane + 64 < a.dim;
            for (int s0 = 0; s0 < a.splits; s0 += 8) {
                float x0[8], x1[8];
#pragma unroll
                for (int s = 0; s < 8; s++) { // the last one again where there are fewer
                    const float *const ps = p + min(s0 + s, a.splits - 1) * all * a.dim;
                    x0[s] = c0 ? ps[lane] : 0.f;
                    x1[s] = c1 ? ps[lane + 64] : 0.f;
                }
#pragma unroll
                for (int s = 0; s < 8; s++) {
                    const float ws = __shfl(w, min(s0 + s, 63), 64);
                    if (s0 + s >= a.splits || ws == 0.f) continue; // a split without keys wrote nothing
                    o0 = fmaf(ws, x0[s], o0);
                    o1 = fmaf(ws, x1[s], o1);
                }
            }
            const float f = 1.f / sum;
            o0 *= f, o1 *= f;
            lse = top + logf(sum);
        }
    }
    if (lane == 0) a.lse[at] = lse;
    T *o = (T *)a.o + head * a.o_head + row * a.o_row;
    if (lane < a.dim) o[lane] = (T)o0;
    if (lane + 64 < a.dim) o[lane + 64] = (T)o1;
}

// ---- backward ---------------------------------------------------------------------------------------------------------
//
// NW waves of 32 rows each (queries for dq, keys for dk and dv); the other axis streams by in blocks of 32 rows through two LDS stages, one barrier a
// block.  delta is where the sums of do . v begin, lse is part of the exponential's fma: one subtraction less each.  A lone wave hides little, so
// registers are kept for more of them: three per SIMD for dq (two under a bias) and two for dk and dv, with heads up to 64.  (Row operands read a block ahead, at the
// price of a wave: dq of one sequence of 8192, 12 heads of 64, 484 us instead of 424.)  The next block goes to LDS ahead of the barrier at the block's
// beginning for dq, in its middle for dk and dv, whose barrier is there too (at the beginning: 578 us instead of 500).
// One sequence of 4096, 12 heads of 64 in bf16: dq 109 us (709 TF), dk and dv 124 (831); capped and biased 178 and 168 us: vector instructions.  64 sequences of
// 277 rows on average: 56 and 68 us.  Of the 16-bit kernels those for dq of short sequences with heads of 128, without a bias, keep 12 to 15 registers in scratch memory
// (of 64 one at most); of the 32-bit ones those for dk and dv with heads above 64.
template <class T, int DP, int MODE> struct AttnGrad {
    static constexpr int TILE = 32 * DP;
    static constexpr bool MEND = sizeof(T) == 2 && (MODE & MODE_SLOPE); // delta and dq are mended, as the comment at k_attn_grad_q says
    static constexpr int LESS = sizeof(T) == 2 && (MODE & MODE_EXACT) ? 1 : 0; // the library's tanh takes the registers of a wave, the sums that mend (MEND) too
    static constexpr int WAVES_Q = sizeof(T) == 4 ? 1 : (DP > 64 ? 2 : 3) - (LESS || MEND), WAVES_KV = sizeof(T) == 4 || DP > 64 ? 1 : 2 - LESS; // per SIMD
};
// What the backward pass makes of one score x, from the product x = q . k and `rest`, which has -lse in it: p, times 2^lift, and the factor of ds, 1 - tanh^2 under
// a cap.  Where tanh is 1 - 2 g, g = 1 / (1 + e^2y), 1 - tanh^2 is 4 g (1 - g): the 4 (BACK) comes with the scale.
template <class T, int MODE> struct GradScore {
    static constexpr bool FAST = attn_fast_tanh<T, MODE>();
    static constexpr float BACK = FAST ? 4.f : 1.f;
    float in, out, slope;
    __device__ __forceinline__ GradScore(const AttnArgs &a, int head)
    {
        const Scores<T, MODE> s(a, head);
        out = s.out;
        if (MODE & MODE_CAP) in = s.in;
        if (MODE & MODE_SLOPE) slope = s.slope;
    }
    __device__ __forceinline__ float p(float x, float rest, float dist, float &factor) const
    {
        if constexpr (MODE & MODE_SLOPE) rest = fmaf(-slope, fabsf(dist), rest);
        if constexpr (FAST) {
            const float g = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * in));
            factor = fmaf(-g, g, g);
            return __builtin_amdgcn_exp2f(fmaf(-2.f * out, g, rest)); // `rest` has the cap in it
        } else if constexpr (MODE & MODE_CAP) {
            const float th = tanhf(x * in);
            factor = fmaf(-th, th, 1.f);
            return __builtin_amdgcn_exp2f(fmaf(th, out, rest));
        }
        return __builtin_amdgcn_exp2f(fmaf(x, out, rest));
    }
    __device__ __forceinline__ float rest(float lse, float lift) const { return (FAST ? out + lift : lift) - lse * LOG2E; }
};

// fp16 has numbers from 2^-24 to 2^16, and eleven bits of them from 2^-14 on: p of long rows is below that, and ds, which no scaling of a loss keeps in place for
// every sequence and head, on either side.  So p is lifted by GRAD_LIFT (it is at most 1: eleven bits down to 2^-26), and ds by the power of two that brings
// its bound to 2^15: |ds_ij| = p |do . (v_j - o)| <= p (1 - p) |do| 2 max|v| <= |do| max|v| / 2, with max|v| over the sequence's keys (k_attn_grad_size).  A factor of
// two is left for the roundings of p, lse and delta.  dq has the own |do| of each query row in it, dk and dv, whose sums go over queries, the sequence's largest.
#define GRAD_LIFT 12
template <class T> constexpr bool grad_lifted() { return std::is_same<T, f16>::value; }
// the power of two for ds; fast: ds lacks a factor of 4
__device__ __forceinline__ int ds_lift(float go, float v, bool fast)
{
    const int e = __builtin_amdgcn_frexp_expf(0.5f * go * v); // bound <= 2^e; of 0, infinities and NaN 0
    return min(max((fast ? 17 : 15) - e, -60), 60);
}
// The largest of a sequence's sizes as k_attn_grad_size left them: of the slots that its rows begin .. end - 1 have tiles in.  The first 64 are asked for at once, for a
// caller that has other things to ask for before it needs them.
struct SeqSize {
    const float *size; // of the key head in slot 0
    int64_t slot, top; // the sequence's first slot, the last slot of all
    int kv_heads, next, last;
    float most;
    __device__ __forceinline__ SeqSize(const float *of, int seq, int begin, int end, int tile, int slots, int kv_heads, int kh) : size(of + kh), top(slots - 1), kv_heads(kv_heads), most(0.f)
    {
        const int c = seq ? begin : 0;
        slot = tile_slot(c, seq, tile);
        next = (begin - c) / tile + (threadIdx.x & 63), last = end > begin ? (end - 1 - c) / tile : -1;
        take();
    }
    __device__ __forceinline__ void take()
    {
        if (next <= last) most = fmaxf(most, size[min(slot + next, top) * kv_heads]);
        next += 64;
    }
    __device__ __forceinline__ float largest()
    {
        while (next <= last) take();
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor(most, s, 64));
        return most;
    }
};

// fp16: the largest norm of a row of v in each tile of keys, and of do in each tile of queries over the heads of a group.  A wave per slot and key head, the keys' slots
// first; the lanes of a row have 16 bytes each, and each lane eight rows under way.  No more than 2^22 work-groups, each of which takes its share.
// It takes 8.5 us for 3 sequences of 4000, 16 heads of 64 on 8 (the whole backward pass 789, 740 in bf16, which needs none of this), 7.9 for 32 of 300, 12 heads of 64 (86, 77), and
// 4.3 for one of 23, a launch and two trips (15, 9.5).
template <class T, int DP> __global__ __launch_bounds__(256) void k_attn_grad_size(AttnArgs a)
{
    constexpr int LANES = DP > 64 ? 16 : DP / 8, STEP = 64 / LANES; // lanes and rows at once
    const int kv_heads = a.heads / a.group, sub = (threadIdx.x & 63) / LANES, col = (threadIdx.x % LANES) * 8;
    const int64_t of_keys = (int64_t)a.slots_k * kv_heads, all = of_keys + (int64_t)a.slots_q * kv_heads;
    for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < all; w += (int64_t)gridDim.x * 4) {
        const bool keys = w < of_keys;
        const int64_t item = keys ? w : w - of_keys;
        const int slot = item / kv_heads, kh = item % kv_heads;
        const TileRows t = keys ? tile_rows(a.sk, a.sq, slot, a.tile_k) : tile_rows(a.sq, a.sk, slot, a.tile_q);
        const int lo = max(t.first, t.begin), hi = min(t.top, t.end);
        const int64_t row = keys ? a.v_row : a.go_row;
        float most = 0.f;
        for (int g = 0; g < (keys ? 1 : a.group); g++) {
            // lanes behind the row's end read its last vector and count nothing
            const T *const base = (keys ? (const T *)a.v + kh * a.v_head : (const T *)a.go + ((int64_t)kh * a.group + g) * a.go_head) + min(col, a.dim - 8);
            for (int r0 = lo; r0 < hi; r0 += 8 * STEP) {
                Vec<T, 8> x[8];
#pragma unroll
                for (int u = 0; u < 8; u++) x[u] = *(const Vec<T, 8> *)(base + min(r0 + u * STEP + sub, hi - 1) * row); // the last row again where there are fewer
#pragma unroll
                for (int u = 0; u < 8; u++) {
                    float sq = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; e++) sq = fmaf((float)x[u][e], (float)x[u][e], sq);
                    most = fmaxf(most, lanes_sum<LANES>(col < a.dim ? sq : 0.f));
                }
            }
        }
#pragma unroll
        for (int k = LANES; k < 64; k <<= 1) most = fmaxf(most, __shfl_xor(most, k, 64));
        if ((threadIdx.x & 63) == 0) (keys ? a.v_size : a.go_size)[item] = sqrtf(most);
    }
}

// dq: queries as columns.  Also leaves -delta for the kernel of dk and dv, which runs after it.
// MEND: what delta lacks, off = sum p (dp - delta), is known when all keys have passed.  So the weighted mean of the keys, sum p k (1 - tanh^2), is summed beside dq, which is
// then less by off times that; dk and dv get the right delta from the start.  That is one product in four, two or three vector instructions per score and a wave per SIMD:
// the whole backward pass of 3 sequences of 4000, 16 heads of 64 on 8, biased, 845 us in bf16 (772 without), of 4096 rows, 12 heads of 128, 594 (449).  Relative error of dq
// over 600 rows in bf16, values of mean 0, 1, 4 and 16 times their spread: 0.0024 each; without it (and so without a bias, where it would take 83 us instead of 75
// for 32 sequences of 300, 577 instead of 429 for heads of 128) 0.0024, 0.0044, 0.016 and 0.061.
template <class T, int DP, int NW, int MODE> __global__ __launch_bounds__(64 * NW, (AttnGrad<T, DP, MODE>::WAVES_Q)) void k_attn_grad_q(AttnArgs a)
{
    typedef AttnTile<T, DP> L;
    constexpr int NT = 64 * NW, KK = DP / 16, DB = DP / 32;
    __shared__ __attribute__((aligned(16))) T lds[2][2][AttnGrad<T, DP, MODE>::TILE];

    int head, slot, split;
    if (!attn_work(a, a.slots, head, slot, split)) return;
    const TileRows t = tile_rows(a.sq, a.sk, slot, 32 * NW);
    if (t.first >= t.top) return;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = t.first + 32 * wave + (lane & 31);
    const bool in = row < t.top && row >= t.begin && row < t.end;
    const int kb = t.other_begin, ke = t.first >= t.end || t.top <= t.begin ? kb : t.other_end;
    const int pos0 = row - t.end + (t.other_end - kb);

    const T *const q = (const T *)a.q + head * a.q_head, *const go = (const T *)a.go + head * a.go_head;
    const T *const oi = (const T *)a.o_in + head * a.oi_head;
    const T *const k = (const T *)a.k + (head / a.group) * a.k_head, *const v = (const T *)a.v + (head / a.group) * a.v_head;
    const typename L::template Reads<32, NT> reads_k(a.k_row, a.dim, tid), reads_v(a.v_row, a.dim, tid);
    typename L::Chunk ck[L::template per<32, NT>()], cv[L::template per<32, NT>()];
    const auto load = [&](int j) {
        reads_k.load(ck, k, a.k_row, j, ke, a.dim);
        reads_v.load(cv, v, a.v_row, j, ke, a.dim);
    };
    load(kb);
    SeqSize size(a.v_size, t.seq, kb, grad_lifted<T>() ? ke : kb, a.tile_k, a.slots_k, a.heads / a.group, head / a.group);
    Vec<T, 8> fq[KK], fg[KK];
    float delta = 0.f, sq = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; kk++) {
        fq[kk] = L::own(q, a.q_row, row, in, kk, a.dim, lane);
        fg[kk] = L::own(go, a.go_row, row, in, kk, a.dim, lane);
        const Vec<T, 8> x = L::own(oi, a.oi_row, row, in, kk, a.dim, lane);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            delta -= (float)x[e] * (float)fg[kk][e];
            if (grad_lifted<T>()) sq = fmaf((float)fg[kk][e], (float)fg[kk][e], sq);
        }
    }
    delta = pair_sum(delta);
    const int lift = grad_lifted<T>() ? ds_lift(sqrtf(pair_sum(sq)), size.largest(), GradScore<T, MODE>::FAST) : 0;
    const GradScore<T, MODE> score(a, head);
    const int64_t at = (int64_t)head * a.sq.rows + row;
    if (!AttnGrad<T, DP, MODE>::MEND && in && h == 0) a.delta[at] = delta;
    const float rest = in ? score.rest(a.lse[at], (float)lift) : -INFINITY; // rows of no sequence: p = 0
    constexpr bool MEND = AttnGrad<T, DP, MODE>::MEND;
    constexpr int W_LIFT = grad_lifted<T>() ? GRAD_LIFT : 0;
    const float w_rest = ldexpf(1.f, W_LIFT - lift); // what p lacks as a weight of the mean when it has ds's lift
    float off = 0.f; // times 2^lift
    f32x16 dq[DB], mean[MEND ? DB : 1];
#pragma unroll
    for (int db = 0; db < DB; db++) {
        dq[db] = f32x16{};
        if constexpr (MEND) mean[db] = f32x16{};
    }

    int stage = 0;
    const auto block = [&](int j, auto tail, auto lone) { // the 32 keys from j on; lone: the only ones
        L::template store<32, NT>(ck, lds[stage][0], tid);
        L::template store<32, NT>(cv, lds[stage][1], tid);
        __syncthreads();
        if (j + 32 < ke) load(j + 32);
        f32x16 s = {}, dp;
#pragma unroll
        for (int r = 0; r < 16; r++) dp[r] = delta;
#pragma unroll
        for (int kk = 0; kk < KK; kk++) {
            s = AttnType<T>::mma(L::rows(lds[stage][0], 0, kk, lane), fq[kk], s);
            dp = AttnType<T>::mma(L::rows(lds[stage][1], 0, kk, lane), fg[kk], dp);
        }
        const float pos = (float)(pos0 - (j - kb) - 4 * h);
        Vec<T, 8> d[2], w[2];
        float ps[lone ? 16 : 1], fs[lone ? 16 : 1], by = 0.f;
#pragma unroll
        for (int r = 0; r < 16; r++) {
            const int m = 8 * (r >> 2) + (r & 3);
            float f = 1.f, p = score.p(s[r], rest, pos - (float)m, f);
            if (tail && m + 4 * h >= ke - j) p = 0.f; // a missing key's score may be anything
            if constexpr (lone) {
                ps[r] = p, fs[r] = f;
                by += p * dp[r];
                continue;
            }
            if constexpr (MEND) {
                by = fmaf(p, dp[r], by);
                if (MODE & MODE_CAP) p *= f;
                w[r >> 3][r & 7] = (T)(grad_lifted<T>() ? p * w_rest : p); // (its rounding is one of the correction alone)
                d[r >> 3][r & 7] = (T)(p * dp[r]);
                continue;
            }
            p *= dp[r];
            if (MODE & MODE_CAP) p *= f;
            d[r >> 3][r & 7] = (T)p; // the scale is put on at the end
        }
        if constexpr (MEND) off += by;
        if constexpr (lone) {
            // All weights of the row are at hand: sum p (dp - delta) is what delta lacks for o as it was before its rounding.
            by = ldexpf(pair_sum(by), -lift);
            delta -= by;
#pragma unroll
            for (int r = 0; r < 16; r++) d[r >> 3][r & 7] = (T)(ps[r] * (dp[r] - by) * fs[r]);
        }
#pragma unroll
        for (int half = 0; half < 2; half++)
#pragma unroll
            for (int db = 0; db < DB; db++) {
                const Vec<T, 8> x = L::cols(lds[stage][0], 16 * half, db, lane);
                dq[db] = AttnType<T>::mma(x, d[half], dq[db]);
                if constexpr (MEND) mean[db] = AttnType<T>::mma(x, w[half], mean[db]);
            }
        stage ^= 1;
    };
    int j = kb;
    if constexpr (NW == 2 && !MEND) // tiles of short sequences (its registers would cost the other tile 5 %)
        if (ke - kb <= 32 && ke > kb) {
            block(j, std::true_type{}, std::true_type{});
            if (in && h == 0) a.delta[at] = delta;
            j = ke;
        }
    for (; j + 32 <= ke; j += 32) block(j, std::false_type{}, std::false_type{});
    if (j < ke) block(j, std::true_type{}, std::false_type{});
    if constexpr (MEND) {
        off = pair_sum(off);
        delta -= ldexpf(off, -lift);
        if (in && h == 0) a.delta[at] = delta;
        off = ldexpf(off, -W_LIFT); // off has 2^lift, as dq has, and the mean 2^W_LIFT
#pragma unroll
        for (int db = 0; db < DB; db++)
#pragma unroll
            for (int r = 0; r < 16; r++) dq[db][r] = fmaf(-off, mean[db][r], dq[db][r]);
    }
    if (row >= t.top || (!in && !a.fill)) return;
    if (!in || ke == kb)
#pragma unroll
        for (int db = 0; db < DB; db++) dq[db] = f32x16{};
    store_row<T, DB>(dq, ldexpf(a.scale * GradScore<T, MODE>::BACK, -lift), (T *)a.dq + head * a.dq_head + row * a.dq_row, a.dim, lane);
}

// dk, dv: keys as columns, the queries of all heads that share the key head stream by, one head after the other.  Where that leaves too few work-groups
// their blocks are cut into a.splits parts, whose sums k_attn_grad_join adds up.
template <class T, int DP, int NW, int MODE> __global__ __launch_bounds__(64 * NW, (AttnGrad<T, DP, MODE>::WAVES_KV)) void k_attn_grad_kv(AttnArgs a)
{
    typedef AttnTile<T, DP> L;
    constexpr int NT = 64 * NW, KK = DP / 16, DB = DP / 32, P_LIFT = grad_lifted<T>() ? GRAD_LIFT : 0;
    __shared__ __attribute__((aligned(16))) T lds[2][2][AttnGrad<T, DP, MODE>::TILE];
    __shared__ __attribute__((aligned(16))) float stat[2][2][32]; // what is added to scores, -delta

    int kh, slot, split;
    if (!attn_work(a, a.slots * a.splits, kh, slot, split)) return;
    const TileRows t = tile_rows(a.sk, a.sq, slot, 32 * NW);
    if (t.first >= t.top) return;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = t.first + 32 * wave + (lane & 31);
    const bool in = row < t.top && row >= t.begin && row < t.end;
    const int qb = t.other_begin, qe = t.first >= t.end || t.top <= t.begin ? qb : t.other_end;
    const int pos0 = row - t.end + (t.other_end - qb); // the row's position among the queries, the first at 0

    const T *const k = (const T *)a.k + kh * a.k_head, *const v = (const T *)a.v + kh * a.v_head;
    const typename L::template Reads<32, NT> reads_q(a.q_row, a.dim, tid), reads_g(a.go_row, a.dim, tid);
    typename L::Chunk cq[L::template per<32, NT>()], cg[L::template per<32, NT>()];
    float cs = 0.f; // lse of 32 queries and -delta of 32, the first 64 threads
    const auto load = [&](int head, int i) {
        reads_q.load(cq, (const T *)a.q + head * a.q_head, a.q_row, i, qe, a.dim);
        reads_g.load(cg, (const T *)a.go + head * a.go_head, a.go_row, i, qe, a.dim);
        if (tid < 64) cs = (h ? a.delta : a.lse)[(int64_t)head * a.sq.rows + min(i + (lane & 31), qe - 1)];
    };
    const auto store = [&](int stage, int head, int i) {
        L::template store<32, NT>(cq, lds[stage][0], tid);
        L::template store<32, NT>(cg, lds[stage][1], tid);
        if (tid < 64) stat[stage][h][lane & 31] = h ? cs : i + lane < qe ? GradScore<T, MODE>(a, head).rest(cs, P_LIFT) : -INFINITY; // a missing query: p = 0
    };
    const bool sized = grad_lifted<T>() && qe > qb;
    SeqSize size_go(a.go_size, t.seq, qb, sized ? qe : qb, a.tile_q, a.slots_q, a.heads / a.group, kh);
    SeqSize size_v(a.v_size, t.seq, t.begin, sized ? t.end : t.begin, a.tile_k, a.slots_k, a.heads / a.group, kh);
    Vec<T, 8> fk[KK], fv[KK];
#pragma unroll
    for (int kk = 0; kk < KK; kk++) {
        fk[kk] = L::own(k, a.k_row, row, in, kk, a.dim, lane);
        fv[kk] = L::own(v, a.v_row, row, in, kk, a.dim, lane);
    }
    const int lift = sized ? ds_lift(size_go.largest(), size_v.largest(), GradScore<T, MODE>::FAST) : 0;
    const float ds_rest = ldexpf(1.f, lift - P_LIFT); // what ds lacks when p has its lift
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int db = 0; db < DB; db++) dk[db] = dv[db] = f32x16{};

    // blocks of queries, one head after the other
    const int per = (qe - qb + 31) >> 5, share = (per * a.group + a.splits - 1) / a.splits;
    const int first = min(split * share, per * a.group), blocks = min(share, per * a.group - first);
    int head = kh * a.group, i = qb; // of the block at hand
    if (blocks > 0) head += first / per, i += first % per * 32;
    int head1 = head, i1 = i, left1 = blocks; // of the block in registers or under way, and how many there are from it on
    const auto advance = [&]() {
        left1--;
        i1 += 32;
        if (i1 >= qe) i1 = qb, head1++;
        if (left1 > 0) load(head1, i1);
    };
    if (blocks > 0) {
        load(head1, i1);
        store(0, head1, i1);
        advance();
        __syncthreads();
    }
    int stage = 0;
    for (int u = 0; u < blocks;) {
        const GradScore<T, MODE> score(a, head);
        for (; u < blocks && i < qe; u++, i += 32, stage ^= 1) {
            const T *const lq = lds[stage][0], *const lg = lds[stage][1];
            f32x16 s = {}, dp;
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x4 d = *(const f32x4 *)&stat[stage][1][2 * r + 4 * h];
#pragma unroll
                for (int e = 0; e < 4; e++) dp[r + e] = d[e];
            }
#pragma unroll
            for (int kk = 0; kk < KK; kk++) {
                s = AttnType<T>::mma(L::rows(lq, 0, kk, lane), fk[kk], s);
                dp = AttnType<T>::mma(L::rows(lg, 0, kk, lane), fv[kk], dp);
            }
            Vec<T, 8> tq[2][DB], tg[2][DB];
#pragma unroll
            for (int half = 0; half < 2; half++)
#pragma unroll
                for (int db = 0; db < DB; db++) {
                    tq[half][db] = L::cols(lq, 16 * half, db, lane);
                    tg[half][db] = L::cols(lg, 16 * half, db, lane);
                }
            f32x4 rest[4];
#pragma unroll
            for (int r4 = 0; r4 < 4; r4++) rest[r4] = *(const f32x4 *)&stat[stage][0][8 * r4 + 4 * h];
            if (left1 > 0) {
                store(stage ^ 1, head1, i1);
                advance();
            }
            const float pos = (float)(pos0 - (i - qb) - 4 * h);
            Vec<T, 8> p[2], d[2];
#pragma unroll
            for (int r = 0; r < 16; r++) {
                float f = 1.f;
                const float w = score.p(s[r], rest[r >> 2][r & 3], pos - (float)(8 * (r >> 2) + (r & 3)), f);
                float x = w * dp[r];
                if (MODE & MODE_CAP) x *= f;
                if (grad_lifted<T>()) x *= ds_rest;
                p[r >> 3][r & 7] = (T)w;
                d[r >> 3][r & 7] = (T)x;
            }
            __syncthreads();
#pragma unroll
            for (int half = 0; half < 2; half++)
#pragma unroll
                for (int db = 0; db < DB; db++) {
                    dv[db] = AttnType<T>::mma(tg[half][db], p[half], dv[db]);
                    dk[db] = AttnType<T>::mma(tq[half][db], d[half], dk[db]);
                }
        }
        head++;
        i = qb;
    }
    if (row >= t.top) return;
    if (!in || blocks <= 0)
#pragma unroll
        for (int db = 0; db < DB; db++) dk[db] = dv[db] = f32x16{};
    const float back_k = ldexpf(a.scale * GradScore<T, MODE>::BACK, -lift), back_v = ldexpf(1.f, -P_LIFT);
    if (a.splits > 1) {
        float *part = a.part_o + (((int64_t)split * 2 * (a.heads / a.group) + kh) * a.sk.rows + row) * a.dim;
        store_row<float, DB>(dk, back_k, part, a.dim, lane);
        store_row<float, DB>(dv, back_v, part + (int64_t)(a.heads / a.group) * a.sk.rows * a.dim, a.dim, lane);
        return;
    }
    if (!in && !a.fill) return;
    store_row<T, DB>(dk, back_k, (T *)a.dk + kh * a.dk_head + row * a.dk_row, a.dim, lane);
    store_row<T, DB>(dv, back_v, (T *)a.dv + kh * a.dv_head + row * a.dv_row, a.dim, lane);
}

// dk and dv from the parts: a wave per row and key head, blockIdx.x * 4 + wave over [kv_heads][rows].
template <class T> __global__ __launch_bounds__(256) void k_attn_grad_join(AttnArgs a)
{
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), all = (int64_t)(a.heads / a.group) * a.sk.rows;
    if (at >= all) return;
    const int lane = threadIdx.x & 63, kh = at / a.sk.rows, row = at % a.sk.rows;
    if (!a.fill && !row_in(a.sk, row)) return;
    T *const dk = (T *)a.dk + kh * a.dk_head + row * a.dk_row, *const dv = (T *)a.dv + kh * a.dv_head + row * a.dv_row;
    for (int c = lane; c < a.dim; c += 64) {
        float k = 0.f, v = 0.f;
        for (int s = 0; s < a.splits; s++) {
            k += a.part_o[(2 * s * all + at) * a.dim + c];
            v += a.part_o[((2 * s + 1) * all + at) * a.dim + c];
        }
        dk[c] = (T)k, dv[c] = (T)v;
    }
}
