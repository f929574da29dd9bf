// What the kernels on token states share: element types, vectors of them, sums over lanes, the sequence of a tile of rows.
//
// Sequences are rows [begin[i], end[i]) of one token axis, in ascending order and apart from one another.  The numbers are device
// data that the host never sees, so every kernel clamps them to the buffer: numbers that break the rule give results
// without meaning, never an access outside the buffers.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

typedef _Float16 f16;
typedef __bf16 bf16;

template <class T, int N> struct VecOf {
    typedef T type __attribute__((ext_vector_type(N)));
};
template <class T, int N> using Vec = typename VecOf<T, N>::type;
typedef Vec<float, 4> f32x4;
typedef Vec<float, 16> f32x16;

// The elements col .. col + VEC - 1 of a row of `width` elements, zeros behind its end.  Rows may begin anywhere: global memory takes 16-byte accesses at every
// address, so rows of any width and stride go by whole vectors, and only a vector across a row's end by elements.
template <class T, int VEC> struct UnalignedVec {
    typedef T type __attribute__((ext_vector_type(VEC), aligned(sizeof(T))));
};
template <class T, int VEC> __device__ __forceinline__ Vec<T, VEC> load_vec(const T *row, int col, int width)
{
    Vec<T, VEC> x = {};
    if (col + VEC <= width)
        x = *(const typename UnalignedVec<T, VEC>::type *)(row + col);
    else
#pragma unroll
        for (int e = 0; e < VEC; e++)
            if (col + e < width) x[e] = row[col + e];
    return x;
}
template <class T, int VEC> __device__ __forceinline__ void store_vec(Vec<T, VEC> x, T *row, int col, int width)
{
    if (col + VEC <= width)
        *(typename UnalignedVec<T, VEC>::type *)(row + col) = x;
    else
#pragma unroll
        for (int e = 0; e < VEC; e++)
            if (col + e < width) row[col + e] = x[e];
}

// A whole vector, whose lines are not kept: rows that one kernel reads once and no other soon.
template <class T, int VEC> __device__ __forceinline__ Vec<T, VEC> load_once(const T *p)
{
    return __builtin_nontemporal_load((const typename UnalignedVec<T, VEC>::type *)p);
}

// Sum over the LANES lanes of an aligned group, the same in each of them.
template <int LANES> __device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int s = LANES / 2; s > 0; s >>= 1) v += __shfl_xor(v, s, 64);
    return v;
}

struct Spans {
    const int32_t *begin, *end;
    int32_t count; // sequences
    int32_t rows;  // of the token axis
};
__device__ __forceinline__ int span_begin(const Spans &s, int i) { return min(max(s.begin[i], 0), s.rows); }
__device__ __forceinline__ int span_end(const Spans &s, int i) { return min(max(s.end[i], 0), s.rows); }

// Tiles of `tile` rows never span two sequences: a neighbour's infinities and NaN stay away from a product with zero weights.
// Sequence i is given the rows from its begin up to the next one's begin (the first one from row 0, the last one to the last row: so
// the rows between and behind sequences have a tile too), cover_i = [c_i, c_{i+1}), and the slots f_i .. f_{i+1} - 1 with f_0 = 0 and
// f_i = ceil(c_i / tile) + i - 1, which are at least ceil((c_{i+1} - c_i) / tile): no sums over the lengths are needed, and ceil(rows / tile) + count - 1
// slots hold them all (one sequence: exactly its tiles).  A slot behind the last row of its sequence's cover is empty.
struct TileRows {
    int seq;        // the sequence
    int first, top; // the tile's rows, [first, top); empty: first >= top
    int begin, end; // of the sequence: rows of the tile outside belong to none
    int other_begin, other_end; // its rows in the other token axis
};
__device__ __forceinline__ int tile_slot(int c, int i, int tile) { return i ? (c ? (c - 1) / tile + 1 : 0) + i - 1 : 0; }
// The sequence is the last i with f_i <= slot, sought by 64 lanes at a time; the last 64 candidates bring all their numbers along, so that up to 64 sequences
// take one trip to memory and up to 4096 two.
__device__ __forceinline__ TileRows tile_rows(const Spans &s, const Spans &other, int slot, int tile)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = s.count; // i is in [lo, lo + n)
    while (n > 64) {
        const int step = (n + 63) >> 6, i = lo + lane * step;
        const bool ok = lane * step < n && (i == 0 || tile_slot(span_begin(s, i), i, tile) <= slot);
        const unsigned long long m = __ballot(ok);
        const int k = m ? 63 - __clzll(m) : 0;
        n = min(step, n - k * step);
        lo += k * step;
    }
    const int i = lo + min(lane, n - 1), next = min(i + 1, s.count - 1);
    const int begin = span_begin(s, i), end = span_end(s, i), after = span_begin(s, next), ob = span_begin(other, i), oe = span_end(other, i);
    const unsigned long long m = __ballot(lane < n && (i == 0 || tile_slot(begin, i, tile) <= slot));
    const int k = m ? 63 - __clzll(m) : 0;
    TileRows t;
    t.seq = __builtin_amdgcn_readfirstlane(lo + k);
    t.begin = __builtin_amdgcn_readlane(begin, k);
    t.end = __builtin_amdgcn_readlane(end, k);
    t.other_begin = __builtin_amdgcn_readlane(ob, k);
    t.other_end = max(__builtin_amdgcn_readlane(oe, k), t.other_begin);
    const int c = t.seq ? t.begin : 0;
    const int top = t.seq + 1 < s.count ? __builtin_amdgcn_readlane(after, k) : s.rows;
    const long long first = c + (long long)(slot - tile_slot(c, t.seq, tile)) * tile;
    t.first = first < c ? top : (int)(first < top ? first : top);
    t.top = top - t.first < tile ? top : t.first + tile;
    return t;
}
static inline int64_t tile_slots(int64_t rows, int64_t count, int tile) { return (rows + tile - 1) / tile + count - 1; } // count >= 1
