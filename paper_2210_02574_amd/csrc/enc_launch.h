// Launchers of the kernels on token states, one table per element type (and head size): each is instantiated in a translation unit of its own, so that
// the library builds in parallel.
#pragma once
#include "launch.h"

struct AttnArgs;
struct NormArgs;
struct NormGradArgs;
struct PoolArgs;
struct PoolGradArgs;

// Whether there are tiles of 256 queries, two blocks of 32 to a wave: they halve what is read of LDS for a product, and pay where the registers still
// hold two waves per SIMD.  12 heads of 64 in bf16, tiles of 256 against 128: one sequence of 16384 1013 us, 1086; 16 of 2048 300, 312; 32 of 1024 146, 150;
// 42 of 768 130, 112.  Heads of 128 (one wave per SIMD): 16384 1771 us, 1822; 4096 1095, 1059; 1024 378, 326.
constexpr bool attn_wide(size_t type_size, int dim) { return type_size == 2 && dim <= 64; }

struct AttnLaunch {
    // tile: queries of a work-group, 32, 64, 128 or 256
    void (*fwd)(he_ctx *c, hipStream_t st, double bytes, int tile, unsigned grid, const AttnArgs &a);
    void (*join)(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a);
    void (*grad_size)(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a); // fp16, else null
    // tile: rows of a work-group, 64 or 128 queries, 32, 64 or 128 keys
    void (*grad_q)(he_ctx *c, hipStream_t st, double bytes, int tile, unsigned grid, const AttnArgs &a);
    void (*grad_kv)(he_ctx *c, hipStream_t st, double bytes, int tile, unsigned grid, const AttnArgs &a);
    void (*grad_join)(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a);
};
#define HE_DECL_ATTN(t)                                                                                              \
    void attn_launch_##t##_32(AttnLaunch &t_);                                                                       \
    void attn_launch_##t##_64(AttnLaunch &t_);                                                                       \
    void attn_launch_##t##_96(AttnLaunch &t_);                                                                       \
    void attn_launch_##t##_128(AttnLaunch &t_);
HE_DECL_ATTN(0)
HE_DECL_ATTN(1)
HE_DECL_ATTN(2)
#undef HE_DECL_ATTN

struct RowsLaunch {
    // wide_w: weights in 32 bits whatever the rows' type
    void (*norm)(he_ctx *c, hipStream_t st, double bytes, bool wide_w, const NormArgs &a);
    void (*norm_grad)(he_ctx *c, hipStream_t st, double bytes, bool wide_w, int parts, const NormGradArgs &a);
    void (*weight_grad)(he_ctx *c, hipStream_t st, double bytes, bool wide_w, const float *part, int parts, int width, void *dw, void *db);
    void (*pool)(he_ctx *c, hipStream_t st, double bytes, unsigned slots, const PoolArgs &a);
    void (*pool_grad)(he_ctx *c, hipStream_t st, double bytes, unsigned slots, const PoolGradArgs &a);
};
void rows_launch_0(RowsLaunch &t);
void rows_launch_1(RowsLaunch &t);
void rows_launch_2(RowsLaunch &t);

#define NORM_MAX_WIDTH 16384
