// Launchers of the kernels on token states, one table per element type (and head size): each is instantiated in a translation unit of its own, so that
// the library builds in parallel.
#pragma once
#include "launch.h"

struct AttnArgs;
struct NormArgs;
struct NormGradArgs;
struct PoolArgs;
struct PoolGradArgs;

struct AttnLaunch {
    // tile: queries of a work-group, 32, 64, 128 or 256
    void (*fwd)(he_ctx *c, hipStream_t st, double bytes, int tile, unsigned grid, const AttnArgs &a);
    void (*join)(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a);
    void (*grad_q)(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a);
    void (*grad_kv)(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a);
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
