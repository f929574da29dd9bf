// Entry points of the operators on token states: attention inside sequences, layer norm, mean over sequences.
#include <cmath>
#include <cstring>

#include "enc_launch.h"
#include "kernels_attn.h"
#include "kernels_norm.h"
#include "kernels_pool.h"

namespace {

// The context's device is the current one while kernels are launched, and the caller's is afterwards.
struct DeviceGuard {
    int before = -1, rc = HE_OK;
    explicit DeviceGuard(he_ctx *c)
    {
        hipError_t e = hipGetDevice(&before);
        if (e == hipSuccess && before != c->device) e = hipSetDevice(c->device);
        else before = -1;
        if (e != hipSuccess) {
            c->hip_err = std::string("hipSetDevice: ") + hipGetErrorString(e);
            rc = HE_EHIP;
        }
    }
    ~DeviceGuard()
    {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

// The arguments are checked ahead of the device, so that a context without one refuses the same ones.
#define NEEDS_DEVICE(c)                                                                                              \
    if ((c)->device < 0) return HE_ENODEV

int32_t launched(he_ctx *c)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return HE_OK;
    c->hip_err = std::string("kernel launch: ") + hipGetErrorString(e);
    return HE_EHIP;
}

constexpr int64_t MAX_ROWS = ((int64_t)1 << 31) - 65536; // row numbers and a tile more fit 32 bits

bool type_ok(int32_t t) { return t == HE_F32 || t == HE_F16 || t == HE_BF16; }
size_t type_size(int32_t t) { return t == HE_F32 ? 4 : 2; }
bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

const RowsLaunch &rows_launch(int32_t t)
{
    static const RowsLaunch tables[3] = {
        [] { RowsLaunch x{}; rows_launch_0(x); return x; }(),
        [] { RowsLaunch x{}; rows_launch_1(x); return x; }(),
        [] { RowsLaunch x{}; rows_launch_2(x); return x; }(),
    };
    return tables[t];
}
const AttnLaunch &attn_launch(int32_t t, int dim)
{
#define ROW(t)                                                                                                        \
    {                                                                                                                \
        [] { AttnLaunch x{}; attn_launch_##t##_32(x); return x; }(), [] { AttnLaunch x{}; attn_launch_##t##_64(x); return x; }(),            \
            [] { AttnLaunch x{}; attn_launch_##t##_96(x); return x; }(), [] { AttnLaunch x{}; attn_launch_##t##_128(x); return x; }(),     \
    }
    static const AttnLaunch tables[3][4] = {ROW(0), ROW(1), ROW(2)};
#undef ROW
    return tables[t][(dim - 1) / 32];
}

// ---- layer norm ------------------------------------------------------------------------------------------------------

int32_t norm_check(const he_norm *n)
{
    if (!n || !type_ok(n->type) || (n->weight_type != n->type && n->weight_type != HE_F32)) return HE_EINVAL;
    if (n->rows < 0 || n->rows > MAX_ROWS || n->width < 1 || n->width > NORM_MAX_WIDTH) return HE_EINVAL;
    return HE_OK;
}
bool rows_ok(const he_rows *r, int64_t width, int32_t type) { return r && r->d && aligned(r->d, type_size(type)) && r->stride >= width; }
bool words_ok(const void *p, size_t size = 4) { return p && aligned(p, size); }

// Work-groups of the backward pass: each writes a partial row of dw and db, so two for each of the 256 CUs and no more than rows need.
int norm_parts(int64_t rows) { return (int)std::max<int64_t>(1, std::min<int64_t>(512, (rows + 3) / 4)); }

// ---- mean ----------------------------------------------------------------------------------------------------------------

int32_t spans_check(const he_spans *s)
{
    if (!s || s->count < 0 || s->rows < 0 || s->rows > MAX_ROWS || s->count > (1 << 23)) return HE_EINVAL;
    if (s->count > 0 && (!words_ok(s->d_begin) || !words_ok(s->d_end))) return HE_EINVAL;
    return HE_OK;
}
Spans spans_of(const he_spans *s) { return Spans{s->d_begin, s->d_end, s->count, (int32_t)s->rows}; }

// A work-group per sequence while they and their rows are few; else tiles of equal length, about 2048 of them, whatever the lengths are, and a second launch that joins
// them.
int pool_tile(const he_spans *s)
{
    if (s->count == 0 || (s->rows <= 8192 && s->count <= 8192 && s->rows / s->count <= 256)) return 0;
    return (int)std::max<int64_t>(64, (s->rows / 2048 + 15) / 16 * 16);
}
// 32 rows, more from 2^27 rows on: a launch holds 2^24 work-groups, of which sequences, 2^23 at most, may take one each.
int pool_grad_tile(const he_spans *s) { return (int)std::max<int64_t>(32, (s->rows >> 22) + 1); }
size_t pool_bytes(const he_spans *s, int32_t width)
{
    const int tile = pool_tile(s);
    return tile ? (size_t)tile_slots(s->rows, s->count, tile) * width * sizeof(float) : 0;
}

// ---- attention -------------------------------------------------------------------------------------------------------------

int32_t attn_check(const he_attn *s)
{
    if (!s || !type_ok(s->type) || s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads || s->heads > 65535) return HE_EINVAL;
    if (s->dim < 8 || s->dim > 128 || s->dim % 8) return HE_EINVAL;
    if (spans_check(&s->q) != HE_OK || spans_check(&s->k) != HE_OK || s->q.count != s->k.count) return HE_EINVAL;
    constexpr double most = 0x1p127; // times log2(e) still finite in 32 bits
    if (!(s->scale > 0.0) || !(s->scale <= most) || !((float)s->scale > 0.f)) return HE_EINVAL;
    if (!(s->cap >= 0.0) || !(s->cap <= most) || (s->cap > 0.0 && !((float)s->cap > 0.f))) return HE_EINVAL;
    if (s->cap > 0.0 && !std::isfinite((float)s->scale / (float)s->cap * 3.f)) return HE_EINVAL; // what scores are multiplied with under tanh
    if (s->d_slopes && !aligned(s->d_slopes, 4)) return HE_EINVAL;
    return HE_OK;
}
bool heads_ok(const he_heads *h, int32_t type)
{
    const int64_t size = (int64_t)type_size(type);
    if (!h || !h->d || !aligned(h->d, 16) || h->row < 0 || h->row >= (1 << 24) / size || h->head < 0 || h->head >= (int64_t)1 << 46) return false;
    return (h->row * size) % 16 == 0 && (h->head * size) % 16 == 0;
}
// Buffers that are written: elements of different rows and heads have different addresses.
bool out_ok(const he_heads *h, const he_attn *s, int64_t rows, int heads)
{
    if (!heads_ok(h, s->type) || (rows > 1 && h->row < s->dim) || (heads > 1 && h->head < s->dim)) return false;
    return rows <= 1 || heads <= 1 || h->row >= (heads - 1) * h->head + s->dim || h->head >= (rows - 1) * h->row + s->dim;
}

struct AttnPlan {
    int tile, splits; // rows of a work-group; parts that the keys are cut into
    int pack;         // query heads to a tile
    int64_t slots;    // tiles
    int64_t groups;   // work-groups
};
// Rules go by the sequences' mean length, the only one that the host knows.  A long sequence among many short ones is given what suits those: one of 8192 rows and 255 of 32
// take 328 us forward and 1060 backward in bf16, 12 heads of 64; in calls of their own 251 and 752, and 19 and 46.
// Tiles: 128 queries, 64 for short sequences, 256 where attn_wide() says so, no cap keeps the vector instructions busy
// anyway (one sequence of 8192, 12 heads of 64, capped: 496 us, with 128 426) and three rounds of them fill the card.  Tiles of 32, whose four waves
// share the keys, where tiles of 128 would leave half of the CUs without one, or few queries meet many keys.  12 heads of 64 in bf16, tiles of 32,
// 64, 128: 64 tokens 5.4, 6.0, 5.4 us; 512 tokens 8.2, 8.8, 10; 1024 16, 17, 15; 4 x 512 14, 13, 13; 64 x 64 13, 9.2, 9.5; 256 x 24 24, 18, 21.
// Query heads that share a key head go into one tile where their queries fit it: 64 sequences of one query and 1152 keys, 12 heads of 64 on 4, 17 us in bf16 (38
// apart) and 51 in 32 bits (95); 16 of them, heads of 128, 32 on 4, 19 and 43 us (28, 124); 10 queries, 1000 keys, 12 heads on 4, 12 and 30 us (16, 46).
// The keys are cut where even so there are few work-groups: the second launch costs 4 us (16 sequences of one query and 1152 keys, 12 heads of 64, cut in
// two: 20 us instead of 14.5).
AttnPlan attn_plan(const he_attn *s)
{
    AttnPlan p{128, 1, 1, 0, 0};
    if (s->q.count == 0) return p;
    const int64_t mean_q = s->q.rows / s->q.count, mean_k = s->k.rows / s->q.count;
    const auto groups = [&](int tile) { return tile_slots(s->q.rows, s->q.count, tile) * s->heads; };
    if (mean_q <= 64) p.tile = 64;
    if (groups(p.tile) < 128 || (mean_q <= 32 && mean_k > 128)) p.tile = 32;
    if (mean_q >= 1024 && s->cap == 0.0 && attn_wide(type_size(s->type), s->dim) && groups(256) >= 768) p.tile = 256;
    const int group = s->heads / s->kv_heads;
    if (group > 1 && mean_q * group <= 32 && group <= 32) p.tile = 32, p.pack = group;
    p.slots = tile_slots(s->q.rows, s->q.count, p.tile / p.pack);
    p.groups = p.slots * (s->heads / p.pack);
    if (p.tile == 32 && p.slots > 0) p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({256 / p.groups, mean_k / 512, ATTN_SPLITS}));
    p.groups *= p.splits;
    return p;
}

// Rows of a work-group of the backward pass.  Short sequences leave a part of a tile empty and a work-group little to do between its first loads and its last
// stores: small ones then waste less and more of them are resident.  12 heads of 64 in bf16, dq with 64 rows against 128: 1000 sequences of 17 rows on average
// 49 us, 79; 128 of 138 45, 48; 64 of 288 59, 58; 32 of 577 92, 89; 4 of 2525 192, 170.  dk and dv with 32, 64, 128: 44 us, 60, 102; 52, 52, 62; 75, 72, 79; 124,
// 116, 119; 250, 232, 220.
int grad_tile_q(const he_spans &s) { return s.rows / s.count < 256 ? 64 : 128; }
int grad_tile_k(const he_spans &s) { return s.rows / s.count < 192 ? 32 : s.rows / s.count < 640 ? 64 : 128; }
// Parts that the queries of a tile of keys are cut into, each a work-group of its own, until there are 2560 waves (two and a half for each SIMD): shared key heads have
// long work and few tiles.  Joining costs 4 to 14 us, so parts keep 512 query rows, or 128 where there is not even a wave for half of the SIMDs.  One sequence of
// 8192, heads of 64 in bf16, 12 on 4: 636 us whole, 472 in two or three; one of 4096 with heads of their own 148, 150; one of 336, 12 on 4, 27 whole, 13 in seven; one of 167,
// 12 on 2, 32, 12; two of 576, heads of 96 of their own, 28, 30.
int grad_splits(const he_attn *s)
{
    if (s->k.count == 0 || s->k.rows == 0) return 1;
    const int tile = grad_tile_k(s->k);
    const int64_t waves = tile_slots(s->k.rows, s->k.count, tile) * s->kv_heads * (tile / 32), work = s->q.rows / s->q.count * (s->heads / s->kv_heads);
    if (work < 640) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>({(2560 + waves / 2) / waves, work / (waves < 512 ? 128 : 512), 8}));
}
int64_t grad_slots_q(const he_attn *s) { return tile_slots(s->q.rows, s->q.count, grad_tile_q(s->q)); }
int64_t grad_slots_k(const he_attn *s) { return tile_slots(s->k.rows, s->k.count, grad_tile_k(s->k)); }
// numbers of k_attn_grad_size, in whole vectors of 16 bytes
size_t grad_sizes(const he_attn *s) { return s->type == HE_F16 ? (size_t)((grad_slots_q(s) + grad_slots_k(s)) * s->kv_heads + 3) / 4 * 4 : 0; }
size_t attn_bytes(const he_attn *s, bool backward)
{
    const size_t rows = (size_t)s->q.rows * s->heads;
    if (backward) {
        if (s->q.count == 0) return 0;
        const int splits = grad_splits(s);
        return (rows + 3) / 4 * 16 + grad_sizes(s) * 4 + (splits > 1 ? (size_t)splits * 2 * s->kv_heads * s->k.rows * s->dim * 4 : 0);
    }
    const AttnPlan p = attn_plan(s);
    return p.splits > 1 ? rows * p.splits * (s->dim + 1) * 4 : 0;
}
AttnArgs attn_args(const he_attn *s)
{
    AttnArgs a;
    memset(&a, 0, sizeof(a));
    a.sq = spans_of(&s->q);
    a.sk = spans_of(&s->k);
    a.heads = s->heads;
    a.group = s->heads / s->kv_heads;
    a.dim = s->dim;
    a.scale = (float)s->scale;
    a.cap = (float)s->cap;
    a.slope = s->d_slopes;
    a.splits = 1;
    a.fill = s->fill;
    return a;
}
// work-groups, a multiple of eight for the eight dies; false: more than a launch holds
bool attn_grid(AttnArgs &a, int64_t slots, int64_t w, unsigned &grid)
{
    if (w >= ((int64_t)1 << 31) / ATTN_THREADS) return false;
    a.slots = (int)slots;
    a.work = (unsigned)w;
    grid = (unsigned)((w + 7) / 8 * 8);
    return true;
}
#define SET(dst, h) a.dst##_row = (h)->row, a.dst##_head = (h)->head

} // namespace

extern "C" int32_t he_layer_norm(he_ctx *ctx, const he_norm *n, const he_rows *x, const he_rows *residual, const void *d_w, const void *d_b,
                                 const he_rows *y, const he_rows *sum, float *d_mean, float *d_rstd, void *stream)
{
    if (!ctx || norm_check(n) != HE_OK || !(n->eps >= 0.0) || !std::isfinite((float)n->eps)) return HE_EINVAL;
    if (n->rows == 0) {
        NEEDS_DEVICE(ctx);
        return HE_OK;
    }
    const size_t size_w = type_size(n->weight_type);
    if (!rows_ok(x, n->width, n->type) || !rows_ok(y, n->width, n->type)) return HE_EINVAL;
    if (!words_ok(d_w, size_w) || !words_ok(d_b, size_w) || !words_ok(d_mean) || !words_ok(d_rstd)) return HE_EINVAL;
    if (residual && (!rows_ok(residual, n->width, n->type) || !rows_ok(sum, n->width, n->type))) return HE_EINVAL;
    NEEDS_DEVICE(ctx);
    if (!residual) sum = nullptr;
    NormArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x->d, a.x_row = x->stride, a.y = y->d, a.y_row = y->stride;
    if (residual) a.r = residual->d, a.r_row = residual->stride, a.s = sum->d, a.s_row = sum->stride;
    a.w = d_w, a.b = d_b, a.mean = d_mean, a.rstd = d_rstd;
    a.rows = (int)n->rows, a.width = n->width, a.eps = (float)n->eps;
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    const double row = (double)n->width * type_size(n->type);
    rows_launch(n->type).norm(ctx, (hipStream_t)stream, n->rows * (row * (residual ? 4 : 2) + 8) + 2.0 * n->width * type_size(n->weight_type),
                              n->weight_type == HE_F32, a);
    return launched(ctx);
}

extern "C" int32_t he_layer_norm_workspace_bytes(const he_ctx *ctx, const he_norm *n, size_t *out)
{
    if (!ctx || !out || norm_check(n) != HE_OK) return HE_EINVAL;
    *out = n->rows ? (size_t)norm_parts(n->rows) * 2 * n->width * sizeof(float) : 0;
    return HE_OK;
}

extern "C" int32_t he_layer_norm_grad(he_ctx *ctx, const he_norm *n, const he_rows *dy, const he_rows *s, const void *d_w, const float *d_mean,
                                      const float *d_rstd, const he_rows *add, const he_rows *ds, void *d_dw, void *d_db, void *d_ws, size_t ws_bytes,
                                      void *stream)
{
    if (!ctx || norm_check(n) != HE_OK) return HE_EINVAL;
    const size_t size_w = type_size(n->weight_type);
    if (!words_ok(d_w, size_w) || !words_ok(d_dw, size_w) || !words_ok(d_db, size_w)) return HE_EINVAL;
    NormGradArgs a;
    memset(&a, 0, sizeof(a));
    a.rows = (int)n->rows, a.width = n->width;
    const int parts = n->rows ? norm_parts(n->rows) : 0;
    if (n->rows) {
        if (!rows_ok(dy, n->width, n->type) || !rows_ok(s, n->width, n->type) || !rows_ok(ds, n->width, n->type)) return HE_EINVAL;
        if (!words_ok(d_mean) || !words_ok(d_rstd) || (add && !rows_ok(add, n->width, n->type))) return HE_EINVAL;
        if (!d_ws || ws_bytes < (size_t)parts * 2 * n->width * sizeof(float)) return HE_EWORKSPACE;
        if (!aligned(d_ws, 4)) return HE_EINVAL;
        a.dy = dy->d, a.dy_row = dy->stride, a.s = s->d, a.s_row = s->stride, a.ds = ds->d, a.ds_row = ds->stride;
        if (add) a.add = add->d, a.add_row = add->stride;
        a.w = d_w, a.mean = d_mean, a.rstd = d_rstd, a.part = (float *)d_ws;
    }
    NEEDS_DEVICE(ctx);
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    const RowsLaunch &l = rows_launch(n->type);
    const bool ww = n->weight_type == HE_F32;
    const double row = (double)n->width * type_size(n->type), part = (double)parts * 2 * n->width * 4;
    if (n->rows) l.norm_grad(ctx, (hipStream_t)stream, n->rows * (row * (add ? 4 : 3) + 8) + part, ww, parts, a);
    l.weight_grad(ctx, (hipStream_t)stream, part + 2.0 * n->width * type_size(n->weight_type), ww, (const float *)d_ws, parts, n->width, d_dw, d_db);
    return launched(ctx);
}

extern "C" int32_t he_pool_workspace_bytes(const he_ctx *ctx, const he_spans *s, int32_t width, size_t *out)
{
    if (!ctx || !out || spans_check(s) != HE_OK || width < 1 || width > (1 << 20)) return HE_EINVAL;
    *out = pool_bytes(s, width);
    return HE_OK;
}

extern "C" int32_t he_pool(he_ctx *ctx, int32_t type, const he_spans *s, int32_t width, const he_rows *x, float *d_e, void *d_ws, size_t ws_bytes,
                           void *stream)
{
    if (!ctx || spans_check(s) != HE_OK || !type_ok(type) || width < 1 || width > (1 << 20)) return HE_EINVAL;
    if (s->count == 0) {
        NEEDS_DEVICE(ctx);
        return HE_OK;
    }
    if (!words_ok(d_e) || (s->rows > 0 && !rows_ok(x, width, type))) return HE_EINVAL;
    PoolArgs a;
    memset(&a, 0, sizeof(a));
    if (s->rows > 0) a.x = x->d, a.x_row = x->stride;
    a.e = d_e, a.s = spans_of(s), a.width = width, a.tile = pool_tile(s), a.part = (float *)d_ws;
    const size_t need = pool_bytes(s, width);
    if (need && (!d_ws || ws_bytes < need)) return HE_EWORKSPACE;
    if (need && !aligned(d_ws, 4)) return HE_EINVAL;
    NEEDS_DEVICE(ctx);
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    rows_launch(type).pool(ctx, (hipStream_t)stream, (double)s->rows * width * type_size(type) + 4.0 * s->count * width,
                           a.tile ? (unsigned)tile_slots(s->rows, s->count, a.tile) : 0, a);
    return launched(ctx);
}

extern "C" int32_t he_pool_grad(he_ctx *ctx, int32_t type, const he_spans *s, int32_t width, const float *d_de, const he_rows *dx, int32_t fill,
                                void *stream)
{
    if (!ctx || spans_check(s) != HE_OK || !type_ok(type) || width < 1 || width > (1 << 20)) return HE_EINVAL;
    if (s->count == 0 || s->rows == 0) {
        NEEDS_DEVICE(ctx);
        return HE_OK;
    }
    if (!words_ok(d_de) || !rows_ok(dx, width, type)) return HE_EINVAL;
    NEEDS_DEVICE(ctx);
    PoolGradArgs a;
    memset(&a, 0, sizeof(a));
    a.de = d_de, a.dx = dx->d, a.dx_row = dx->stride, a.s = spans_of(s), a.width = width, a.fill = fill, a.tile = pool_grad_tile(s);
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    rows_launch(type).pool_grad(ctx, (hipStream_t)stream, (double)s->rows * width * type_size(type) + 4.0 * s->count * width,
                                (unsigned)tile_slots(s->rows, s->count, a.tile), a);
    return launched(ctx);
}

extern "C" int32_t he_attention_workspace_bytes(const he_ctx *ctx, const he_attn *s, int32_t backward, size_t *out)
{
    if (!ctx || !out || attn_check(s) != HE_OK) return HE_EINVAL;
    *out = attn_bytes(s, backward != 0);
    return HE_OK;
}

extern "C" int32_t he_attention(he_ctx *ctx, const he_attn *s, const he_heads *q, const he_heads *k, const he_heads *v, const he_heads *o,
                                float *d_lse, void *d_ws, size_t ws_bytes, void *stream)
{
    if (!ctx || attn_check(s) != HE_OK) return HE_EINVAL;
    if (s->q.rows == 0 || s->q.count == 0) {
        NEEDS_DEVICE(ctx);
        return HE_OK;
    }
    if (!heads_ok(q, s->type) || !out_ok(o, s, s->q.rows, s->heads) || !words_ok(d_lse)) return HE_EINVAL;
    if (s->k.rows > 0 && (!heads_ok(k, s->type) || !heads_ok(v, s->type))) return HE_EINVAL;
    const size_t need = attn_bytes(s, false);
    if (need && (!d_ws || ws_bytes < need)) return HE_EWORKSPACE;
    if (need && !aligned(d_ws, 16)) return HE_EINVAL;
    const AttnPlan p = attn_plan(s);
    AttnArgs a = attn_args(s);
    a.q = q->d, a.o = o->d, a.lse = d_lse, a.splits = p.splits, a.pack = p.pack;
    SET(q, q), SET(o, o);
    if (s->k.rows > 0) {
        a.k = k->d, a.v = v->d;
        SET(k, k), SET(v, v);
    }
    a.part_o = (float *)d_ws;
    a.part_lse = a.part_o + (size_t)p.splits * s->heads * s->q.rows * s->dim;
    unsigned grid;
    if (!attn_grid(a, p.slots, p.groups, grid)) return HE_EINVAL;
    const int64_t rows = s->q.rows * s->heads;
    NEEDS_DEVICE(ctx);
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    const AttnLaunch &l = attn_launch(s->type, s->dim);
    const double size = (double)type_size(s->type) * s->dim, kv = 2.0 * s->k.rows * s->kv_heads * size;
    l.fwd(ctx, (hipStream_t)stream, rows * (2 * size + 4) + kv, p.tile, grid, a);
    if (p.splits > 1)
        l.join(ctx, (hipStream_t)stream, rows * (size + 4 + 4.0 * p.splits * (s->dim + 1)), (unsigned)((rows + 3) / 4), a);
    return launched(ctx);
}

extern "C" int32_t he_attention_grad(he_ctx *ctx, const he_attn *s, const he_heads *go, const he_heads *q, const he_heads *k, const he_heads *v,
                                     const he_heads *o, const float *d_lse, const he_heads *dq, const he_heads *dk, const he_heads *dv, void *d_ws,
                                     size_t ws_bytes, void *stream)
{
    if (!ctx || attn_check(s) != HE_OK) return HE_EINVAL;
    if (s->q.count == 0) {
        NEEDS_DEVICE(ctx);
        return HE_OK;
    }
    const bool some_q = s->q.rows > 0, some_k = s->k.rows > 0;
    if (some_q && (!heads_ok(q, s->type) || !heads_ok(o, s->type) || !heads_ok(go, s->type) || !out_ok(dq, s, s->q.rows, s->heads) || !words_ok(d_lse)))
        return HE_EINVAL;
    if (some_k && (!heads_ok(k, s->type) || !heads_ok(v, s->type) || !out_ok(dk, s, s->k.rows, s->kv_heads) ||
                   !out_ok(dv, s, s->k.rows, s->kv_heads)))
        return HE_EINVAL;
    const size_t need = attn_bytes(s, true);
    if (need && (!d_ws || ws_bytes < need)) return HE_EWORKSPACE;
    if (need && !aligned(d_ws, 16)) return HE_EINVAL;
    AttnArgs a = attn_args(s);
    if (some_q) {
        a.q = q->d, a.o_in = o->d, a.go = go->d, a.dq = dq->d;
        SET(q, q), SET(oi, o), SET(go, go), SET(dq, dq);
    }
    if (some_k) {
        a.k = k->d, a.v = v->d, a.dk = dk->d, a.dv = dv->d;
        SET(k, k), SET(v, v), SET(dk, dk), SET(dv, dv);
    }
    a.lse = const_cast<float *>(d_lse);
    const int64_t slots_q = grad_slots_q(s), slots_k = grad_slots_k(s);
    const int tile_q = grad_tile_q(s->q), tile_k = grad_tile_k(s->k);
    a.delta = (float *)d_ws;
    a.v_size = a.delta + (s->q.rows * s->heads + 3) / 4 * 4;
    a.go_size = a.v_size + slots_k * s->kv_heads;
    a.slots_q = (int)std::min<int64_t>(slots_q, INT32_MAX), a.tile_q = tile_q, a.slots_k = (int)std::min<int64_t>(slots_k, INT32_MAX), a.tile_k = tile_k;
    AttnArgs b = a;
    b.splits = grad_splits(s);
    b.part_o = a.v_size + grad_sizes(s);
    unsigned grid_q = 0, grid_kv = 0;
    if (!attn_grid(a, slots_q, slots_q * s->heads, grid_q) || !attn_grid(b, slots_k, slots_k * s->kv_heads * b.splits, grid_kv)) return HE_EINVAL;
    const int64_t rows_kv = s->k.rows * s->kv_heads;
    NEEDS_DEVICE(ctx);
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    const AttnLaunch &l = attn_launch(s->type, s->dim);
    const double size = (double)type_size(s->type) * s->dim, qb = s->q.rows * s->heads * size, kb = s->k.rows * s->kv_heads * size;
    if (l.grad_size && some_q && some_k)
        l.grad_size(ctx, (hipStream_t)stream, qb + kb, (unsigned)std::min<int64_t>(((slots_q + slots_k) * s->kv_heads + 3) / 4, 1 << 22), a);
    if (some_q) l.grad_q(ctx, (hipStream_t)stream, 4 * qb + 2 * kb + 8.0 * s->q.rows * s->heads, tile_q, grid_q, a);
    if (some_k) l.grad_kv(ctx, (hipStream_t)stream, 2 * qb + 4 * kb + 8.0 * s->q.rows * s->heads, tile_k, grid_kv, b);
    if (some_k && b.splits > 1) l.grad_join(ctx, (hipStream_t)stream, 2.0 * rows_kv * (size + 4.0 * b.splits * s->dim), (unsigned)((rows_kv + 3) / 4), b);
    return launched(ctx);
}
