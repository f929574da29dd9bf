// Entry points of the operators on token states: attention inside sequences, layer norm and root-mean-square norm, mean over sequences, rows in 8 bits and their
// products.
#include <cmath>
#include <cstring>

#include "enc_launch.h"
#include "kernels_attn.h"
#include "kernels_linear8.h"
#include "kernels_norm.h"
#include "kernels_pool.h"
#include "kernels_rows8.h"
#include "linear8_plan.h"

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

// ---- rows in 8 bits ----------------------------------------------------------------------------------------------------------

const Rows8Launch &rows8_launch(int32_t t)
{
    static const Rows8Launch tables[3] = {
        [] { Rows8Launch x{}; rows8_launch_0(x); return x; }(),
        [] { Rows8Launch x{}; rows8_launch_1(x); return x; }(),
        [] { Rows8Launch x{}; rows8_launch_2(x); return x; }(),
    };
    return tables[t];
}
const Linear8Launch &linear8_launch(int32_t t)
{
    static const Linear8Launch tables[3] = {
        [] { Linear8Launch x{}; linear8_launch_0(x); return x; }(),
        [] { Linear8Launch x{}; linear8_launch_1(x); return x; }(),
        [] { Linear8Launch x{}; linear8_launch_2(x); return x; }(),
    };
    return tables[t];
}
// rows that are written, and rows that a product reads by pieces of 16 bytes
bool rows8_ok(const he_rows8 *r, int64_t width) { return r && r->d && words_ok(r->d_scale) && r->stride >= width; }
bool pieces_ok(const he_rows8 *r, int64_t width) { return rows8_ok(r, width) && aligned(r->d, 16) && r->stride % 16 == 0 && r->stride < 1 << 23; }

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

namespace {

// What both forms of the root-mean-square norm take; `y` and `out` are the caller's to set.
int32_t rms_args(RmsArgs &a, const he_norm *n, const he_rows *x, const he_rows *residual, const void *d_w, const he_rows *sum)
{
    memset(&a, 0, sizeof(a));
    if (!rows_ok(x, n->width, n->type) || !words_ok(d_w, type_size(n->weight_type))) return HE_EINVAL;
    if (residual && (!rows_ok(residual, n->width, n->type) || !rows_ok(sum, n->width, n->type))) return HE_EINVAL;
    a.x = x->d, a.x_row = x->stride, a.w = d_w;
    if (residual) a.r = residual->d, a.r_row = residual->stride, a.s = sum->d, a.s_row = sum->stride;
    a.rows = (int)n->rows, a.width = n->width, a.eps = (float)n->eps;
    return HE_OK;
}
// Work-groups of its backward pass: a lone one where it has no more than two rounds of rows, four of narrow ones, which saves a launch (bf16, us with one and with one to a round: in a
// captured graph 118 x 64, four rounds of 32 rows, 5.5, 5.7; five 6.1, 5.6; 59 x 100, four of 16, 5.3, 5.5; five 5.9, 5.4; 22 x 400, three of 8, 5.3, 5.4; four 6.2, 5.5; 14 x 768, two,
// 5.5, 6.1; three 6.7, 6.2; 2 x 8192 5.8, 6.2; 3 7.6, 6.2; a call by itself takes 5.2 to 6.3 in all of these up to the limit, with two launches 8.6 to 9.1); else one for each of the 256
// CUs and no more than rows need, two where these would take more than three rounds (bf16 with ds', captured, one and two to a CU: 768 x 8192 17.3, 18.1 and 520 x 8192 17.8, 20.0; 800 x 8192
// 19.2, 18.5; 6142 x 768, 768 work-groups' rows, 12.5, 12.2; 6398 x 768 13.9, 12.9; 3071 x 1901 18.5, 17.8; 3199 x 1901 21.1, 19.3; 24566 x 64 7.9, 8.3; 31990 x 64 9.1, 8.7; fp32
// 768 x 4096 13.3, 14.3; 2799 x 1021 13.7, 13.7; 3199 x 1021 15.7, 14.8).
int rms_parts(const he_norm *n)
{
    const int vec = 16 / (int)type_size(n->type);
    const int rows = n->width <= vec * 8 ? 32 : n->width <= vec * 16 ? 16 : n->width <= vec * 128 ? 8 : n->width <= vec * 256 ? 4 : 1; // of a work-group at a time
    const int64_t need = (n->rows + rows - 1) / rows;
    return need <= (n->width <= vec * 64 ? 4 : 2) ? 1 : (int)std::min<int64_t>(need <= 768 ? 256 : 512, need);
}
size_t rms_bytes(const he_norm *n) { return n->rows && rms_parts(n) > 1 ? (size_t)rms_parts(n) * n->width * sizeof(float) : 0; }
// Whether rows of `width` bytes, `stride` bytes apart, are whole lines.
bool whole_lines(const void *d, int64_t stride, int64_t width) { return (((int64_t)d | stride | width) & 127) == 0; }
// How results of `span` bytes are written, one to a row or two, by a call that moves `bytes` in all.  Times in us in bf16, kept, through and past: root-mean-square norm, one result,
// 16384 x 768 8.2, 6.2, 6.3; 65536 x 768 30, 29, 29; 131072 x 768 72, 72, 57; two results 16384 x 768 15.5, 16.1, 15.9; 49152 x 768 48, 48, 44; 65536 x 768 74, 73, 58; rows in 8 bits
// 16384 x 768 9.3, 7.9, 8.1; 131072 x 768 51, 50, 44; gradients with ds' 32768 x 768 37, 37, 37; 65536 x 768 81, 80, 72.  With two kernels that read the results:
// 32768 x 768 62, 60, 62; 65536 x 768 126, 125, 118.
int how_written(double bytes, int64_t span, bool one, bool whole)
{
    if (!whole) return KEEP;
    if (bytes > 256.0 * (1 << 20)) return PAST; // the last-level cache's size
    return one && span <= INT32_MAX ? THROUGH : KEEP;
}
bool eps_ok(const he_norm *n) { return n->eps >= 0.0 && std::isfinite((float)n->eps); }

} // namespace

extern "C" int32_t he_rms_norm(he_ctx *ctx, const he_norm *n, const he_rows *x, const he_rows *residual, const void *d_w, const he_rows *y,
                               const he_rows *sum, float *d_rstd, void *stream)
{
    if (!ctx || norm_check(n) != HE_OK || !eps_ok(n)) return HE_EINVAL;
    if (n->rows == 0) {
        NEEDS_DEVICE(ctx);
        return HE_OK;
    }
    RmsArgs a;
    if (rms_args(a, n, x, residual, d_w, sum) != HE_OK || !rows_ok(y, n->width, n->type) || !words_ok(d_rstd)) return HE_EINVAL;
    a.y = y->d, a.y_row = y->stride, a.out = d_rstd;
    NEEDS_DEVICE(ctx);
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    const int64_t size = type_size(n->type), row = n->width * size;
    const double bytes = n->rows * ((double)row * (residual ? 4 : 2) + 4) + (double)n->width * type_size(n->weight_type);
    a.how = how_written(bytes, n->rows * y->stride * size, !residual, whole_lines(y->d, y->stride * size, row) && (!residual || whole_lines(sum->d, sum->stride * size, row)));
    rows8_launch(n->type).rms(ctx, (hipStream_t)stream, bytes, n->weight_type == HE_F32, a);
    return launched(ctx);
}

extern "C" int32_t he_rms_norm8(he_ctx *ctx, const he_norm *n, const he_rows *x, const he_rows *residual, const void *d_w, const he_rows8 *y,
                                const he_rows *sum, void *stream)
{
    if (!ctx || norm_check(n) != HE_OK || !eps_ok(n)) return HE_EINVAL;
    if (n->rows == 0) {
        NEEDS_DEVICE(ctx);
        return HE_OK;
    }
    RmsArgs a;
    if (rms_args(a, n, x, residual, d_w, sum) != HE_OK || !rows8_ok(y, n->width)) return HE_EINVAL;
    a.y = y->d, a.y_row = y->stride, a.out = y->d_scale;
    NEEDS_DEVICE(ctx);
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    const int64_t size = type_size(n->type), row = n->width * size;
    const double bytes = n->rows * ((double)row * (residual ? 3 : 1) + n->width + 4) + (double)n->width * type_size(n->weight_type);
    a.how = how_written(bytes, n->rows * y->stride, !residual, whole_lines(y->d, y->stride, n->width) && (!residual || whole_lines(sum->d, sum->stride * size, row)));
    rows8_launch(n->type).rms8(ctx, (hipStream_t)stream, bytes, n->weight_type == HE_F32, a);
    return launched(ctx);
}

extern "C" int32_t he_rms_norm_workspace_bytes(const he_ctx *ctx, const he_norm *n, size_t *out)
{
    if (!ctx || !out || norm_check(n) != HE_OK) return HE_EINVAL;
    *out = rms_bytes(n);
    return HE_OK;
}

extern "C" int32_t he_rms_norm_grad(he_ctx *ctx, const he_norm *n, const he_rows *dy, const he_rows *s, const void *d_w, const float *d_rstd,
                                    const he_rows *add, const he_rows *ds, void *d_dw, void *d_ws, size_t ws_bytes, void *stream)
{
    if (!ctx || norm_check(n) != HE_OK) return HE_EINVAL;
    const size_t size_w = type_size(n->weight_type);
    if (!words_ok(d_w, size_w) || !words_ok(d_dw, size_w)) return HE_EINVAL;
    RmsGradArgs a;
    memset(&a, 0, sizeof(a));
    a.rows = (int)n->rows, a.width = n->width;
    const int parts = n->rows ? rms_parts(n) : 0;
    const size_t need = rms_bytes(n);
    if (n->rows) {
        if (!rows_ok(dy, n->width, n->type) || !rows_ok(s, n->width, n->type) || !rows_ok(ds, n->width, n->type)) return HE_EINVAL;
        if (!words_ok(d_rstd) || (add && !rows_ok(add, n->width, n->type))) return HE_EINVAL;
        if (need && (!d_ws || ws_bytes < need)) return HE_EWORKSPACE;
        if (need && !aligned(d_ws, 4)) return HE_EINVAL;
        a.dy = dy->d, a.dy_row = dy->stride, a.s = s->d, a.s_row = s->stride, a.ds = ds->d, a.ds_row = ds->stride;
        if (add) a.add = add->d, a.add_row = add->stride;
        a.w = d_w, a.rstd = d_rstd, a.part = (float *)d_ws, a.dw = d_dw;
    }
    NEEDS_DEVICE(ctx);
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    const Rows8Launch &l = rows8_launch(n->type);
    const bool ww = n->weight_type == HE_F32;
    const int64_t size = type_size(n->type), row = n->width * size;
    const double part = (double)need, bytes = n->rows * ((double)row * (add ? 4 : 3) + 4) + part;
    if (n->rows) {
        a.how = how_written(bytes, 0, false, whole_lines(ds->d, ds->stride * size, row));
        l.rms_grad(ctx, (hipStream_t)stream, bytes, ww, parts, a);
    }
    if (parts != 1)
        l.weight_grad(ctx, (hipStream_t)stream, part + (double)n->width * type_size(n->weight_type), ww, (const float *)d_ws, parts, n->width, d_dw);
    return launched(ctx);
}

extern "C" int32_t he_quantize8(he_ctx *ctx, int32_t type, int64_t rows, int32_t width, int32_t gelu, const he_rows *x, const he_rows8 *y, void *stream)
{
    if (!ctx || !type_ok(type) || rows < 0 || rows > MAX_ROWS || width < 1 || width > NORM_MAX_WIDTH) return HE_EINVAL;
    if (rows == 0) {
        NEEDS_DEVICE(ctx);
        return HE_OK;
    }
    if (!rows_ok(x, width, type) || !rows8_ok(y, width)) return HE_EINVAL;
    NEEDS_DEVICE(ctx);
    Rows8Args a;
    memset(&a, 0, sizeof(a));
    a.x = x->d, a.x_row = x->stride, a.y = y->d, a.y_row = y->stride, a.scale = y->d_scale, a.rows = (int)rows, a.width = width;
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    const double bytes = rows * ((double)width * (type_size(type) + 1) + 4);
    a.how = how_written(bytes, rows * y->stride, true, whole_lines(y->d, y->stride, width));
    rows8_launch(type).quantize(ctx, (hipStream_t)stream, bytes, gelu != 0, a);
    return launched(ctx);
}

namespace {

int32_t product8_check(const he_product8 *p)
{
    if (!p || !type_ok(p->type) || (p->bias_type != p->type && p->bias_type != HE_F32)) return HE_EINVAL;
    if (p->rows < 0 || p->rows > MAX_ROWS || p->width < 1 || p->width > LINEAR8_MAX_WIDTH || p->channels < 1 || p->channels > 1 << 24) return HE_EINVAL;
    return HE_OK;
}

} // namespace

extern "C" int32_t he_linear8(he_ctx *ctx, const he_product8 *p, const he_rows8 *x, const he_rows8 *w, const void *d_bias, const he_rows *o, void *stream)
{
    if (!ctx || product8_check(p) != HE_OK || !pieces_ok(w, p->width)) return HE_EINVAL;
    if (d_bias && !words_ok(d_bias, type_size(p->bias_type))) return HE_EINVAL;
    if (p->rows == 0) {
        NEEDS_DEVICE(ctx);
        return HE_OK;
    }
    if (!pieces_ok(x, p->width) || !rows_ok(o, p->channels, p->type)) return HE_EINVAL;
    const Product8Plan plan = product8_plan(p->rows, p->width, p->channels, p->type == HE_F32);
    if (plan.tiles > 1 << 22) return HE_EINVAL; // more than a launch holds
    Linear8Args a;
    memset(&a, 0, sizeof(a));
    a.x = x->d, a.x_row = x->stride, a.x_scale = x->d_scale, a.w = w->d, a.w_row = w->stride, a.w_scale = w->d_scale;
    a.bias = d_bias, a.bias32 = p->bias_type == HE_F32, a.o = o->d, a.o_row = o->stride;
    a.rows = (int)p->rows, a.width = p->width, a.channels = p->channels;
    NEEDS_DEVICE(ctx);
    DeviceGuard dg(ctx);
    if (dg.rc != HE_OK) return dg.rc;
    const double bytes = (double)p->rows * (p->width + 4) + (double)p->channels * (p->width + 4) + (double)p->rows * p->channels * type_size(p->type) +
                         (d_bias ? (double)p->channels * type_size(p->bias_type) : 0.0);
    linear8_launch(p->type).product(ctx, (hipStream_t)stream, bytes, plan.tile, plan.groups, a);
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
