// Layer norm and mean of one element type (HE_TYPE: HE_F32, HE_F16, HE_BF16).
#include "enc_launch.h"
#include "kernels_norm.h"
#include "kernels_pool.h"

#if HE_TYPE == 0
typedef float T;
#elif HE_TYPE == 1
typedef f16 T;
#else
typedef bf16 T;
#endif
static constexpr int VEC = 16 / sizeof(T);

// Threads per row and vectors per thread by the width: the fewest threads that hold a row in few registers, since a sum over a wave or less costs no
// barrier.
template <class F> static void row_shape(bool vec, int width, F f)
{
#define SHAPE(v, tpr, nc)                                                                                            \
    if (width <= (v) * (tpr) * (nc)) return f(std::integral_constant<int, v>{}, std::integral_constant<int, tpr>{}, std::integral_constant<int, nc>{});
    if (vec) {
        SHAPE(VEC, 32, 1) SHAPE(VEC, 32, 2) SHAPE(VEC, 32, 3) SHAPE(VEC, 32, 4)
        SHAPE(VEC, 64, 3) SHAPE(VEC, 64, 4)
        SHAPE(VEC, 256, 2) SHAPE(VEC, 256, 3) SHAPE(VEC, 256, 4)
        SHAPE(VEC, 1024, 2) SHAPE(VEC, 1024, 4)
    } else {
        SHAPE(1, 64, 2) SHAPE(1, 64, 4) SHAPE(1, 64, 8)
        SHAPE(1, 256, 4) SHAPE(1, 256, 8)
        SHAPE(1, 1024, 4) SHAPE(1, 1024, 8) SHAPE(1, 1024, 16)
    }
#undef SHAPE
}

static void norm(he_ctx *c, hipStream_t st, double bytes, bool vec, bool wide_w, const NormArgs &a)
{
    row_shape(vec, a.width, [&](auto v, auto tpr, auto nc) {
        constexpr int threads = tpr > 256 ? tpr : 256, rpw = threads / tpr;
        const unsigned grid = (unsigned)((a.rows + rpw - 1) / rpw);
        if (wide_w)
            KLAUNCH_T(c, st, KID_NORM, bytes, (k_layer_norm<T, float, v, tpr, nc>), grid, threads, a);
        else
            KLAUNCH_T(c, st, KID_NORM, bytes, (k_layer_norm<T, T, v, tpr, nc>), grid, threads, a);
    });
}
static void norm_grad(he_ctx *c, hipStream_t st, double bytes, bool vec, bool wide_w, int parts, const NormGradArgs &a)
{
    row_shape(vec, a.width, [&](auto v, auto tpr, auto nc) {
        constexpr int threads = tpr > 256 ? tpr : 256;
        if (wide_w)
            KLAUNCH_T(c, st, KID_NORM_GRAD, bytes, (k_layer_norm_grad<T, float, v, tpr, nc>), (unsigned)parts, threads, a);
        else
            KLAUNCH_T(c, st, KID_NORM_GRAD, bytes, (k_layer_norm_grad<T, T, v, tpr, nc>), (unsigned)parts, threads, a);
    });
}
static void weight_grad(he_ctx *c, hipStream_t st, double bytes, bool wide_w, const float *part, int parts, int width, void *dw, void *db)
{
    const dim3 grid((unsigned)((width + 15) / 16), 2);
    if (wide_w)
        KLAUNCH(c, st, KID_NORM_WEIGHT_GRAD, bytes, (k_norm_weight_grad<float>), grid, part, parts, width, (float *)dw, (float *)db);
    else
        KLAUNCH(c, st, KID_NORM_WEIGHT_GRAD, bytes, (k_norm_weight_grad<T>), grid, part, parts, width, (T *)dw, (T *)db);
}

static void pool(he_ctx *c, hipStream_t st, double bytes, bool vec, const PoolArgs &a)
{
    const int v = vec ? VEC : 1, chunks = (a.width + v - 1) / v, cl = chunks < 256 ? chunks : 256;
    const dim3 grid((unsigned)a.s.count, (unsigned)((chunks + cl - 1) / cl), (unsigned)a.splits);
    if (vec)
        KLAUNCH_T(c, st, KID_POOL, bytes, (k_pool<T, VEC>), grid, POOL_THREADS, a, cl);
    else
        KLAUNCH_T(c, st, KID_POOL, bytes, (k_pool<T, 1>), grid, POOL_THREADS, a, cl);
    if (a.splits > 1) KLAUNCH(c, st, KID_POOL_JOIN, 4.0 * a.s.count * a.width * (a.splits + 1), k_pool_join, dim3((unsigned)a.s.count, (unsigned)((a.width + 255) / 256)), a);
}
static void pool_grad(he_ctx *c, hipStream_t st, double bytes, bool vec, unsigned slots, const PoolGradArgs &a)
{
    const int v = vec ? VEC : 1, chunks = (a.width + v - 1) / v, cl = chunks < 256 ? chunks : 256;
    const dim3 grid(slots, (unsigned)((chunks + cl - 1) / cl));
    if (vec)
        KLAUNCH(c, st, KID_POOL_GRAD, bytes, (k_pool_grad<T, VEC>), grid, a, cl);
    else
        KLAUNCH(c, st, KID_POOL_GRAD, bytes, (k_pool_grad<T, 1>), grid, a, cl);
}

#define NAME_(t) rows_launch_##t
#define NAME(t) NAME_(t)
void NAME(HE_TYPE)(RowsLaunch &t)
{
    t.norm = norm;
    t.norm_grad = norm_grad;
    t.weight_grad = weight_grad;
    t.pool = pool;
    t.pool_grad = pool_grad;
}
