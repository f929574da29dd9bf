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
static constexpr unsigned GRID_THREADS = 1u << 31; // of one launch: the hardware counts them in 32 bits

// Threads per row and vectors per thread by the width: the fewest threads that hold a row in few registers, since a sum over a wave or less costs no
// barrier.
template <int N> using Int = std::integral_constant<int, N>;
template <class F> static void row_shape(int width, F f)
{
    if (width < VEC) return f(Int<32>{}, Int<1>{}, Int<WIDTH_SMALL>{});
#define SHAPE(tpr, nc)                                                                                               \
    if (width <= VEC * (tpr) * (nc)) {                                                                               \
        if (width % VEC) return f(Int<tpr>{}, Int<nc>{}, Int<WIDTH_ODD>{});                                          \
        return f(Int<tpr>{}, Int<nc>{}, Int<WIDTH_EVEN>{});                                                          \
    }
    SHAPE(32, 1) SHAPE(32, 2) SHAPE(32, 3) SHAPE(32, 4)
    SHAPE(64, 3) SHAPE(64, 4)
    SHAPE(256, 2) SHAPE(256, 3) SHAPE(256, 4)
    SHAPE(1024, 2) SHAPE(1024, 4)
#undef SHAPE
}

static void norm(he_ctx *c, hipStream_t st, double bytes, bool wide_w, const NormArgs &a)
{
    row_shape(a.width, [&](auto tpr, auto nc, auto kind) {
        constexpr int threads = tpr > 256 ? tpr : 256, rpw = threads / tpr;
        constexpr int64_t most = GRID_THREADS / threads;
        NormArgs part = a;
        for (int64_t first = 0; first < a.rows; first += most * rpw) {
            part.first = (int)first;
            const unsigned grid = (unsigned)std::min(most, (a.rows - first + rpw - 1) / rpw);
            if (wide_w)
                KLAUNCH_T(c, st, KID_NORM, bytes, (k_layer_norm<T, float, VEC, tpr, nc, kind>), grid, threads, part);
            else
                KLAUNCH_T(c, st, KID_NORM, bytes, (k_layer_norm<T, T, VEC, tpr, nc, kind>), grid, threads, part);
            bytes = 0.0; // the profile counts them once
        }
    });
}
static void norm_grad(he_ctx *c, hipStream_t st, double bytes, bool wide_w, int parts, const NormGradArgs &a)
{
    row_shape(a.width, [&](auto tpr, auto nc, auto kind) {
        constexpr int threads = tpr > 256 ? tpr : 256;
        if (wide_w)
            KLAUNCH_T(c, st, KID_NORM_GRAD, bytes, (k_layer_norm_grad<T, float, VEC, tpr, nc, kind>), (unsigned)parts, threads, a);
        else
            KLAUNCH_T(c, st, KID_NORM_GRAD, bytes, (k_layer_norm_grad<T, T, VEC, tpr, nc, kind>), (unsigned)parts, threads, a);
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

static void pool(he_ctx *c, hipStream_t st, double bytes, unsigned slots, const PoolArgs &a)
{
    const int chunks = (a.width + VEC - 1) / VEC, cl = chunks < 256 ? chunks : 256;
    const unsigned cols = (unsigned)((chunks + cl - 1) / cl);
    if (a.tile) {
        KLAUNCH_T(c, st, KID_POOL, bytes, (k_pool<T, VEC, 256>), dim3(slots, cols), 256, a, cl);
        bytes = 4.0 * a.width * (slots + a.s.count);
        if (slots >= (unsigned)a.s.count * POOL_SHARED_TILES)
            KLAUNCH(c, st, KID_POOL_JOIN, bytes, k_pool_join<8>, dim3((unsigned)a.s.count, (unsigned)((a.width + 31) / 32)), a);
        else
            KLAUNCH(c, st, KID_POOL_JOIN, bytes, k_pool_join<1>, dim3((unsigned)a.s.count, (unsigned)((a.width + 255) / 256)), a);
    } else
        KLAUNCH_T(c, st, KID_POOL, bytes, (k_pool<T, VEC, 1024>), dim3((unsigned)a.s.count, cols), 1024, a, cl);
}
static void pool_grad(he_ctx *c, hipStream_t st, double bytes, unsigned slots, const PoolGradArgs &a)
{
    const int chunks = (a.width + VEC - 1) / VEC, cl = chunks < 256 ? chunks : 256;
    KLAUNCH(c, st, KID_POOL_GRAD, bytes, (k_pool_grad<T, VEC>), dim3(slots, (unsigned)((chunks + cl - 1) / cl)), a, cl);
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
