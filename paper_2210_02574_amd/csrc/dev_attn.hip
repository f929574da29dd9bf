// Attention kernels of one element type (HE_TYPE: HE_F32, HE_F16, HE_BF16) and one head size (HE_DIM: heads up to that many elements).
#include "enc_launch.h"
#include "kernels_attn.h"

#if HE_TYPE == 0
typedef float T;
#elif HE_TYPE == 1
typedef f16 T;
#else
typedef bf16 T;
#endif

static constexpr bool ATTN_WIDE = attn_wide(sizeof(T), HE_DIM);

// f with the variant of cap and distance bias
template <class F> static void by_mode(const AttnArgs &a, F f)
{
    const int mode = (a.cap > 0.f ? MODE_CAP : 0) | (a.slope ? MODE_SLOPE : 0);
    if constexpr (sizeof(T) == 2)
        if (a.cap > ATTN_FAST_CAP) {
            if (a.slope) return f(std::integral_constant<int, MODE_CAP | MODE_SLOPE | MODE_EXACT>{});
            return f(std::integral_constant<int, MODE_CAP | MODE_EXACT>{});
        }
    if (mode == 0)
        f(std::integral_constant<int, 0>{});
    else if (mode == MODE_CAP)
        f(std::integral_constant<int, MODE_CAP>{});
    else if (mode == MODE_SLOPE)
        f(std::integral_constant<int, MODE_SLOPE>{});
    else
        f(std::integral_constant<int, MODE_CAP | MODE_SLOPE>{});
}

static void attn_fwd(he_ctx *c, hipStream_t st, double bytes, int tile, unsigned grid, const AttnArgs &a)
{
    by_mode(a, [&](auto mode) {
        if (tile == 32)
            KLAUNCH_T(c, st, KID_ATTN_FEW, bytes, (k_attn_few<T, HE_DIM, 1, mode>), grid, ATTN_THREADS, a);
        else if (tile == 64)
            KLAUNCH_T(c, st, KID_ATTN_FEW, bytes, (k_attn_few<T, HE_DIM, 2, mode>), grid, ATTN_THREADS, a);
        else if (tile == 128)
            KLAUNCH_T(c, st, KID_ATTN, bytes, (k_attn<T, HE_DIM, 1, mode>), grid, ATTN_THREADS, a);
        else if constexpr (ATTN_WIDE && !(mode & MODE_CAP)) // (no plan has wide tiles under a cap)
            KLAUNCH_T(c, st, KID_ATTN, bytes, (k_attn<T, HE_DIM, 2, mode>), grid, ATTN_THREADS, a);
    });
}
static void attn_join(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a)
{
    KLAUNCH(c, st, KID_ATTN_JOIN, bytes, (k_attn_join<T>), grid, a);
}
static void attn_grad_size(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a)
{
    if constexpr (grad_lifted<T>()) KLAUNCH(c, st, KID_ATTN_GRAD_SIZE, bytes, (k_attn_grad_size<T, HE_DIM>), grid, a);
}
static void attn_grad_q(he_ctx *c, hipStream_t st, double bytes, int tile, unsigned grid, const AttnArgs &a)
{
    by_mode(a, [&](auto mode) {
        if (tile == 64)
            KLAUNCH_T(c, st, KID_ATTN_GRAD_Q, bytes, (k_attn_grad_q<T, HE_DIM, 2, mode>), grid, 128, a);
        else
            KLAUNCH_T(c, st, KID_ATTN_GRAD_Q, bytes, (k_attn_grad_q<T, HE_DIM, 4, mode>), grid, 256, a);
    });
}
static void attn_grad_kv(he_ctx *c, hipStream_t st, double bytes, int tile, unsigned grid, const AttnArgs &a)
{
    by_mode(a, [&](auto mode) {
        if (tile == 32)
            KLAUNCH_T(c, st, KID_ATTN_GRAD_KV, bytes, (k_attn_grad_kv<T, HE_DIM, 1, mode>), grid, 64, a);
        else if (tile == 64)
            KLAUNCH_T(c, st, KID_ATTN_GRAD_KV, bytes, (k_attn_grad_kv<T, HE_DIM, 2, mode>), grid, 128, a);
        else
            KLAUNCH_T(c, st, KID_ATTN_GRAD_KV, bytes, (k_attn_grad_kv<T, HE_DIM, 4, mode>), grid, 256, a);
    });
}
static void attn_grad_join(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a)
{
    KLAUNCH(c, st, KID_ATTN_GRAD_JOIN, bytes, (k_attn_grad_join<T>), grid, a);
}

#define NAME_(t, d) attn_launch_##t##_##d
#define NAME(t, d) NAME_(t, d)
void NAME(HE_TYPE, HE_DIM)(AttnLaunch &t)
{
    t.fwd = attn_fwd;
    t.join = attn_join;
    t.grad_size = grad_lifted<T>() ? attn_grad_size : nullptr;
    t.grad_q = attn_grad_q;
    t.grad_kv = attn_grad_kv;
    t.grad_join = attn_grad_join;
}
