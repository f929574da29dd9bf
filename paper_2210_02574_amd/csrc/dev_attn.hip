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

template <int NWQ> static void fwd(he_ctx *c, hipStream_t st, double bytes, bool mods, unsigned grid, const AttnArgs &a)
{
    if (mods)
        KLAUNCH_T(c, st, KID_ATTN, bytes, (k_attn<T, HE_DIM, NWQ, true>), grid, ATTN_THREADS, a);
    else
        KLAUNCH_T(c, st, KID_ATTN, bytes, (k_attn<T, HE_DIM, NWQ, false>), grid, ATTN_THREADS, a);
}

static void attn_fwd(he_ctx *c, hipStream_t st, double bytes, int nwq, bool mods, unsigned grid, const AttnArgs &a)
{
    if (nwq == 1)
        fwd<1>(c, st, bytes, mods, grid, a);
    else if (nwq == 2)
        fwd<2>(c, st, bytes, mods, grid, a);
    else
        fwd<4>(c, st, bytes, mods, grid, a);
}
static void attn_join(he_ctx *c, hipStream_t st, double bytes, unsigned grid, const AttnArgs &a)
{
    KLAUNCH(c, st, KID_ATTN_JOIN, bytes, (k_attn_join<T>), grid, a);
}
static void attn_grad_q(he_ctx *c, hipStream_t st, double bytes, bool mods, unsigned grid, const AttnArgs &a)
{
    if (mods)
        KLAUNCH_T(c, st, KID_ATTN_GRAD_Q, bytes, (k_attn_grad_q<T, HE_DIM, true>), grid, ATTN_THREADS, a);
    else
        KLAUNCH_T(c, st, KID_ATTN_GRAD_Q, bytes, (k_attn_grad_q<T, HE_DIM, false>), grid, ATTN_THREADS, a);
}
static void attn_grad_kv(he_ctx *c, hipStream_t st, double bytes, bool mods, unsigned grid, const AttnArgs &a)
{
    if (mods)
        KLAUNCH_T(c, st, KID_ATTN_GRAD_KV, bytes, (k_attn_grad_kv<T, HE_DIM, true>), grid, ATTN_THREADS, a);
    else
        KLAUNCH_T(c, st, KID_ATTN_GRAD_KV, bytes, (k_attn_grad_kv<T, HE_DIM, false>), grid, ATTN_THREADS, a);
}

#define NAME_(t, d) attn_launch_##t##_##d
#define NAME(t, d) NAME_(t, d)
void NAME(HE_TYPE, HE_DIM)(AttnLaunch &t)
{
    t.fwd = attn_fwd;
    t.join = attn_join;
    t.grad_q = attn_grad_q;
    t.grad_kv = attn_grad_kv;
}
