// Product of 8-bit rows and weights with results of one type (HE_TYPE: HE_F32, HE_F16, HE_BF16).
#include "enc_launch.h"
#include "kernels_linear8.h"

#if HE_TYPE == 0
typedef float T;
#elif HE_TYPE == 1
typedef f16 T;
#else
typedef bf16 T;
#endif

template <int MB, int NB> static void tiles(he_ctx *c, hipStream_t st, double bytes, Linear8Args a)
{
    a.tiles_m = (a.rows + 64 * MB - 1) / (64 * MB), a.tiles_n = (a.channels + 64 * NB - 1) / (64 * NB);
    KLAUNCH_T(c, st, KID_LINEAR8, bytes, (k_linear8<T, MB, NB>), (unsigned)(a.tiles_m * a.tiles_n), 256, a);
}
template <int MB> static void few(he_ctx *c, hipStream_t st, double bytes, int waves, const Linear8Args &a)
{
    const dim3 grid((unsigned)((a.channels + 15) / 16), (unsigned)((a.rows + 16 * MB - 1) / (16 * MB)));
    KLAUNCH_T(c, st, KID_LINEAR8_FEW, bytes, (k_linear8_few<T, MB>), grid, 64 * waves, a);
}

static void product(he_ctx *c, hipStream_t st, double bytes, int tile, const Linear8Args &a)
{
    if (tile == 256)
        tiles<4, 4>(c, st, bytes, a);
    else if (tile == 128)
        tiles<2, 2>(c, st, bytes, a);
    else
        tiles<1, 1>(c, st, bytes, a);
}
static void product_few(he_ctx *c, hipStream_t st, double bytes, int blocks, int waves, const Linear8Args &a)
{
    if (blocks == 1)
        few<1>(c, st, bytes, waves, a);
    else if (blocks == 2)
        few<2>(c, st, bytes, waves, a);
    else
        few<4>(c, st, bytes, waves, a);
}

#define NAME_(t) linear8_launch_##t
#define NAME(t) NAME_(t)
void NAME(HE_TYPE)(Linear8Launch &t)
{
    t.tiles = product;
    t.few = product_few;
}
