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

template <int MB, int NB, int WM, int WN, int G, int OCC> static void tiles(he_ctx *c, hipStream_t st, double bytes, Linear8Args a)
{
    constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN;
    a.tiles_m = (a.rows + BM - 1) / BM, a.tiles_n = (a.channels + BN - 1) / BN;
    KLAUNCH_T(c, st, KID_LINEAR8, bytes, (k_linear8<T, MB, NB, WM, WN, G, OCC>), (unsigned)(a.tiles_m * a.tiles_n), 64 * WM * WN * G, a);
}
template <int BLK, int G> static void few(he_ctx *c, hipStream_t st, double bytes, Linear8Args a)
{
    a.tiles_m = (a.rows + BLK - 1) / BLK, a.tiles_n = (a.channels + BLK - 1) / BLK;
    KLAUNCH_T(c, st, KID_LINEAR8_FEW, bytes, (k_linear8_few<T, BLK, G>), (unsigned)(a.tiles_m * a.tiles_n), 64 * G, a);
}
static void product(he_ctx *c, hipStream_t st, double bytes, int tile, int groups, const Linear8Args &a)
{
    if (tile == 256)
        tiles<4, 2, 2, 4, 1, 2>(c, st, bytes, a);
    else if (tile == 192)
        tiles<2, 3, 4, 2, 1, 2>(c, st, bytes, a);
    else if (tile == 128)
        tiles<2, 1, 2, 4, 1, 4>(c, st, bytes, a);
    else if (tile == 64 && groups == 1)
        tiles<1, 1, 2, 2, 1, 4>(c, st, bytes, a);
    else if (tile == 64)
        tiles<1, 1, 2, 2, 4, 4>(c, st, bytes, a);
    else if (tile == 32)
        few<32, 4>(c, st, bytes, a);
    else if (groups == 4)
        few<16, 4>(c, st, bytes, a);
    else
        few<16, 8>(c, st, bytes, a);
}

#define NAME_(t) linear8_launch_##t
#define NAME(t) NAME_(t)
void NAME(HE_TYPE)(Linear8Launch &t)
{
    t.product = product;
}
