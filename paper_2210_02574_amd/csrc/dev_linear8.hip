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

template <int MB, int NB, int WM, int WN, int G, int OCC, bool PART = false> static void tiles(he_ctx *c, hipStream_t st, double bytes, Linear8Args a)
{
    constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN;
    a.tiles_m = (a.rows + BM - 1) / BM, a.tiles_n = (a.channels + BN - 1) / BN;
    KLAUNCH_T(c, st, KID_LINEAR8, bytes, (k_linear8<T, MB, NB, WM, WN, G, OCC, PART>), dim3((unsigned)(a.tiles_m * a.tiles_n), PART ? a.splits : 1), 64 * WM * WN * G, a);
}
static void product(he_ctx *c, hipStream_t st, double bytes, int tile, const Linear8Args &a)
{
    if (tile == LINEAR8_256)
        tiles<4, 2, 2, 4, 1, 2>(c, st, bytes, a);
    else if (tile == LINEAR8_128)
        tiles<2, 1, 2, 4, 1, 4>(c, st, bytes, a);
    else if (tile == LINEAR8_64)
        tiles<1, 1, 2, 2, 1, 4>(c, st, bytes, a);
    else if (a.splits == 1)
        tiles<1, 1, 2, 2, 4, 4>(c, st, bytes, a);
    else {
        tiles<1, 1, 2, 2, 4, 4, true>(c, st, bytes, a);
        const double part = 4.0 * a.splits * a.rows * a.channels;
        KLAUNCH(c, st, KID_LINEAR8_JOIN, part + (double)sizeof(T) * a.rows * a.channels, (k_linear8_join<T>), (unsigned)((a.rows * (int64_t)((a.channels + 3) / 4) + 255) / 256), a);
    }
}

#define NAME_(t) linear8_launch_##t
#define NAME(t) NAME_(t)
void NAME(HE_TYPE)(Linear8Launch &t)
{
    t.product = product;
}
