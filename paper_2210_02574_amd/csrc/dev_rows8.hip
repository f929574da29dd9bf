// Root-mean-square norm and rows in 8 bits, of one element type (HE_TYPE: HE_F32, HE_F16, HE_BF16).
#include "enc_launch.h"
#include "kernels_rows8.h"

#if HE_TYPE == 0
typedef float T;
#elif HE_TYPE == 1
typedef f16 T;
#else
typedef bf16 T;
#endif
#include "row_shape.h"

// Eight or sixteen threads to narrow rows, of whose 32 most would idle while each wave computes scales for two rows alone: 64253 x 77 in fp16 in 8 bits 8.7 us, with 32 threads 13.9;
// error units 12.0, 20.8; the norm 6.2, 8.8; its gradients 13.7, 19.1; 65536 x 128 in bf16 in 8 bits 7.4, 12.7.
template <class F> static void narrow_shape(int width, F f)
{
    if (width < VEC) return f(Int<8>{}, Int<1>{}, Int<WIDTH_SMALL>{});
#define SHAPE(tpr)                                                                                                   \
    if (width <= VEC * (tpr)) {                                                                                      \
        if (width % VEC) return f(Int<tpr>{}, Int<1>{}, Int<WIDTH_ODD>{});                                           \
        return f(Int<tpr>{}, Int<1>{}, Int<WIDTH_EVEN>{});                                                           \
    }
    SHAPE(8) SHAPE(16)
#undef SHAPE
    row_shape(width, f);
}

// f(threads, grid, arguments) for each launch that the rows take
template <int TPR, class A, class F> static void by_rows(const A &a, F f)
{
    constexpr int threads = TPR > 256 ? TPR : 256, rpw = threads / TPR;
    constexpr int64_t most = GRID_THREADS / threads;
    A part = a;
    for (int64_t first = 0; first < a.rows; first += most * rpw) {
        part.first = (int)first;
        f(threads, (unsigned)std::min(most, (a.rows - first + rpw - 1) / rpw), part);
    }
}

static void rms(he_ctx *c, hipStream_t st, double bytes, bool wide_w, const RmsArgs &a)
{
    narrow_shape(a.width, [&](auto tpr, auto nc, auto kind) {
        by_rows<tpr>(a, [&](int threads, unsigned grid, const RmsArgs &part) {
            if (wide_w)
                KLAUNCH_T(c, st, KID_RMS, bytes, (k_rms_norm<T, float, VEC, tpr, nc, kind>), grid, threads, part);
            else
                KLAUNCH_T(c, st, KID_RMS, bytes, (k_rms_norm<T, T, VEC, tpr, nc, kind>), grid, threads, part);
            bytes = 0.0; // the profile counts them once
        });
    });
}
static void rms8(he_ctx *c, hipStream_t st, double bytes, bool wide_w, const RmsArgs &a)
{
    narrow_shape(a.width, [&](auto tpr, auto nc, auto kind) {
        by_rows<tpr>(a, [&](int threads, unsigned grid, const RmsArgs &part) {
            if (wide_w)
                KLAUNCH_T(c, st, KID_RMS8, bytes, (k_rms_norm8<T, float, VEC, tpr, nc, kind>), grid, threads, part);
            else
                KLAUNCH_T(c, st, KID_RMS8, bytes, (k_rms_norm8<T, T, VEC, tpr, nc, kind>), grid, threads, part);
            bytes = 0.0; // the profile counts them once
        });
    });
}
static void rms_grad(he_ctx *c, hipStream_t st, double bytes, bool wide_w, int parts, const RmsGradArgs &a)
{
    narrow_shape(a.width, [&](auto tpr, auto nc, auto kind) {
        constexpr int threads = tpr > 256 ? tpr : 256;
        if (wide_w)
            KLAUNCH_T(c, st, KID_RMS_GRAD, bytes, (k_rms_norm_grad<T, float, VEC, tpr, nc, kind>), (unsigned)parts, threads, a);
        else
            KLAUNCH_T(c, st, KID_RMS_GRAD, bytes, (k_rms_norm_grad<T, T, VEC, tpr, nc, kind>), (unsigned)parts, threads, a);
    });
}
static void weight_grad(he_ctx *c, hipStream_t st, double bytes, bool wide_w, const float *part, int parts, int width, void *dw)
{
    const unsigned grid = (unsigned)((width + 15) / 16);
    if (wide_w)
        KLAUNCH(c, st, KID_RMS_WEIGHT_GRAD, bytes, (k_rms_weight_grad<float>), grid, part, parts, width, (float *)dw);
    else
        KLAUNCH(c, st, KID_RMS_WEIGHT_GRAD, bytes, (k_rms_weight_grad<T>), grid, part, parts, width, (T *)dw);
}
static void quantize(he_ctx *c, hipStream_t st, double bytes, bool gelu, const Rows8Args &a)
{
    narrow_shape(a.width, [&](auto tpr, auto nc, auto kind) {
        by_rows<tpr>(a, [&](int threads, unsigned grid, const Rows8Args &part) {
            if (gelu)
                KLAUNCH_T(c, st, KID_QUANTIZE8, bytes, (k_quantize8<T, VEC, tpr, nc, kind, true>), grid, threads, part);
            else
                KLAUNCH_T(c, st, KID_QUANTIZE8, bytes, (k_quantize8<T, VEC, tpr, nc, kind, false>), grid, threads, part);
            bytes = 0.0;
        });
    });
}

#define NAME_(t) rows8_launch_##t
#define NAME(t) NAME_(t)
void NAME(HE_TYPE)(Rows8Launch &t)
{
    t.rms = rms;
    t.rms8 = rms8;
    t.rms_grad = rms_grad;
    t.weight_grad = weight_grad;
    t.quantize = quantize;
}
