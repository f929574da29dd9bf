// How the rows of a width are laid over threads; T is the translation unit's element type.
#pragma once
#include "enc_launch.h"
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
    SHAPE(1024, 2)
    if constexpr (VEC * 1024 * 2 < NORM_MAX_WIDTH) { SHAPE(1024, 4) }
#undef SHAPE
}
