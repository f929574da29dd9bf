// Which tiles a product of 8-bit rows and weights takes, by its sizes.
#pragma once
#include <cstdint>

struct Product8Plan {
    int tile, groups; // channels of a work-group and rows, but 256 rows with 192 channels; groups of waves that share its sums
    int64_t tiles;
};
// wide: results of 32 bits.  Rules go by the number of tiles.  Times in us with results in bf16, rows x width x channels: tiles of 256, 128, 64, of 64 with four groups;
//   16384 x 4096 x 4096 236, 281, 400, 582; 4096 x 4096 x 4096 63, 73, 112; 2048 x 4096 x 4096 50, 37, 54; 768 x 4096 x 4096 44, 24, 21; 16384 x 2048 x 768 30, 32, 43;
//   16384 x 768 x 768 15.8, 15.3, 21; 4096 x 768 x 2304 15, 14, 17; 4096 x 768 x 768 14, 6.9, 7.0; 1000 x 768 x 768 13, 5.9, 4.8, 4.9;
//   1000 x 4096 x 1024 42, 23, 13, 10; 512 x 4096 x 4096 43, 22, 17, 20.
// Of 64, of 64 with four groups, of 32 with four, of 16 with four and with eight:
//   1000 x 768 x 768 4.9, 5.1, 6.1; 300 x 2048 x 2048 7.9, 6.9, 7.7, 9.4; 500 x 768 x 768 4.7, 5.0, 4.2, 5.3; 200 x 8192 x 2000 22, 15, 12, 19; 64 x 4096 x 4096 12, 9.0, 6.2, 7.8;
//   8 x 8192 x 8192 33, 18, 11.8, 11.6; 16 x 1024 x 8192 5.2, 5.2, 3.7, 3.3; 100 x 8192 x 1024 20, 14, 7.0, 7.0, 7.3; 20 x 3000 x 3000 9.8, 7.7, 4.5, 4.2, 4.4;
//   32 x 8192 x 1024 20, 14, 6.7, 5.0, 4.6; 5 x 4861 x 1900 13, 9.8, 5.4, 4.1, 3.9; 23 x 768 x 768 4.6, 4.8, 3.5, 3.0, 3.1; 1 x 768 x 768 4.4, 4.7, 3.6, 2.9, 3.0.
// 256 rows by 192 channels, 256 and 128: 16384 x 2048 x 768 27, 29, 31; 4096 x 768 x 2304 14, 16, 15; 12500 x 4096 x 768 44, 52, 58; 13000 x 384 x 768 10.3, 12.0, 11.6;
//   16384 x 768 x 768 14, 16, 15; 16384 x 2048 x 1500 58, 68, 63; 16384 x 4096 x 2304 151, 163, 169; 9351 x 1536 x 2304 43, 49, 44; 8192 x 1024 x 2304 32, 36, 28;
//   16384 x 2048 x 3800 (5 rounds for 4) 146, 139, 158; 4007 x 1024 x 2048 17, 19, 12; 10000 x 768 x 768 12.5, 14.9, 11.0; of short sums in more rounds 8537 x 768 x 4096 47, 48, 43;
//   16384 x 768 x 2304 40, 44, 41 and with results in 32 bits 47, 53, 48.
// The same on another card, short sums in rounds that are full of tiles of 192, results of whole lines and not: 16384 x 768 x 2304 45, 50, 46 and 2300 channels 53, 56, 51;
//   16384 x 640 x 1536 29, 31, 29 and 1532 33, 34, 32; 32768 x 768 x 768 31, 34, 32 and 764 37, 37, 36; 8192 x 768 x 4608 45, 50, 50 and 4600 51, 55, 48; 16000 x 896 x 1536 34, 37, 44 and
//   1530 39, 39, 38; 48000 x 600 x 768 43, 47, 44 and 760 59, 54, 53; 8000 x 700 x 3008 34, 36, 34 and 3000 37, 38, 35; 16384 x 512 x 2304 38, 41, 38; 16384 x 1000 x 2304 54, 60, 56.
// 192: where they need no more rounds of the 256 CUs than tiles of 256, from two thirds of a round on, and tiles of 128 are more than two to a CU; more than one round only of long
// sums, or where the last one is full too and results are whole lines of 16 bits.  256: from three quarters of a round on.  Neither where sums are not long and the last round has few tiles (16384 x 768 x 2304, 2.25 rounds), or where edges leave an eighth
// more of the area empty than in tiles of 128 (65536 x 2048 x 64: 256 34, 128 23, 64 22), nor 256 for the shortest sums (16818 x 23 x 3078 38, 33).  128: from 0.8 tiles to a CU on (5284 x 768 x 768 7.4, 64 8.0; 3001 x 1000 x 1021 9.0, 8.1).
// 32 and 16: as long as two tiles to a CU are all there are.  Eight groups: a tile to a CU, and sums that are long enough for all.
inline Product8Plan product8_plan(int64_t rows, int32_t width, int32_t channels, bool wide)
{
    const auto tiles = [&](int m, int n) { return ((rows + m - 1) / m) * ((channels + n - 1) / n); };
    const auto rounds = [](int64_t t) { return (t + 255) / 256; };
    const int64_t t256 = tiles(256, 256), t192 = tiles(256, 192), t128 = tiles(128, 128), t64 = tiles(64, 64), t32 = tiles(32, 32), t16 = tiles(16, 16);
    const auto full = [&](int64_t t) { return t <= 256 || width >= 2048 || 10 * rounds(t) * 256 <= 13 * t; };
    const bool brim = width >= 512 && !wide && channels % 64 == 0 && 39 * rounds(t192) * 256 <= 40 * t192;
    if (t192 >= 176 && t128 > 512 && (t192 <= 256 || width >= 1024 || brim) && full(t192) && rounds(t192) == rounds(t256) && 8 * t192 <= 3 * t128) return {192, 1, t192};
    if (t256 >= 192 && width > 256 && full(t256) && 32 * t256 <= 9 * t128) return {256, 1, t256};
    if (t128 >= 205 && 32 * t128 <= 9 * t64) return {128, 1, t128};
    if (t16 <= 512) return {16, t16 <= 256 && width >= 2048 ? 8 : 4, t16};
    if (t32 <= 512) return {32, 4, t32};
    return {64, t64 <= 256 && width >= 1024 ? 4 : 1, t64};
}
