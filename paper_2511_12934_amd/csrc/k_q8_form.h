// Which kernel and which tile makes an 8-bit product (include/aif_q8.h: aif_q8_linear): by its sizes, type and end.
#pragma once
#include "aif_q8_dev.h"

namespace aif {

// few: k_q8_few, a block makes rows x cols of the result; else k_q8_many, a tile is that.
struct Q8Form {
    bool few;
    int rows, cols;
};

inline Q8Form q8_form(const Q8LinearCall &c, int n_cu)
{
    const bool gate = c.act == Q8_ACT_GATE;
    auto tiles_of = [&](int rows, int cols) { return ((int64_t)c.m + rows - 1) / rows * ((c.n + cols - 1) / cols); };
    auto rounds = [&](int rows, int cols, int units) { return (tiles_of(rows, cols) + units - 1) / units; };
    // Small tiles as long as no unit gets many: 16 mt rows of them by 16 columns (8-bit results: 16 by 128) take a unit about 0.07 mt us for 128 columns of k,
    // and a round of the large tiles takes 0.55 us (fp32: 0.95) for them however few the tiles are.  Large against small, us: 64 x 4096 x 4096 23.1 and
    // 12.1, 64 x 1024 x 8192 (8 by this count) 8.6 and 6.4, 768 x 1024 x 1024 (12) 8.9 and 8.8, 64 x 1024 x 16384 (16) 9.1 and 12.6; fp32 512 x 1024 x 1024 (8) 12.4 and
    // 7.1, 1000 x 1024 x 1024 (16) 12.9 and 12.9; gated with 8-bit results 256 x 1024 x 4096 (2 rounds) 14.5 and 11.3, 512 x 1024 x 4096 (4) 14.7 and 21.0.
    const int strip = c.out ? 16 : Q8_BLOCK;
    int mt = 1;                                                                  // as few rows as leave no unit two tiles
    while (c.out && mt < 4 && c.m > 16 * mt && tiles_of(16 * mt, strip) > n_cu) mt *= 2;
    if (rounds(16 * mt, strip, n_cu) * mt <= (!c.out ? 2 : c.f32 ? 12 : 8)) return {true, 16 * mt, strip};
    if (c.f32) return {false, 128, 128};
    // With a gate of 256 or 128 rows by 128 columns, one to a unit: 6000 x 1024 x 1024 (1, 2) 18.1 and 26.4, 10000 x 1024 x 1024 (2, 3) 30.5 and 34.7.
    if (gate) return {false, rounds(256, 128, n_cu) < rounds(128, 128, n_cu) ? 256 : 128, 128};
    // Tiles of 256 by 256, one to a unit, or of 128 by 128, two to one.  By what 31 sizes of 32 to 2500 large tiles took, each with up to 8192 columns of k and several
    // ends: with 0.5 us, a small tile's time for 128 columns of k with the unit to itself, as one, a small tile to each unit takes 1 + steps and a large one 4 + 2.2 steps,
    // with a bias 7 + 2.2 steps, with a residual or 8-bit results 10 + 2.2 steps, and a call with large ones 2 more (below, all by five).  Large against small, us, by columns of k:
    //   10000 x 1024 (160 large tiles)      256 12.2 and 10.8, 1024 18.8 and 18.7, 4096 44.9 and 55.8, 8192 85 and 132; in 8 bits 1024 23.0 and 22.2, 4096 49.4 and 59.5
    //   8192 x 1024 (128)                   256 12.1 and 8.9, 4096 45.0 and 39.8
    //   16384 x 1024 (256)                  256 13.0 and 13.1, 4096 57.8 and 85.5; with residual 256 19.9 and 17.7, 1024 27.0 and 27.8
    //   24576 x 1024 (384)                  256 19.8 and 17.1, 1024 33.1 and 34.7, 4096 100 and 128; in 8 bits 1024 42.4 and 38.3, 4096 107 and 130
    //   65536 x 1024 (1024)                 256 39.8 and 59.3; in 8 bits 256 55.3 and 51.3, 512 69.1 and 75.8
    //   with bias 10168 x 1752 (280)        1440 49.4 and 44.1; 39434 x 736 (465) 1368 53.2 and 63.7
    // On 16 other sizes, 48 calls, the choice takes 0.8 % more than the faster of both on average, 9 % at most.  The results are the same bits either way.
    const int64_t steps = (c.k + Q8_BLOCK - 1) / Q8_BLOCK, end = c.residual || !c.out ? 10 : c.bias ? 7 : 4;
    const bool large = rounds(256, 256, n_cu) * (5 * end + 11 * steps) + 10 <= 5 * rounds(128, 128, n_cu) * (1 + steps);
    return large ? Q8Form{false, 256, 256} : Q8Form{false, 128, 128};
}

}  // namespace aif
