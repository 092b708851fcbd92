// The matrix product's choice of kernel and of splits of K.  Host code only, so that
// it can be compiled and checked by itself.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace dcb {

// Beside what the second launch of a split call takes the device: what it and its
// workspace take the host of a call outside a graph is about 3.5 us, of which this counts a part.
constexpr double kSecondLaunch = 1.5;

enum LinearKind { kFew16, kFew32, kTile64, kTile128, kTile256, kPlane64, kPlane128, kPlane256, kRing128, kLinearKinds };

// A kernel's block, and what it costs: microseconds fitted to calls of 1 to 20,000
// rows, n_in and n_out from 16 to 8,192, in one to eight splits each (110 sizes, 900
// calls in a graph over buffers past the caches; most within a tenth, all within 0.6
// to 1.3).  A CU that has k of the blocks takes
//   base + steps (own ceil(k / fit) + step k) + round ceil(k / fit) + block k,
// `fit` being fitted as the others are, not counted (one 256 x 256 block fills a CU's
// LDS, and calls of up to four a CU fit best as one round), a step 128 bytes of a row
// (few rows: 256, the four waves' together), `out` for a megabyte of the result, and
// with splits `join` and `part` for a megabyte of partial sums.  By the fit's choice calls of more than 32 rows took 1.01 times
// their best choice on average, and 1.16 at most; by rules on the number of blocks
// (at least 192 of the largest tile) 1.07 and 1.83.  Us of one call by choice
// (* the fit's), in 64 x 64, 128 x 128, 128 x 128 through the longer ring (one block
// a CU) and 256 x 256 tiles, bf16, /splits:
//     128 x 4,096 -> 8,192    *25.0     30.0/4    26.4/4    37.9/4
//     512 x 4,096 -> 8,192     66.1     56.2/2   *43.9      55.6/4
//   1,024 x 1,024 -> 1,024     *8.1     16.6      13.2      26.2/2
//   2,048 x 2,048 -> 2,048     29.7     27.9     *23.0      42.7/2
//  14,336 x   512 -> 2,048     74.7     51.2      62.5     *45.1
//  14,336 x 2,048 ->   512     59.3    *41.1      46.5      54.7/2
//   4,096 x 4,096 -> 4,096    228.4    140.0     161.5    *113.6
// and few rows' kernel against 64 x 64 tiles
//      16 x 4,096 -> 8,192    *20.0     20.4/4
//      32 x 4,096 -> 8,192     28.4    *21.6/4
//      32 x 2,048 ->   512     *7.3/4    8.6/4
struct LinearCost {
    int bm, bn, fit;
    double base, own, step, round, block, join, part, out;
};
constexpr LinearCost kLinearCost[2][kLinearKinds] = {
    {   // fp32 (tiles: three bf16 planes)
        {16, 16, 8, 2.51, 0.030, 0.220, 0.0, 0.066, 2.96, 2.59, 0.0},
        {32, 16, 2, 3.06, 0.0, 0.389, 0.0, 0.0, 2.88, 1.52, 0.0},
        {}, {}, {},
        {64, 64, 3, 3.11, 0.415, 0.255, 0.0, 0.71, 3.59, 0.229, 0.076},
        {128, 128, 2, 3.20, 0.0, 1.132, 0.0, 1.92, 3.23, 0.413, 0.247},
        {256, 128, 1, 3.67, 1.860, 0.0, 0.0, 3.45, 2.71, 0.393, 0.199},
        {},
    },
    {   // bf16
        {16, 16, 4, 2.65, 0.0, 0.206, 0.0, 0.028, 2.85, 1.59, 0.0},
        {32, 16, 4, 2.94, 0.0, 0.339, 0.0, 0.0, 2.94, 0.85, 0.0},
        {64, 64, 2, 2.64, 0.086, 0.170, 0.40, 0.92, 3.28, 0.247, 0.017},
        {128, 128, 2, 4.30, 0.339, 0.322, 2.16, 0.0, 1.93, 0.339, 0.177},
        {256, 256, 4, 0.0, 0.0, 1.296, 4.91, 4.49, 1.79, 0.336, 0.176},
        {}, {}, {},
        {128, 128, 1, 3.10, 0.494, 0.0, 1.535, 0.0, 2.88, 0.385, 0.354},
    },
};

// Columns of a block: with glu, half as many and their factors (few rows: as many).
constexpr int linear_columns(int kind, int bn, int glu) { return glu && kind > kFew32 ? bn / 2 : bn; }

// A row of partial sums: columns padded to eight, with glu the factors behind them.
constexpr int part_half(int N) { return (N + 7) / 8 * 8; }
constexpr int64_t part_row(int N, int glu) { return (int64_t)part_half(N) * (glu ? 2 : 1); }

struct LinearPlan {
    int kind, splits;
    int64_t ws_bytes;
};

// M rows, n_in K, n_out N.
inline LinearPlan plan_linear(int64_t M, int N, int K, int glu, int bf16)
{
    const int64_t row = (int64_t)K * (bf16 ? 2 : 4);   // bytes
    LinearPlan best{kFew16, 1, 0};
    double least = 0.0;
    bool any = false;
    const int first = M <= 16 ? kFew16 : M <= 32 ? kFew32 : bf16 ? kTile64 : kPlane64;
    for (int kind = first; kind < kLinearKinds; kind++) {
        const LinearCost& c = kLinearCost[bf16 ? 1 : 0][kind];
        if (c.bm == 0 || (M <= 16 && kind != kFew16)) continue;
        if ((kind == kTile256 || kind == kRing128) && K % 8 != 0) continue;   // (rows of whole chunks only)
        const int64_t bc = linear_columns(kind, c.bn, glu), tiles = (M + c.bm - 1) / c.bm * ((N + bc - 1) / bc);
        const int64_t unit = kind <= kFew32 ? 256 : 128, steps = (row + unit - 1) / unit;
        for (int s : {1, 2, 3, 4, 6, 8}) {
            if (s > 1 && (steps < 2 * s || tiles * s > 4096)) break;
            const double k = (double)((tiles * s + 255) / 256), rounds = (double)(int64_t)((k + c.fit - 1) / c.fit);
            const double wide = kind <= kFew32 && glu ? 2.0 : 1.0;   // (a block of few rows has the factors besides)
            double us = c.base + (double)steps / s * (c.own * rounds + c.step * k * wide) + c.round * rounds + c.block * k +
                        c.out * (double)M * N * (bf16 ? 2e-6 : 4e-6);
            if (s > 1) us += c.join + kSecondLaunch + c.part * (double)(M * part_row(N, glu) * s) * 4e-6;
            if (any && us >= least) continue;
            any = true;
            least = us;
            best = {kind, s, s > 1 ? s * M * part_row(N, glu) * 4 : 0};
        }
    }
    return best;
}

}  // namespace dcb
