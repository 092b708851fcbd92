// The paged attention's choice of kernel and key splits.  Host code only, so that it
// can be compiled and checked by itself.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace dcb {

struct PagedPlan {
    int rows, splits;   // query rows of a block (16, 64 or 128), blocks that share a row's keys
    int64_t ws_bytes;
};

// What a kernel costs: microseconds fitted to calls of 1 to 2,000 tokens over 30 to
// 60,000 others, 1 to 128 entries of 1 to 16 key heads and 1 to 8 query heads each,
// unsplit and in up to 64 splits (270 calls, 3,300 choices, in a graph; all but a few
// within a fifth).  A CU that has k of the blocks takes
//   base + tiles (own ceil(k / fit) + tile k) + round ceil(k / fit) + block k
// of its blocks' tiles (16 rows: of one wave's, a quarter), `fit` being fitted as the
// others are, not the blocks that a CU holds at once (three of 128 bf16 rows of 64,
// fitted as six), and with splits `join`, `part` for a megabyte of partial results and `split`
// for each.  By the fit's choice
// calls took 1.02 times their best choice on average; by rules (16 rows for up to 16,
// splits to fill the card) 1.15, and 4 at most.  Us of one call by choice (* the
// fit's), in blocks of 16, 64 and 128 rows, /splits:
//   entries tokens  heads     keys  width
//        1      1  15, 15    1,467    128 bf16   *11.7/12    ~20
//       71      1    8, 1   15,208    128 bf16   103.4/3   *100.9/6
//       10     33    5, 5    1,263    128 fp32    41.2/3    *36.6/8
//        7     18    2, 2    1,036    128 fp32   *15.6/8     63.5
//       23    110    2, 2      936     64 bf16    19.0      *16.5/4     32.7
//       14    384    1, 1    7,284     64 bf16               35.2/12   *36.7/8
//      114     39    8, 1    7,018    128 bf16              420.5/3   *315.3
struct PagedCost {
    int fit;
    double base, own, tile, round, block, join, part, split;
};
// Beside `join`: a part of what a second launch and a workspace take the host, 3.5 us.
constexpr double kSecondJoin = 1.5;
constexpr int kPagedRows[3] = {16, 64, 128};
constexpr PagedCost kPagedCost[3][2][2] = {   // [rows][128 wide][bf16]
    {{{2, 2.92, 0.808, 0.819, 0.0, 0.499, 2.94, 0.322, 0.0}, {1, 3.59, 1.047, 0.0, 0.511, 0.0, 2.99, 0.0, 0.017}},
     {{2, 2.05, 0.438, 2.167, 1.083, 0.708, 3.23, 0.170, 0.028}, {3, 2.95, 0.0, 2.146, 0.059, 1.542, 2.82, 0.0, 0.055}}},
    {{{4, 3.32, 1.299, 0.360, 0.0, 1.047, 2.90, 0.739, 0.020}, {4, 3.78, 0.572, 0.330, 0.182, 0.949, 3.11, 0.213, 0.029}},
     {{2, 2.91, 2.358, 0.526, 0.0, 2.26, 2.20, 0.903, 0.069}, {2, 2.29, 0.320, 0.966, 2.377, 1.273, 2.38, 0.230, 0.043}}},
    {{{}, {6, 5.64, 0.804, 0.419, 0.0, 1.909, 3.38, 0.213, 0.054}}, {{}, {2, 9.34, 1.115, 0.670, 0.0, 0.416, 1.44, 0.432, 0.0}}},
};

// n tokens of `group` rows each in each of `regions` (entries times key heads), over
// up to `limit` positions.
inline PagedPlan plan_paged(int D, int bf16, int64_t regions, int n, int group, int limit, int window, int sinks)
{
    const int64_t rows = (int64_t)n * group;
    PagedPlan best{64, 1, 0};
    double least = 0.0;
    bool any = false;
    for (int kind = 0; kind < 3; kind++) {
        const int rb = kPagedRows[kind], KT = kind == 0 ? (bf16 ? 32 : 16) : bf16 ? 64 : 32;
        if ((rb == 16 && rows > 256) || (rb == 128 && (!bf16 || rows <= 64))) continue;
        const PagedCost& c = kPagedCost[kind][D == 128][bf16 ? 1 : 0];
        const int64_t blocks = regions * ((rows + rb - 1) / rb);
        // a block's keys: its rows' windows, or (causal calls: of the middle rows) all before them
        int64_t keys = rows > rb ? limit - n / 2 : limit;
        if (window) keys = std::min(keys, (int64_t)sinks + window + std::min((int64_t)n, (int64_t)rb / group + 1) + 2 * KT);
        const double tiles = (double)((keys + KT - 1) / KT);
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 64}) {
            if (s > 1 && (keys < 64 * s || blocks * s > 6000)) break;
            double per = tiles / s;
            if (kind == 0) per = (double)(int64_t)(per / 4 + 0.999);   // (the waves' turns)
            const double k = (double)((blocks * s + 255) / 256), rounds = (double)(int64_t)((k + c.fit - 1) / c.fit);
            double us = c.base + per * (c.own * rounds + c.tile * k) + c.round * rounds + c.block * k;
            if (s > 1) us += c.join + kSecondJoin + c.part * (double)(regions * rows * s) * (D + 2) * 4e-6 + c.split * s;
            if (any && us >= least) continue;
            any = true;
            least = us;
            best = {rb, s, s > 1 ? regions * rows * s * (D + 2) * 4 : 0};
        }
    }
    return best;
}

}  // namespace dcb
