// The attention operators' choice of kernel and key splits.  Host code only, so
// that it can be compiled and checked by itself.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace dcf {

// Which kernel an attention call takes, and over how many blocks its keys are
// split.  Us of a call in a graph, bf16, one window for the whole call (c: causal, a
// window of as many keys), in blocks of 16, 64 and 128 rows; behind a slash the
// splits, the best of one to eight and of what fills the card.  * marks the one that
// the rules take, with their splits, and the last column is that kernel unsplit.
//
// regions    rows     keys  width     16        64       128      unsplit
//       8       1    2,000     64     *8.2/15     9.2/8               16.5
//       8       1   19,000     64    *11.3/32   12.4/64              121.8
//     200       1   17,400     64    *60.1/10   60.7/10              113.8
//     256       1    2,000     64     *17.9/2    17.6/4               18.4
//     492       1    7,600     64     *64.7/4    64.2/6               72.2
//   2,048       1    1,500     64       *54.6      51.5
//     256      24      724     64       *12.1      12.3
//      64      40      540     64        *8.2     9.9/4
//      32       1    8,000    128    *15.9/16   18.6/16               72.9
//     707       1    5,200    128      *107.5     125.4
//     800       1   10,000    128      *246.3   256.2/6
//      32     128      828    128       *13.6    14.9/4    17.6/4
//     800       4   10,000     64     137.1/4  *135.8/8              155.7
//     840       4    6,350     64      95.3/4   *91.7/3              102.3
//     256      24    6,024     64      55.0/3   *37.9/5               71.3
//      88      36      836     64        13.0   *12.5/3               13.7
//     260      40    4,500     64      67.7/4   *43.1/4               70.4
//     400      40    4,500     64      91.9/4   *54.1/3               71.4
//   1,024      40    4,500     64       225.1    *122.4
//     256      56      458     64        13.7     *10.3
//     400     200    1,500     64       124.4     *67.3      69.2
//      40     300   16,000     64               *93.0/6    91.2/6    195.2
//     400     300    1,500     64                 *82.6      83.8
//     600      20    6,020    128       184.1  *146.9/5              175.0
//      80      40    4,500    128      35.3/3   *29.3/6               74.7
//     260      40    4,500    128      92.8/3   *70.4/5              107.7
//      32     128    2,100    128      24.0/2   *20.1/4    23.7/6     37.3
//      64     256    1,000    128                 *21.4    29.1/4
//      84     776    1,450    128                 *89.2      88.0
//      64   1,000    2,000     64                  62.8     *54.3
//     215     101    3,230    128       110.1    82.2/4   *75.0/2     81.3
//       4  16,384    4,096c   128                 225.0    *153.0
//
// (800 regions over 10,000 keys of 128 would take 200.9 in six.)  Keys are counted for
// the whole call; a causal block visits its own rows' window only, so a call much
// longer than its window is counted with too many.
//
//   16 rows up to 16 rows, and for as many keys in all as a block of 832 on each CU
//     visits, 1,500 up to 32 rows; bf16 rows of 64 up to 4,000,000 keys in all;
//   128 rows from 1.5 blocks a CU on, its own splits included, where that nearly
//     halves the blocks; at width 64 only past 256 rows.  Blocks of 256 rows gained
//     2% on the longest and lost 20% on calls of 200;
//   splits: the join is a launch of its own, about 2 us, which grows with them.
//     16 rows: for a block a CU, of 128 keys or more, all of two blocks a CU where
//     that leaves 448; from fewer than two a CU, up to eight of 1,024 in 32
//     splits, so that a CU always holds its four or five;
//     wider, 64 blocks or fewer: for a block a CU of 256 keys, or two of 1,024;
//     wider, more: by what a tile takes a CU that has k of the blocks, `fit` of them
//     at once, fitted to calls of 80 to 1,024 blocks and 1,800 and 4,500 keys in
//     one to four splits, all within a fifth but for a few (own: what one block
//     alone waits for; a second costs far less than the first), and the join's
//     bytes at 4 TB/s.
struct Plan4 {
    int rows;     // query rows of a block: 16 (one set for four waves), 64 or 128 (16 or 32 a wave)
    int splits;
};

// n tokens of `group` rows each, in each of `regions` (entries times key heads).
inline Plan4 plan4(int D, int sinks, int ring, int64_t regions, int n, int group, int window, bool bf16)
{
    const int64_t rows = (int64_t)n * group;
    const int64_t most = (int64_t)sinks + (window < ring ? window : ring) + n;   // keys of a list
    const int64_t in16 = regions * ((rows + 15) / 16), in64 = regions * ((rows + 63) / 64),
                  in128 = regions * ((rows + 127) / 128);
    // the most splits that make up to `blocks` blocks of `of` and leave each `keys` keys or more
    auto split = [&](int64_t of, int64_t blocks, int64_t keys) { return std::max((int64_t)1, std::min(blocks / of, most / keys)); };
    const bool few = rows <= 16 && (!bf16 || D == 128 || in16 * most <= 4000000);
    if (few || in16 * most <= 256 * (rows <= 32 ? 1500 : 832)) {
        const int64_t two = 512 / in16;
        const int64_t s = std::max(most < 640 ? 1 : split(in16, 256, 128), in16 > 512 ? 1 : std::min((int64_t)32, split(in16, 2048, 1024)));
        return {16, (int)(two * 448 <= most ? std::max(two, s) : s)};
    }
    // (three planes of 32 fp32 rows do not fit the registers)
    const bool wide = bf16 && rows > (D == 64 ? 256 : 96) && 8 * in64 >= 15 * in128 && in128 * split(in128, 512, 1024) >= 384;
    // a tile takes a CU with k blocks us (own ceil(k / fit) + k) microseconds
    const double us = D == 64 ? (wide ? 0.40 : 0.23) : wide ? 0.62 : 0.48;
    const double own = D == 64 ? (wide ? 1.2 : 2.4) : wide ? 1.5 : 1.25;
    const int64_t fit = (D == 64 ? 5 : 3) - (wide ? (D == 64 ? 2 : 1) : 0), blocks = wide ? in128 : in64;
    if (blocks <= 64) return {wide ? 128 : 64, (int)std::max(split(blocks, 256, 256), split(blocks, 512, 1024))};
    int best = 1;
    double least = 0.0;
    // (of very many blocks, splits balance the last few only, and could pass a launch's 2^24)
    for (int s = 1; s <= 8 && (s == 1 || (most >= 256 * s && blocks * s <= 1 << 20)); s++) {
        const int64_t k = (blocks * s + 255) / 256;
        double cost = us * (own * (double)((k + fit - 1) / fit) + (double)k) * (double)(most / 64 + 1) / s;
        if (s > 1) cost += 2.0 + (double)(regions * rows * s) * (D + 2) * 2e-6;   // the join, and its 8 bytes a value
        if (s > 1 && cost >= least) continue;
        best = s;
        least = cost;
    }
    return {wide ? 128 : 64, best};
}

}  // namespace dcf
