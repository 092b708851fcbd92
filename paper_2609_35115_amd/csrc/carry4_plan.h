// The attention operators' choice of kernel and key splits.  Host code only, so
// that it can be compiled and checked by itself.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace dcf {

// Which kernel an attention call takes, and over how many blocks its keys are
// split.  Us of a call in a graph, bf16, both sides of each border:
//   16 rows a block up to 16 rows, and for as many keys in all as a block of 832
//     on each CU visits, 1,500 up to 32 rows (40 rows, 64 regions, 540 keys: 8.2 and
//     11.1; 128 rows, 32 regions, 828 keys of 128: 12.1 and 15.3; 36 rows, 88
//     regions, 836 keys: 16.6 and 15.7; 24 rows, 256 regions, 724 keys 11.8 and
//     12.4, 6,024 keys 55 and 38; 20 rows, 600 regions, 6,020 keys of 128: 171 and 146); bf16 rows
//     of 64 up to 4,000,000 keys in all (one token, 1,500 keys, 2,048 regions: 51 and
//     51; 6,350, 840 regions 104 and 89; 10,000, 800 regions 158 and 136);
//   128 rows from 1.5 blocks a CU on, its own splits included, where that halves
//     the blocks nearly (16,384 rows, 4 regions, 4,100 keys of 128: 148, in 64-row
//     blocks 197, in 256-row ones 146; 101 rows, 215 regions, 3,230 keys: 73 and
//     82; 256 rows, 64 regions, 1,000 keys: 27 and 18; 776 rows, 13 blocks or 7 of 84
//     regions, 1,450 keys: 92 and 89; 192, three or two: 120 and 102); at width 64
//     only past 256 rows (1,000, 64 regions, 2,000 keys: 52 and 57; 200, 400
//     regions, 1,500 keys: 75 and 70);
//   splits: the join is a launch of its own, about 2 us, which grows with them.
//     16 rows: for a block a CU, of 128 keys or more (2,000 keys, 8 regions 8.4,
//     of 256 9.2, unsplit 16.9; 458 keys 7.2 unsplit, 8.1 split); all of two
//     blocks a CU where that leaves 448 (8,000 keys of 128, 32 regions 16.5, one a
//     CU 17.4; 19,000, 8 regions 15.8 and 14.0); from fewer than two
//     a CU, up to eight of 1,024 in 32 splits, so that a CU always holds its four
//     or five (17,400 keys, 200 regions 63 in ten, 85 in two, 116 unsplit; 7,600,
//     492 regions 65 in four, 72; but 5,200 of 128, 707 regions 105 in two, 100);
//     wider, 64 blocks or fewer: for a block a CU of 256 keys, or two of 1,024
//     (2,100 keys of 128, 32 regions of 128 rows 20.4 and, in two a CU, 25.5);
//     wider, more: by what a tile takes a CU that has k of the blocks, `fit` of them
//     at once, fitted to calls of 80 to 1,024 blocks and 1,800 and 4,500 keys in
//     one to four splits, all within a fifth but for a few (own: what one block
//     alone waits for; a second costs far less than the first), and the join's
//     bytes at 4 TB/s.  40 rows, 4,500 keys of 64: 260 regions 42 in four, 70
//     unsplit, 400 52 in three and 71, 1,024 unsplit 107, 111 in two; of 128: 260
//     70 and 107, 80 30 in six, 37 in three; 300 rows, 16,000 of 64, 40 regions 92
//     in four, 133 in two; but 56 rows, 458 keys, 256 regions 16.3 unsplit, 25.5 in two.
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
    // (three planes of 32 rows do not fit the registers)
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
