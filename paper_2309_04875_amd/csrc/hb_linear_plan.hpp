// How a linear layer is shared out: which form its kernel takes and what part of the layer a workgroup has.  Whole numbers alone, for the host and the kernel.
#pragma once

#include <stdint.h>

namespace hb {

constexpr uint32_t kDies = 8;

// Which form a layer takes: the one that costs least.  More rows and tiles of outputs in a workgroup use its digits and weights more often, and fewer fill
// the chip.  A form's time is first + (rounds of 256 workgroups, one for each compute unit) x round, in tenths of a us as measured at 4096 inputs in groups
// of 128; all of them grow alike with the inputs, and in groups of 32 to about twice as much.  us by form, for rows x (inputs -> outputs), the form taken
// in brackets (one call after the other in a graph, with weights that no cache holds yet):
//               rows, tiles a workgroup:   1, 1    2, 1    2, 2    2, 4    4, 4    4, 8    8, 8   8, 16    1, 4
//    1 x (4096 -> 4096)                   [5.8]    7.1     7.6     9.2    12.5    19.8    30.8    42.3     8.7
//    2 x                                   9.5    [7.5]    8.0    10.0    12.6    19.8    30.7    42.5     8.8
//    4 x                                  16.9    10.2    [8.2]   10.0    13.0    20.4    31.3    43.0     9.3
//    8 x                                  31.3    17.2    14.3   [10.3]   13.0    20.3    31.8    43.8    16.8
//   16 x                                  59.2    29.4    26.3    18.6   [13.5]   20.4    32.0    43.3    30.9
//   32 x                                   115    53.9    50.7    35.1    24.9   [21.1]   32.2    43.5    57.1
//   64 x                                   237     112     103    70.2    50.3   [33.3]   35.7    47.0     114
//   16 x (4096 -> 16384)                   234     112     104    71.8    49.3   [34.6]   35.6    46.8     118
//   64 x                                   957     446     414     283     199     124     106   [95.2]    457
//   64 x, groups of 32                    1138     535     556     405     234     195     217   [169]
//    1 x                                  18.2    17.2    15.1    11.8    13.7    21.1    31.1    44.4   [11.3]
//    1 x (4096 -> 32768)                  34.8    31.2    30.1    24.5    28.0    23.0    32.3    44.9   [22.2]
//    1 x (4096 -> 65536)                  66.5    58.2    55.5    45.3    50.2   [35.5]   48.4    47.4    40.5
//    3 x (4096 -> 5000)                                   14.1    10.1            20.0                    [9.0]
//    8 x (512 -> 512)                     [3.6]    4.2     4.0     4.2     4.9     5.6     7.8    10.4     4.1
// The last form, one row that shares its digits among four tiles, is none for groups of 32, whose scales take the registers of four steps (with two rows and
// two steps 16 instead of 22).  Up to 1024 inputs, four steps, one tile a workgroup needs no sixteen wavefronts (512 -> 1000 4.0 instead of 4.5).
struct LinearForm {
    uint64_t rows, tiles, first, round;
};
constexpr int kLinearForms = 9;
constexpr LinearForm kLinearForm[kLinearForms] = {{1, 1, 23, 37}, {2, 1, 44, 31}, {2, 2, 24, 60}, {2, 4, 20, 83}, {4, 4, 13, 121}, {4, 8, 60, 143}, {8, 8, 125, 230},
                                                  {8, 16, 10, 480}, {1, 4, 19, 83}};

// Workgroups: a tile of rows by a group of outputs each.
constexpr uint64_t linear_row_tiles(const LinearForm &f, uint64_t rows) { return (rows + f.rows - 1) / f.rows; }
constexpr uint64_t linear_groups(const LinearForm &f, uint64_t outs) { return ((outs + 15) / 16 + f.tiles - 1) / f.tiles; }

// flush: inputs that go into one sum before it is scaled (128, 64 or 32).
constexpr int linear_form(int flush, uint64_t rows, uint64_t outs)
{
    int best = 0;
    uint64_t least = ~0ull;
    for (int i = 0; i < (flush == 32 ? kLinearForms - 1 : kLinearForms); ++i) {
        const LinearForm &f = kLinearForm[i];
        const uint64_t blocks = linear_row_tiles(f, rows) * linear_groups(f, outs), cost = f.first + (blocks + 255) / 256 * f.round;
        if (cost < least) least = cost, best = i;
    }
    return best;
}

// Which of `count` (group, tile of rows) pairs, a group's side by side, workgroup `block` has.  Workgroups go to the eight dies in turn, and each die gets
// an eighth of the pairs one after the other: a group's weights are read into one die's cache, or into those of the few that share its rows, and no die
// has more than one pair more than another.  (Where whole groups went to dies, layers of fewer groups than dies left dies idle: 2048 x (4096 -> 1024)
// 198 us for 374, 2048 x (4096 -> 256) 52 for 370, 2048 x (4096 -> 128) 37 for 224, 48 x (1000 -> 640) 6.4 for 10.4; 64 x (4096 -> 16384) 103 and 106.)
constexpr uint32_t linear_pair(uint32_t block, uint32_t count)
{
    const uint32_t die = block % kDies, more = count % kDies;
    return die * (count / kDies) + (die < more ? die : more) + block / kDies;
}

// Tiles of rows that one launch takes, three at least: a grid has fewer than 2^32 threads, and what is more goes into further launches.
constexpr uint64_t linear_launch_tiles(uint64_t groups, uint64_t threads) { return 0xffffffffull / threads / groups; }

}  // namespace hb
