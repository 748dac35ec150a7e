// How a linear layer is shared out: which form its kernel takes and what part of the layer a workgroup has.  Whole numbers alone, for the host and the kernel.
#pragma once

#include <stdint.h>

namespace hb {

constexpr uint32_t kDies = 8;

// Which form a layer takes: the one that costs least.  More rows and tiles of outputs in a workgroup use its digits and weights more often, and fewer fill
// the chip.  A form's time is first + (rounds of 256 workgroups, one for each compute unit) x round, in tenths of a us as measured at 4096 inputs in groups
// of 128; all of them grow alike with the inputs, and in groups of 32 to about twice as much.  us by form, for rows x (inputs -> outputs), the form taken
// in brackets:
//               rows, tiles a workgroup:   1, 1    2, 1    2, 2    2, 4    4, 4    4, 8    8, 8   8, 16
//    1 x (4096 -> 4096)                   [6.0]    7.4     7.8     9.3    12.6    19.8    30.3    41.6
//    2 x                                   9.8    [7.6]    8.1    10.0    12.8    19.8    30.4    41.7
//    4 x                                  17.3    10.4    [8.4]   10.2    13.2    20.5    31.1    42.2
//    8 x                                  31.4    17.3    14.4   [10.4]   13.2    20.4    32.1    43.2
//   16 x                                  58.8    29.5    26.4    18.5   [13.6]   20.4    32.1    43.2
//   32 x                                   115    53.4    50.4    34.9    24.8   [20.9]   32.3    43.5
//   64 x                                   240     114     103    69.4    49.9   [32.9]   35.7    47.2
//   16 x (4096 -> 16384)                   239     112     104    71.4    49.9   [34.0]   35.3    46.8
//   64 x                                   967     452     413     280     197     121     104   [97.3]
//   64 x, groups of 32                    1150     528     558     406     233     192     217    [169]
//    8 x (512 -> 512)                     [3.6]    4.2     4.0     4.2     5.0     5.6     7.8    10.5
// One row of many outputs (16384: 11.4 instead of 17.9) shares its digits among four tiles, but for groups of 32, whose scales take the registers of four steps
// (with two rows and two steps 16 instead of 22); up to 1024 inputs, four steps, it needs no sixteen wavefronts (512 -> 1000 4.0 instead of 4.5).
struct LinearForm {
    uint64_t rows, tiles, first, round;
};
constexpr int kLinearForms = 9;
constexpr LinearForm kLinearForm[kLinearForms] = {{1, 1, 23, 37}, {2, 1, 44, 31}, {2, 2, 24, 60}, {2, 4, 20, 83}, {4, 4, 13, 121}, {4, 8, 60, 143}, {8, 8, 125, 230},
                                                  {8, 16, 10, 480}, {1, 4, 44, 70}};

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
