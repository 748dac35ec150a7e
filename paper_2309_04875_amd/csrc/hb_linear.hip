// C ABI of the linear layer: argument checks, launch on the caller's stream.
#include "hb_check.hpp"
#include "hb_linear.hpp"

namespace {

template <int TM, int RT, int WN, int WK, int P, int FLUSH>
hipError_t go(hb::LinearArgs &a, hipStream_t stream)
{
    const uint64_t tiles = ((uint64_t)a.outs + 16 * WN * RT - 1) / (16 * WN * RT);
    a.row_tiles = (a.rows + TM - 1) / TM;
    const uint64_t blocks = (tiles + hb::kDies - 1) / hb::kDies * hb::kDies * a.row_tiles;
    if (blocks > 0xffffffffull / (64 * WN * WK)) return hipErrorInvalidConfiguration;     // a grid has fewer than 2^32 threads
    hipLaunchKernelGGL((hb::linear_q4_kernel<TM, RT, WN, WK, P, FLUSH>), dim3((unsigned)blocks), dim3(64 * WN * WK), 0, stream, a);
    return hipGetLastError();
}

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
struct Form {
    uint64_t rows, tiles, first, round;
};
constexpr Form kForms[] = {{1, 1, 23, 37}, {2, 1, 44, 31}, {2, 2, 24, 60}, {2, 4, 20, 83}, {4, 4, 13, 121}, {4, 8, 60, 143}, {8, 8, 125, 230},
                           {8, 16, 10, 480}, {1, 4, 44, 70}};

template <int FLUSH>
hipError_t by_shape(hb::LinearArgs &a, hipStream_t stream)
{
    const uint64_t tiles = ((uint64_t)a.outs + 15) / 16;
    int best = 0;
    uint64_t least = ~0ull;
    for (int i = 0; i < (FLUSH == 32 ? 8 : 9); ++i) {
        const Form &f = kForms[i];
        const uint64_t blocks = (a.rows + f.rows - 1) / f.rows * ((tiles + f.tiles - 1) / f.tiles), cost = f.first + (blocks + 255) / 256 * f.round;
        if (cost < least) least = cost, best = i;
    }
    if constexpr (FLUSH != 32) {
        if (best == 8) return go<1, 1, 4, 4, 4, FLUSH>(a, stream);
    }
    switch (best) {
    case 0: return a.in <= 4 * hb::kLinearStep ? go<1, 1, 1, 4, 1, FLUSH>(a, stream) : go<1, 1, 1, 16, 1, FLUSH>(a, stream);
    case 1: return go<2, 1, 1, 8, 1, FLUSH>(a, stream);
    case 2: return go<2, 1, 2, 8, 1, FLUSH>(a, stream);
    case 3: return go<2, 1, 4, 4, 2, FLUSH>(a, stream);
    case 4: return go<4, 1, 4, FLUSH == 32 ? 2 : 4, 1, FLUSH>(a, stream);      // (scaling every 32 inputs takes more registers than sixteen wavefronts leave)
    case 5: return go<4, 1, 8, 1, 2, FLUSH>(a, stream);
    case 6: return go<8, 1, 8, 1, 1, FLUSH>(a, stream);
    default: return go<8, 2, 8, 1, 1, FLUSH>(a, stream);
    }
}

hipError_t launch(hb::LinearArgs &a, uint64_t group, hipStream_t stream)
{
    if (group % 128 == 0) return by_shape<128>(a, stream);
    if (group % 64 == 0) return by_shape<64>(a, stream);
    return by_shape<32>(a, stream);
}

}  // namespace

extern "C" int hb_linear_q4(const int64_t *x0, const int64_t *x1, size_t rows, size_t in, size_t out, const uint8_t *weight,
                            const int32_t *scales, int group, int frac, uint64_t seed, int64_t *out0, int64_t *out1,
                            uint64_t *opened_bits, void *stream)
{
    if (group < 32 || group % 32 != 0 || frac < 1 || frac > 31) return HB_EINVAL;
    if (in == 0 || in > HB_LINEAR_MAX_IN || out > HB_LINEAR_MAX || rows > HB_LINEAR_MAX) return HB_EINVAL;
    const size_t groups = (in + group - 1) / group, row_bytes = (in + 1) / 2;
    if (rows != 0 && out != 0) {
        const size_t sizes[6] = {8 * rows * in, 8 * rows * in, 8 * rows * out, 8 * rows * out, out * row_bytes, 4 * out * groups};
        const void *ptrs[6] = {x0, x1, out0, out1, weight, scales};
        const unsigned align[6] = {8, 8, 8, 8, 1, 4};
        int st = hb::check_buffers(ptrs, sizes, align, 6);
        if (st != HB_OK) return st;
        // outputs overlap nothing: other workgroups still read the inputs
        if (!hb::outputs_disjoint(ptrs, sizes, 6, 2, 4)) return HB_EINVAL;
        const uint64_t a_group = (size_t)group < in ? group : (in + 127) / 128 * 128;      // one group: the last step's end is in it
        hb::LinearArgs a = {};
        a.x[0] = (const uint64_t *)x0;
        a.x[1] = (const uint64_t *)x1;
        a.out[0] = (uint64_t *)out0;
        a.out[1] = (uint64_t *)out1;
        a.weight = weight;
        a.scales = scales;
        a.seedA = hb::stream_word(seed, 1);
        a.rows = (uint32_t)rows;
        a.in = (uint32_t)in;
        a.outs = (uint32_t)out;
        a.groups = (uint32_t)groups;
        a.frac = frac;
        a.weight_bytes = out * row_bytes;
        a.group_inverse = ((1ull << 40) + a_group - 1) / a_group;
        const hipError_t e = launch(a, a_group, (hipStream_t)stream);
        if (e != hipSuccess) return hb::fail_hip(e, "kernel launch");
    }
    if (opened_bits) *opened_bits = 64ull * rows * out;
    return HB_OK;
}
