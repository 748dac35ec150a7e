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
    if (blocks > 0x7fffffffull) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((hb::linear_q4_kernel<TM, RT, WN, WK, P, FLUSH>), dim3((unsigned)blocks), dim3(64 * WN * WK), 0, stream, a);
    return hipGetLastError();
}

// Which form a layer takes: the one whose rounds of 256 workgroups, one for each compute unit, cost least.  More rows and tiles of outputs in a
// workgroup use its digits and weights more often, and fewer fill the chip.  A round's time in tenths of a us, measured at 4096 inputs in
// groups of 128; all of them grow alike with the inputs, and in groups of 32 to about 2.5 times as much.  us by form, for rows x (inputs ->
// outputs), the form taken in brackets:
//               rows, tiles a workgroup:   1, 1    2, 1    2, 2    2, 4    4, 4    8, 4    8, 8
//    1 x (4096 -> 4096)                   [6.1]    7.1     8.9    12.7    14.3    21.2    32.3
//    2 x                                   9.8    [7.9]    9.5    13.4    14.8    21.2    32.3
//    4 x                                  16.7    11.8   [10.0]   13.7    16.1    21.6    32.9
//    8 x                                  29.7    20.3    17.9   [14.6]   16.6    23.6    32.7
//   16 x                                  56.8    35.0    32.7    26.5   [17.8]   24.3    33.5
//   32 x                                   110    63.3    61.9    48.6    32.1   [25.4]   34.5
//   64 x                                   219     122     122    94.9    59.2    48.1   [37.3]
//   64 x (4096 -> 16384)                   886     494     503     384     240     187    [116]
//    8 x (512 -> 512)                      3.8    [4.1]    3.9     3.9     4.9     6.3     8.0
// Eight rows by sixteen tiles, with groups of 128, halve the digits to be made and read for each weight, at two wavefronts a SIMD for four: from two rounds of
// the last on they are 4 to 11 % faster (64 x (4096 -> 16384) 109 for 113, 128 x (4096 -> 4096) 51 for 58, 512 x (1024 -> 2048) 37 for 41, but
// 64 x (4096 -> 4096) 50 for 36).  Scaling every 64 or 32 inputs takes the registers of the second tile.
// One row of many outputs (16384: 13.1 instead of 17.7) shares its digits among four tiles; up to 1024 inputs, four steps, it needs no sixteen
// wavefronts (512 -> 1000 4.0 instead of 4.5).
struct Form {
    uint64_t rows, tiles, round;
};
constexpr Form kForms[] = {{1, 1, 38}, {2, 1, 41}, {2, 2, 75}, {2, 4, 120}, {4, 4, 143}, {8, 4, 227}, {8, 8, 345}, {1, 4, 105}, {8, 16, 540}};

template <int FLUSH>
hipError_t by_shape(hb::LinearArgs &a, hipStream_t stream)
{
    const uint64_t tiles = ((uint64_t)a.outs + 15) / 16;
    int best = 0;
    uint64_t least = ~0ull;
    for (int i = 0; i < (int)(sizeof(kForms) / sizeof(kForms[0])); ++i) {
        const Form &f = kForms[i];
        if (f.tiles == 16 && FLUSH != 128) continue;
        const uint64_t blocks = (a.rows + f.rows - 1) / f.rows * ((tiles + f.tiles - 1) / f.tiles), cost = (blocks + 255) / 256 * f.round;
        if (cost < least) least = cost, best = i;
    }
    switch (best) {
    case 0: return a.in <= 4 * hb::kLinearStep ? go<1, 1, 1, 4, 1, FLUSH>(a, stream) : go<1, 1, 1, 16, 1, FLUSH>(a, stream);
    case 1: return go<2, 1, 1, 8, 1, FLUSH>(a, stream);
    case 2: return go<2, 1, 2, 8, 1, FLUSH>(a, stream);
    case 3: return go<2, 1, 4, 4, 2, FLUSH>(a, stream);
    // (eight wavefronts where scaling every 32 inputs takes more registers than sixteen leave: 16 x (4096 -> 4096) 39 instead of 58)
    case 4: return go<4, 1, 4, FLUSH == 32 ? 2 : 4, 1, FLUSH>(a, stream);
    case 5: return go<8, 1, 4, 2, 1, FLUSH>(a, stream);
    case 6: return go<8, 1, 8, 1, 1, FLUSH>(a, stream);
    case 8:
        if constexpr (FLUSH == 128) return go<8, 2, 8, 1, 1, FLUSH>(a, stream);
        [[fallthrough]];
    default: return go<1, 1, FLUSH == 32 ? 1 : 4, FLUSH == 32 ? 16 : 4, FLUSH == 32 ? 1 : 4, FLUSH>(a, stream);
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
