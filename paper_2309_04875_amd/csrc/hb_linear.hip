// C ABI of the linear layer: argument checks, launch on the caller's stream.
#include "hb_check.hpp"
#include "hb_linear.hpp"

namespace {

template <int TM, int RT, int WN, int WK, int P, int FLUSH>
hipError_t go(hb::LinearArgs &a, hipStream_t stream)
{
    constexpr hb::LinearForm form{TM, WN * RT, 0, 0};
    constexpr uint64_t threads = 64 * WN * WK;
    const uint64_t tiles = hb::linear_row_tiles(form, a.rows), groups = hb::linear_groups(form, a.outs), most = hb::linear_launch_tiles(groups, threads);
    for (uint64_t first = 0; first < tiles; first += most) {
        a.first_tile = (uint32_t)first;
        a.row_tiles = (uint32_t)(tiles - first < most ? tiles - first : most);
        a.pairs = (uint32_t)(groups * a.row_tiles);
        hipLaunchKernelGGL((hb::linear_q4_kernel<TM, RT, WN, WK, P, FLUSH>), dim3(a.pairs), dim3((unsigned)threads), 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int FLUSH>
hipError_t by_shape(hb::LinearArgs &a, hipStream_t stream)
{
    const int best = hb::linear_form(FLUSH, a.rows, a.outs);
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
