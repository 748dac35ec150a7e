// C ABI of the linear layer: argument checks, launch on the caller's stream.
#include "hb_check.hpp"
#include "hb_linear.hpp"

extern "C" int hb_linear_q4(const int64_t *x0, const int64_t *x1, size_t rows, size_t in, size_t out, const uint8_t *weight,
                            const int32_t *scales, int group, int frac, uint64_t seed, int64_t *out0, int64_t *out1,
                            uint64_t *opened_bits, void *stream)
{
    if (group < 32 || group % 32 != 0 || frac < 1 || frac > 31) return HB_EINVAL;
    if (in == 0 || in > HB_LINEAR_MAX || out > HB_LINEAR_MAX || rows > HB_LINEAR_MAX) return HB_EINVAL;
    const size_t groups = (in + group - 1) / group, row_bytes = (in + 1) / 2;
    if (rows != 0 && out != 0) {
        const size_t sizes[6] = {8 * rows * in, 8 * rows * in, 8 * rows * out, 8 * rows * out, out * row_bytes, 4 * out * groups};
        const void *ptrs[6] = {x0, x1, out0, out1, weight, scales};
        const unsigned align[6] = {8, 8, 8, 8, 1, 4};
        int st = hb::check_buffers(ptrs, sizes, align, 6);
        if (st != HB_OK) return st;
        // outputs overlap nothing: other workgroups still read the inputs
        if (!hb::outputs_disjoint(ptrs, sizes, 6, 2, 4)) return HB_EINVAL;
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
        a.group = group;
        a.frac = frac;
        const uint64_t per = hb::kLinearBlock / 64, blocks = ((uint64_t)rows * out + per - 1) / per;
        if (blocks > 0x7fffffffull) return HB_EINVAL;
        hipLaunchKernelGGL(hb::linear_q4_kernel, dim3((unsigned)blocks), dim3(hb::kLinearBlock), 0, (hipStream_t)stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hb::fail_hip(e, "kernel launch");
    }
    if (opened_bits) *opened_bits = 64ull * rows * out;
    return HB_OK;
}
