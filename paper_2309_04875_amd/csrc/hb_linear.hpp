// Matrix-vector products of shared activations with public 4-bit weights and group scales.
#pragma once

#include "hb_fixed.hpp"

namespace hb {

struct LinearArgs {
    const uint64_t *x[2];       // [rows][in]
    uint64_t *out[2];           // [rows][out]
    const uint8_t *weight;      // [out][(in + 1) / 2]
    const int32_t *scales;      // [out][groups]
    uint64_t seedA;
    uint32_t rows, in, outs, groups;
    int group, frac;
};

constexpr int kLinearBlock = 256;

// One wavefront per output number, lanes over the inputs.
__global__ void __launch_bounds__(kLinearBlock)
linear_q4_kernel(LinearArgs a)
{
    const uint64_t i = (uint64_t)blockIdx.x * (kLinearBlock / 64) + threadIdx.x / 64;
    if (i >= (uint64_t)a.rows * a.outs) return;
    const uint32_t row = (uint32_t)(i / a.outs), n = (uint32_t)(i % a.outs), lane = threadIdx.x % 64;
    const uint8_t *w = a.weight + (uint64_t)n * ((a.in + 1) / 2);
    const int32_t *s = a.scales + (uint64_t)n * a.groups;
    const uint64_t *x0 = a.x[0] + (uint64_t)row * a.in, *x1 = a.x[1] + (uint64_t)row * a.in;
    Pair y{0, 0};
    for (uint32_t j = lane; j < a.in; j += 64) {
        const int code = (w[j / 2] >> (4 * (j & 1))) & 15;
        const int64_t weight = (int64_t)((code ^ 8) - 8) * s[j / (uint32_t)a.group];
        y.p0 += (uint64_t)weight * x0[j];
        y.p1 += (uint64_t)weight * x1[j];
    }
    y.p0 = wave_sum(y.p0);
    y.p1 = wave_sum(y.p1);
    if (lane != 0) return;
    const Pair t = truncate_drawn(y, a.frac, state_of(a.seedA, kTruncateWords * i));
    a.out[0][i] = t.p0;
    a.out[1][i] = t.p1;
}

}  // namespace hb
