// Matrix-vector products of shared activations with public 4-bit weights and group scales.
#pragma once

#include "hb_digits.hpp"

namespace hb {

struct LinearArgs {
    const uint64_t *x[2];       // [rows][in]
    uint64_t *out[2];           // [rows][out]
    const uint8_t *weight;      // [out][(in + 1) / 2]
    const int32_t *scales;      // [out][groups]
    uint64_t seedA, weight_bytes;
    uint64_t group_inverse;     // ceil(2^40 / group): input / group is (input * group_inverse) >> 40
    uint32_t rows, in, outs, groups;
    uint32_t row_tiles, out_tiles;
    int frac;
};

constexpr int kLinearStep = 256;                     // inputs of a step
constexpr int kLinearPlane = kLinearStep + 16;       // bytes of a digit's plane in LDS: rows of it fall into different banks

typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_any_t __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32_any_t __attribute__((aligned(1)));
typedef uint64_t u64x2_any_t __attribute__((ext_vector_type(2), aligned(8)));

// Digits of one row's inputs k0 .. k0 + 255 of both parties, 64 lanes at a time: lane l takes eight inputs of party l / 32.  In a plane (one digit
// of one party) eight inputs lie as their even ones, then their odd ones: the order in which a weight's low and high four bits come.
__device__ __forceinline__ void load_inputs(const LinearArgs &a, uint32_t row, uint32_t k0, uint32_t lane, uint64_t (&v)[8])
{
    const uint32_t k = k0 + 8 * (lane % 32);
    const uint64_t *x = a.x[lane / 32] + (uint64_t)row * a.in + k;
    if (row < a.rows && k + 8 <= a.in) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const u64x2_any_t p = *reinterpret_cast<const u64x2_any_t *>(x + 2 * j);
            v[2 * j] = p.x;
            v[2 * j + 1] = p.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = row < a.rows && k + j < a.in ? x[j] : 0;
    }
}
__device__ __forceinline__ void store_digits(uint8_t *planes, uint32_t lane, const uint64_t (&v)[8])
{
    uint32_t even[8], odd[8];
    digits_of({v[0], v[2], v[4], v[6]}, even);
    digits_of({v[1], v[3], v[5], v[7]}, odd);
    uint8_t *to = planes + (lane / 32 * 8) * kLinearPlane + 8 * (lane % 32);
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint64_t *>(to + i * kLinearPlane) = ((uint64_t)odd[i] << 32) | even[i];
}

// A step's weights of one lane, 32 bytes of row n = lane mod 16 of a tile.  FLUSH, the inputs that go into one sum before it is scaled (what
// divides the group): of 128 and 64 inputs of one matrix instruction lane quarter q holds 16, of 32 eight.
template <int FLUSH>
struct StepWeights {
    uint32_t w[8];
};
template <int FLUSH>
__device__ __forceinline__ uint32_t piece_offset(uint32_t piece, uint32_t q)
{
    if (FLUSH == 128) return 64 * piece + 16 * q;            // two pieces of 16 bytes
    if (FLUSH == 64) return 32 * piece + 8 * q;              // four of 8
    return 16 * piece + 4 * q;                               // eight of 4
}
template <int FLUSH>
__device__ __forceinline__ void load_weights(const LinearArgs &a, uint32_t n, uint32_t k0, uint32_t q, StepWeights<FLUSH> &s)
{
    const uint64_t at = (uint64_t)n * ((a.in + 1) / 2) + k0 / 2;
    const uint8_t *p = a.weight + at;
    constexpr int kPieces = FLUSH == 128 ? 2 : FLUSH == 64 ? 4 : 8, kWords = 8 / kPieces;
    if (at + kLinearStep / 2 <= a.weight_bytes) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint8_t *from = p + piece_offset<FLUSH>(i, q);
            if constexpr (kWords == 4) {
                const u32x4_any_t v = *reinterpret_cast<const u32x4_any_t *>(from);
                s.w[4 * i] = v.x, s.w[4 * i + 1] = v.y, s.w[4 * i + 2] = v.z, s.w[4 * i + 3] = v.w;
            } else if constexpr (kWords == 2) {
                const u32x2_any_t v = *reinterpret_cast<const u32x2_any_t *>(from);
                s.w[2 * i] = v.x, s.w[2 * i + 1] = v.y;
            } else {
                s.w[i] = *reinterpret_cast<const u32_any_t *>(from);
            }
        }
    } else {                                                  // the last rows' ends: what lies behind the weights is not read
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t from = piece_offset<FLUSH>(i / kWords, q) + 4 * (i % kWords);
            uint32_t v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) v |= at + from + j < a.weight_bytes ? (uint32_t)p[from + j] << (8 * j) : 0;
            s.w[i] = v;
        }
    }
}

// Products of TM rows and RT tiles of 16 outputs by each wavefront; WN wavefronts side by side over the outputs, WK over the inputs.
//
// A row of inputs is 16 rows of digits, eight of each party: with one vector the matrix instruction's 16 rows are full.  Its columns are 16
// outputs' weights, four bits in the upper half of a byte (16 q: both halves of a packed byte become multiplicands by one AND and one
// shift).  Sums over FLUSH inputs are scaled into 64-bit sums, one for each digit (int32 x int32 + 64: one instruction), which stay below
// 2^62 (2^31 2^14 inputs), so that the factor 16 can be shifted out exactly at the end.
template <int TM, int RT, int WN, int WK, int FLUSH>
__global__ void __launch_bounds__(64 * WN * WK)
linear_q4_kernel(LinearArgs a)
{
    static_assert(WN == 1 || WK == 1, "wavefronts share digits over the outputs or split the inputs");
    constexpr int kDigitBytes = 16 * kLinearPlane, kBuffers = WN > 1 ? 2 : 1;
    static_assert(WN * RT * 256 <= kDigitBytes, "the sums' exchange takes the digits' place");
    __shared__ __align__(16) uint8_t lds[kBuffers * WK * TM * kDigitBytes];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t q = lane / 16, wn = wave % WN, wk = wave / WN;
    const uint32_t row0 = (blockIdx.x % a.row_tiles) * TM, tile0 = (blockIdx.x / a.row_tiles) * (WN * RT) + wn * RT;
    const uint32_t steps = (a.in + kLinearStep - 1) / kLinearStep;
    uint32_t n[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        n[t] = 16 * (tile0 + t) + lane % 16;
        n[t] = n[t] < a.outs ? n[t] : a.outs - 1;
    }
    int64_t sum[TM][RT][4] = {};
    StepWeights<FLUSH> weights[RT];
    constexpr int kOwn = WN > 1 ? TM / WN : TM;               // rows whose digits this wavefront makes
    uint64_t inputs[kOwn][8];
    const uint32_t own = WN > 1 ? wn * kOwn : 0;
    auto load = [&](uint32_t step) {
#pragma unroll
        for (int m = 0; m < kOwn; ++m) load_inputs(a, row0 + own + m, kLinearStep * step, lane, inputs[m]);
#pragma unroll
        for (int t = 0; t < RT; ++t) load_weights<FLUSH>(a, n[t], kLinearStep * step, q, weights[t]);
    };
    uint32_t buffer = 0;
    if (wk < steps) load(wk);
    for (uint32_t step = wk; step < steps; step += WK) {
        uint8_t *planes = lds + (WN > 1 ? buffer * TM : wk * TM) * kDigitBytes;
#pragma unroll
        for (int m = 0; m < kOwn; ++m) store_digits(planes + (own + m) * kDigitBytes, lane, inputs[m]);
        StepWeights<FLUSH> now[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) now[t] = weights[t];
        if (step + WK < steps) load(step + WK);
        if constexpr (WN > 1) __syncthreads();                // (two buffers: the next step's digits go to the other one)
        else wave_exchange();
        buffer ^= 1;
        const uint8_t *column = planes + (lane % 16) * kLinearPlane;
#pragma unroll
        for (int f = 0; f < kLinearStep / FLUSH; ++f) {
            const uint32_t k = kLinearStep * step + FLUSH * f;
            uint32_t group = (uint32_t)((k * a.group_inverse) >> 40);
            group = group < a.groups ? group : a.groups - 1;
            int32_t scale[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) scale[t] = a.scales[(uint64_t)n[t] * a.groups + group];
            i32x4_t part[TM][RT] = {};
            if constexpr (FLUSH == 32) {
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    const i32x2_t digits = *reinterpret_cast<const i32x2_t *>(column + m * kDigitBytes + 32 * f + 8 * q);
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const uint32_t w = now[t].w[f];
                        part[m][t] = mfma_16x16x32(digits, i32x2_t{(int)((w << 4) & 0xF0F0F0F0u), (int)(w & 0xF0F0F0F0u)}, part[m][t]);
                    }
                }
            } else {
#pragma unroll
                for (int h = 0; h < FLUSH / 64; ++h) {
                    const uint32_t place = FLUSH == 128 ? 128 * f + 32 * q + 16 * h : 64 * f + 16 * q;
#pragma unroll
                    for (int m = 0; m < TM; ++m) {
                        const i32x4_t digits = *reinterpret_cast<const i32x4_t *>(column + m * kDigitBytes + place);
#pragma unroll
                        for (int t = 0; t < RT; ++t) {
                            const uint32_t u = now[t].w[2 * (f * (FLUSH / 64) + h)], v = now[t].w[2 * (f * (FLUSH / 64) + h) + 1];
                            const i32x4_t w{(int)((u << 4) & 0xF0F0F0F0u), (int)(u & 0xF0F0F0F0u), (int)((v << 4) & 0xF0F0F0F0u), (int)(v & 0xF0F0F0F0u)};
                            part[m][t] = mfma_16x16x64(digits, w, part[m][t]);
                        }
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < TM; ++m) {
#pragma unroll
                for (int t = 0; t < RT; ++t) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[m][t][r] += (int64_t)part[m][t][r] * scale[t];
                }
            }
        }
        if constexpr (WN == 1) wave_exchange();               // the digits have been read
    }
    // A lane's four digits of party q / 2, upper or lower half; then the other half's and the other wavefronts'.
    if constexpr (WN > 1 || WK > 1) __syncthreads();
    uint64_t *sums = reinterpret_cast<uint64_t *>(lds);       // [wk][row][tile of the workgroup][party][16]
    constexpr int kSums = TM * RT * WN * 32;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            uint64_t y = 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) y += (uint64_t)(sum[m][t][r] >> 4) << (8 * r);
            if (q & 1) y <<= 32;
            y += __shfl_xor((unsigned long long)y, 16, 64);
            if ((q & 1) == 0) sums[wk * kSums + ((m * WN + wn) * RT + t) * 32 + 16 * (q / 2) + lane % 16] = y;
        }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kSums / 2; i += 64 * WN * WK) {
        const uint32_t m = i / (RT * WN * 16), tile = (blockIdx.x / a.row_tiles) * (WN * RT) + i / 16 % (RT * WN);
        const uint32_t row = row0 + m, out = 16 * tile + i % 16;
        if (row >= a.rows || out >= a.outs) continue;
        const uint64_t at = (uint64_t)row * a.outs + out;
        uint64_t v[kTruncateWords];
#pragma unroll
        for (int j = 0; j < kTruncateWords; ++j) v[j] = stream_word(a.seedA, kTruncateWords * at + j);
        Pair y{0, 0};
#pragma unroll
        for (int w = 0; w < WK; ++w) {
            const uint64_t *from = sums + w * kSums + i / 16 * 32 + i % 16;
            y.p0 += from[0];
            y.p1 += from[16];
        }
        const Pair t = truncate(y, a.frac, v);
        a.out[0][at] = t.p0;
        a.out[1][at] = t.p1;
    }
}

}  // namespace hb
