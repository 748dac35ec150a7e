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
    uint32_t row_tiles;
    int frac;
};

constexpr uint32_t kDies = 8;
constexpr int kLinearStep = 256;                     // inputs of a step
constexpr int kLinearPlane = kLinearStep + 16;       // bytes of a digit's plane in LDS: rows of it fall into different banks

typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_any_t __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32_any_t __attribute__((aligned(1)));
typedef uint64_t u64x2_any_t __attribute__((ext_vector_type(2), aligned(8)));

// Digits of one row's inputs k0 .. k0 + 255 of both parties, 64 lanes at a time: lane l takes eight inputs of party l / 32.  In a plane (one digit
// of one party) eight inputs lie as their even ones, then their odd ones: the order in which a weight's low and high four bits come.
// whole: all of them are there, for every lane (otherwise what is not there is a zero, and its place is read from elsewhere in the row).
__device__ __forceinline__ void load_inputs(const LinearArgs &a, uint32_t row, uint32_t k0, uint32_t lane, bool whole, uint64_t (&v)[8])
{
    const uint32_t k = k0 + 8 * (lane % 32);
    if (whole) {
        const uint64_t *x = a.x[lane / 32] + (uint64_t)row * a.in + k;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const u64x2_any_t p = *reinterpret_cast<const u64x2_any_t *>(x + 2 * j);
            v[2 * j] = p.x;
            v[2 * j + 1] = p.y;
        }
    } else {
        const uint64_t *x = a.x[lane / 32] + (uint64_t)(row < a.rows ? row : 0) * a.in;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint64_t one = x[k + j < a.in ? k + j : 0];
            v[j] = row < a.rows && k + j < a.in ? one : 0;
            if (j % 2) __builtin_amdgcn_sched_barrier(0);
        }
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

// Half a step's weights of one lane, 16 bytes of row n = lane mod 16 of a tile: 32 inputs.  FLUSH, the inputs that go into one sum before it is scaled
// (what divides the group): of 128 and 64 inputs lane quarter q holds 16 for one matrix instruction, of 32 eight.
struct HalfWeights {
    uint32_t w[4];
};
template <int FLUSH>
__device__ __forceinline__ uint32_t piece_offset(uint32_t piece, uint32_t q)
{
    if (FLUSH == 128) return 16 * q;                         // one piece of 16 bytes
    if (FLUSH == 64) return 32 * piece + 8 * q;              // two of 8
    return 16 * piece + 4 * q;                               // four of 4
}
// p: the half's first byte of a lane's output.
template <int FLUSH>
__device__ __forceinline__ void load_weights(const uint8_t *p, uint32_t q, HalfWeights &s)
{
    constexpr int kPieces = 128 / FLUSH, kWords = 4 / kPieces;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const uint8_t *from = p + piece_offset<FLUSH>(i, q);
        if constexpr (kWords == 4) {
            const u32x4_any_t v = *reinterpret_cast<const u32x4_any_t *>(from);
            s.w[0] = v.x, s.w[1] = v.y, s.w[2] = v.z, s.w[3] = v.w;
        } else if constexpr (kWords == 2) {
            const u32x2_any_t v = *reinterpret_cast<const u32x2_any_t *>(from);
            s.w[2 * i] = v.x, s.w[2 * i + 1] = v.y;
        } else {
            s.w[i] = *reinterpret_cast<const u32_any_t *>(from);
        }
    }
}
// The same a byte at a time where bytes of some lane lie behind the last row: the last one instead, for no input has them.  A word after the other: what
// this rare path would hold at once would be taken from the loop's registers.
template <int FLUSH>
__device__ __forceinline__ void load_weights_end(const uint8_t *p, uint32_t q, const uint8_t *last, HalfWeights &s)
{
    constexpr int kWords = FLUSH / 32;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint8_t *word = p + piece_offset<FLUSH>(i / kWords, q) + 4 * (i % kWords);
        uint32_t v = 0;
        for (int j = 3; j >= 0; --j) {
            const uint8_t *from = word + j;
            v = v << 8 | *(from < last ? from : last);
        }
        s.w[i] = v;
        __builtin_amdgcn_sched_barrier(0);
    }
}
// 16 q of the even inputs, then of the odd ones.
__device__ __forceinline__ void unpack_weights(uint32_t w, int &even, int &odd)
{
    even = (int)((w << 4) & 0xF0F0F0F0u);
    odd = (int)(w & 0xF0F0F0F0u);
}

// Products of TM rows and RT tiles of 16 outputs by each wavefront; WN wavefronts side by side over the outputs, WK over the inputs.
//
// A row of inputs is 16 rows of digits, eight of each party: with one vector the matrix instruction's 16 rows are full.  Its columns are 16
// outputs' weights, four bits in the upper half of a byte (16 q: both halves of a packed byte become multiplicands by one AND and one
// shift).  A lane's four sums over FLUSH inputs, four digits of a party, are put together by twos, p + 256 p' (below 2^30), and scaled into 64-bit
// sums (int32 x int32 + 64: one instruction).  The factor 16 leaves the lower two before they are scaled, for their sum counts up to its 64th bit;
// the upper two's has 48 that count and keeps it to the end.
//
// A workgroup goes through the inputs in blocks of WK * P steps, whose digits its wavefronts make together and all of them read (with
// WN = P = 1 each makes its own); wavefront (wn, wk) multiplies steps wk, wk + WK, .. of a block with its own RT tiles.
template <int TM, int RT, int WN, int WK, int P, int FLUSH>
__global__ void __launch_bounds__(64 * WN * WK, 2)
linear_q4_kernel(LinearArgs a)
{
    constexpr int kWaves = WN * WK, kSteps = WK * P, kOwn = kSteps * TM / kWaves;      // kOwn: pieces of digits that a wavefront makes
    static_assert(kOwn * kWaves == kSteps * TM, "every wavefront makes as many pieces");
    constexpr bool kShared = WN > 1 || P > 1;
    constexpr int kDigitBytes = 16 * kLinearPlane, kBlockBytes = kSteps * TM * kDigitBytes, kBuffers = kShared && kBlockBytes <= 72 * 1024 ? 2 : 1;
    static_assert(kWaves * RT * TM * 256 <= kBuffers * kBlockBytes, "the sums' exchange takes the digits' place");
    __shared__ __align__(16) uint8_t lds[kBuffers * kBlockBytes];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t q = lane / 16, wn = wave % WN, wk = wave / WN;
    // Workgroups with the same weights run on the same die (they are dealt out to the eight in turn), whose cache then reads them once.
    const uint32_t place = blockIdx.x / kDies, group0 = place / a.row_tiles * kDies + blockIdx.x % kDies;
    const uint32_t row0 = place % a.row_tiles * TM, tile0 = group0 * (WN * RT) + wn * RT;
    if (16 * group0 * (WN * RT) >= a.outs) return;
    const uint32_t steps = (a.in + kLinearStep - 1) / kLinearStep;
    // A lane's rows of weights and scales; outputs behind the last are the last.
    const uint8_t *weight_row[RT];
    const int32_t *scale_row[RT];
    const uint32_t row_bytes = (a.in + 1) / 2;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const uint32_t out = 16 * (tile0 + t) + lane % 16, n = out < a.outs ? out : a.outs - 1;
        weight_row[t] = a.weight + (uint64_t)n * row_bytes;
        scale_row[t] = a.scales + (uint64_t)n * a.groups;
    }
    const uint32_t last_out = 16 * (tile0 + RT) < a.outs ? 16 * (tile0 + RT) - 1 : a.outs - 1;
    const uint64_t last_row = (uint64_t)last_out * row_bytes;
    int64_t sum[TM][RT][2] = {};
    constexpr int kScales = 128 / FLUSH;
    HalfWeights weights[P][2][RT];
    int32_t scales[P][2][RT][kScales];
    uint64_t inputs[kOwn][8];
    auto load_rows = [&](uint32_t first) {                    // of the block that begins with step `first`
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const uint32_t piece = wave * kOwn + i, step = first + piece / TM, row = row0 + piece % TM;
            if (step < steps) load_inputs(a, row, kLinearStep * step, lane, kLinearStep * (step + 1) <= a.in && row < a.rows, inputs[i]);
        }
    };
    auto load_half = [&](uint32_t step, int p, int half) {
        const uint32_t k = kLinearStep * step + 128 * half;
        if (last_row + k / 2 + 64 <= a.weight_bytes) {
#pragma unroll
            for (int t = 0; t < RT; ++t) load_weights<FLUSH>(weight_row[t] + k / 2, q, weights[p][half][t]);
        } else {
#pragma unroll
            for (int t = 0; t < RT; ++t) load_weights_end<FLUSH>(weight_row[t] + k / 2, q, a.weight + a.weight_bytes - 1, weights[p][half][t]);
        }
#pragma unroll
        for (int f = 0; f < kScales; ++f) {
            uint32_t group = (uint32_t)(((k + FLUSH * f) * a.group_inverse) >> 40);
            group = group < a.groups ? group : a.groups - 1;
#pragma unroll
            for (int t = 0; t < RT; ++t) scales[p][half][t][f] = scale_row[t][group];
        }
    };
    load_rows(0);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (p * WK + wk < steps) {
            load_half(p * WK + wk, p, 0);
            load_half(p * WK + wk, p, 1);
        }
    }
    uint32_t buffer = 0;
    for (uint32_t first = 0; first < steps; first += kSteps) {
        uint8_t *block = lds + buffer * kBlockBytes;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const uint32_t piece = wave * kOwn + i;
            if (first + piece / TM < steps) store_digits(block + piece * kDigitBytes, lane, inputs[i]);
        }
        load_rows(first + kSteps);
        if constexpr (kShared) __syncthreads();
        else wave_exchange();
        if constexpr (kBuffers == 2) buffer ^= 1;             // the next block's digits go to the other one
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const uint32_t step = first + p * WK + wk;
            if (step >= steps) break;
            const uint8_t *column = block + (p * WK + wk) * (TM * kDigitBytes) + (lane % 16) * kLinearPlane;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                int w[RT][8];
                int32_t scale[RT][kScales];
#pragma unroll
                for (int t = 0; t < RT; ++t) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) unpack_weights(weights[p][half][t].w[i], w[t][2 * i], w[t][2 * i + 1]);
#pragma unroll
                    for (int f = 0; f < kScales; ++f) scale[t][f] = scales[p][half][t][f];
                }
                if (step + kSteps < steps) load_half(step + kSteps, p, half);
#pragma unroll
                for (int f = 0; f < kScales; ++f) {
                    // A row's sums are scaled while the next one's are under way.
                    i32x4_t part[2][RT];
                    auto scaled = [&](int m) {
#pragma unroll
                        for (int t = 0; t < RT; ++t) {
                            const i32x4_t &s = part[m % 2][t];
                            const int low = (s[0] >> 4) + s[1] * 16, high = s[2] + s[3] * 256;
                            sum[m][t][0] += (int64_t)low * scale[t][f];
                            sum[m][t][1] += (int64_t)high * scale[t][f];
                        }
                    };
#pragma unroll
                    for (int m = 0; m < TM; ++m) {
                        const uint8_t *row = column + m * kDigitBytes + 128 * half;
                        const i32x4_t zero{0, 0, 0, 0};
                        if constexpr (FLUSH == 32) {
                            const i32x2_t digits = *reinterpret_cast<const i32x2_t *>(row + 32 * f + 8 * q);
#pragma unroll
                            for (int t = 0; t < RT; ++t) part[m % 2][t] = mfma_16x16x32(digits, i32x2_t{w[t][2 * f], w[t][2 * f + 1]}, zero);
                        } else {
#pragma unroll
                            for (int h = 0; h < FLUSH / 64; ++h) {
                                const int at = FLUSH == 128 ? h : f;
                                const i32x4_t digits = *reinterpret_cast<const i32x4_t *>(row + (FLUSH == 128 ? 32 * q + 16 * h : 64 * f + 16 * q));
#pragma unroll
                                for (int t = 0; t < RT; ++t)
                                    part[m % 2][t] = mfma_16x16x64(digits, i32x4_t{w[t][4 * at], w[t][4 * at + 1], w[t][4 * at + 2], w[t][4 * at + 3]},
                                                                   h == 0 ? zero : part[m % 2][t]);
                            }
                        }
                        if (m > 0) scaled(m - 1);
                        if constexpr (FLUSH == 32) __builtin_amdgcn_sched_barrier(0);
                    }
                    scaled(TM - 1);
                    if constexpr (TM > 1 || FLUSH == 32) __builtin_amdgcn_sched_barrier(0);   // (what is hoisted over this costs registers)
                }
            }
        }
        if constexpr (!kShared) wave_exchange();              // the digits have been read
        else if constexpr (kBuffers == 1) __syncthreads();
    }
    // A lane's four digits of party q / 2, upper or lower half; then the other half's and the other wavefronts'.
    __syncthreads();
    uint64_t *sums = reinterpret_cast<uint64_t *>(lds);       // [wk][row][tile of the workgroup][party][16]
    constexpr int kSums = TM * RT * WN * 32;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            uint64_t y = (uint64_t)sum[m][t][0] + ((uint64_t)(sum[m][t][1] >> 4) << 16);
            if (q & 1) y <<= 32;
            y += __shfl_xor((unsigned long long)y, 16, 64);
            if ((q & 1) == 0) sums[wk * kSums + ((m * WN + wn) * RT + t) * 32 + 16 * (q / 2) + lane % 16] = y;
        }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kSums / 2; i += 64 * WN * WK) {
        const uint32_t m = i / (RT * WN * 16), tile = group0 * (WN * RT) + i / 16 % (RT * WN);
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
