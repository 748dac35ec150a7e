// Matrix-vector products of shared activations with public 4-bit weights and group scales.
#pragma once

#include "hb_digits.hpp"
#include "hb_linear_plan.hpp"

namespace hb {

struct LinearArgs {
    const uint64_t *x[2];       // [rows][in]
    uint64_t *out[2];           // [rows][out]
    const uint8_t *weight;      // [out][(in + 1) / 2]
    const int32_t *scales;      // [out][groups]
    uint64_t seedA, weight_bytes;
    uint64_t group_inverse;     // ceil(2^40 / group): input / group is (input * group_inverse) >> 40
    uint32_t rows, in, outs, groups;
    uint32_t first_tile, row_tiles, pairs;     // of this launch: tiles of rows; workgroups, a tile of rows and a group of outputs each
    int frac;
};

constexpr int kLinearStep = 256;                     // inputs of a step
constexpr int kPieceBytes = 16 * kLinearStep;        // one row's digits of a step in LDS: 16 planes of a byte an input, eight of each party

typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint64_t u64x2_any_t __attribute__((ext_vector_type(2), aligned(8)));

// Digits of one row's inputs k0 .. k0 + 255 of both parties, 64 lanes at a time: lane l takes eight inputs of party l / 32.  In a plane r (one digit
// of one party) eight inputs lie as their even ones, then their odd ones: the order in which a weight's low and high four bits come.  Inputs 16 j .. 16 j + 15
// of plane r are at 16 (16 j + (r xor j)), where no two lanes meet in a bank.
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
    const uint32_t j = lane % 32 / 2, to = 256 * j + 16 * ((lane / 32 * 8) ^ j) + 8 * (lane % 2);
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint64_t *>(planes + (to ^ (16 * i))) = ((uint64_t)odd[i] << 32) | even[i];
}

// A step's weights of a tile, 16 rows of 128 bytes: lane l loads 16 bytes l mod 8 of rows l / 8 and l / 8 + 8, and they go through LDS to where the matrix
// instruction takes them.  (Loaded from there at once, 16 rows by 64 bytes an instruction, 16 cache lines are asked for in each quarter of it:
// 64 x (4096 -> 16384) 97 us for 109, 1 x (4096 -> 4096) 5.0 for 5.5, 64 x (4096 -> 16384) in groups of 32, then eight rows by eight tiles, 217 for 339.)
struct StepWeights {
    u32x4_t w[2];
};
// In LDS bytes 16 p .. of row r lie at 128 r + 16 (p xor r mod 8): no two lanes meet in a bank.
__device__ __forceinline__ void store_weights(uint8_t *tile, uint32_t lane, const StepWeights &s)
{
    const uint32_t row = lane / 8;
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<u32x4_t *>(tile + 128 * (8 * i + row) + 16 * (lane % 8 ^ row)) = s.w[i];
}
// The same from memory a byte at a time, where bytes of some lane lie behind the last row: the last one instead, for no input has them.
__device__ __forceinline__ void store_weights_end(uint8_t *tile, uint32_t lane, const uint8_t *p, uint32_t eight_rows, const uint8_t *last)
{
    const uint32_t row = lane / 8;
#pragma unroll 8
    for (uint32_t j = 0; j < 32; ++j) {
        const uint8_t *from = p + (j / 16 != 0 ? eight_rows : 0) + j % 16;
        tile[128 * (8 * (j / 16) + row) + 16 * (lane % 8 ^ row) + j % 16] = *(from < last ? from : last);
    }
}
// Half a step's weights of one lane, row n = lane mod 16: 32 inputs.  FLUSH, the inputs that go into one sum before it is scaled (what divides the group): of
// 128 and 64 inputs lane quarter q takes 16 for one matrix instruction, of 32 eight.
template <int FLUSH>
__device__ __forceinline__ void half_weights(const uint8_t *tile, uint32_t lane, int half, uint32_t (&w)[4])
{
    const uint32_t q = lane / 16;
    const uint8_t *row = tile + lane % 16 * 128;
    auto at = [&](uint32_t p) { return row + 16 * (p ^ lane % 8); };
    if constexpr (FLUSH == 128) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t *>(at(4 * half + q));
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else if constexpr (FLUSH == 64) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x2_t v = *reinterpret_cast<const u32x2_t *>(at(4 * half + 2 * i + q / 2) + 8 * (q % 2));
            w[2 * i] = v.x, w[2 * i + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint32_t *>(at(4 * half + i) + 4 * q);
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
//
// What bounds it: one row, the launch and the chain of loads, digits, product, join and truncation (4096 -> 4096, 9 MB, 4.9 us); many rows, waiting: of the
// 214,000 cycles of 64 rows, 4096 -> 16384, 137 G int8 operations, 93 us, the vector ALU takes 42 % (scaling, five instructions for two matrix instructions, and
// digits), the matrix cores 31 %, and these overlap little; the rest are loads, LDS and barriers that two wavefronts a SIMD, all that their
// registers leave, do not cover.
template <int TM, int RT, int WN, int WK, int P, int FLUSH>
__global__ void __launch_bounds__(64 * WN * WK, (TM * RT <= (FLUSH == 32 ? 4 : 8) && WN * WK == 8 ? 4 : 2))
linear_q4_kernel(LinearArgs a)
{
    constexpr int kWaves = WN * WK, kSteps = WK * P, kOwn = kSteps * TM / kWaves;      // kOwn: pieces of digits that a wavefront makes
    static_assert(kOwn * kWaves == kSteps * TM, "every wavefront makes as many pieces");
    constexpr bool kShared = WN > 1 || P > 1;
    // Shared digits of two blocks: one is written while the one before is still read.
    constexpr int kBlockBytes = kSteps * TM * kPieceBytes, kBuffers = kShared ? 2 : 1;
    static_assert(kBuffers * kBlockBytes + kWaves * RT * 2048 <= 160 * 1024, "LDS of a compute unit");
    static_assert(kWaves * RT * TM * 256 <= kBuffers * kBlockBytes, "the sums' exchange takes the digits' place");
    __shared__ __align__(256) uint8_t lds[kBuffers * kBlockBytes + kWaves * RT * 2048];
    const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t q = lane / 16, wn = wave % WN, wk = wave / WN;
    const uint32_t pair = linear_pair(blockIdx.x, a.pairs), group0 = pair / a.row_tiles;
    const uint32_t row0 = (a.first_tile + pair % a.row_tiles) * TM, tile0 = group0 * (WN * RT) + wn * RT;
    const uint32_t steps = (a.in + kLinearStep - 1) / kLinearStep;
    // A lane's rows of weights and scales; outputs behind the last are the last.
    const uint8_t *weight_row[RT];
    uint32_t eight_rows[RT];                                  // bytes from a lane's first row of weights to its second
    const int32_t *scale_row[RT];
    const uint32_t row_bytes = (a.in + 1) / 2;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        auto row = [&](uint32_t n) { return 16 * (tile0 + t) + n < a.outs ? 16 * (tile0 + t) + n : a.outs - 1; };
        weight_row[t] = a.weight + (uint64_t)row(lane / 8) * row_bytes + 16 * (lane % 8);
        eight_rows[t] = (row(lane / 8 + 8) - row(lane / 8)) * row_bytes;
        scale_row[t] = a.scales + (uint64_t)row(lane % 16) * a.groups;
    }
    uint8_t *my_weights = lds + kBuffers * kBlockBytes + wave * (RT * 2048);
    const uint32_t last_out = 16 * (tile0 + RT) < a.outs ? 16 * (tile0 + RT) - 1 : a.outs - 1;
    const uint64_t last_row = (uint64_t)last_out * row_bytes;
    uint64_t sum[TM][RT][2] = {};                             // mod 2^64: a long row of large scales goes round
    // Scales: lane quarter q loads that of the q-th FLUSH inputs of every four in a step.
    constexpr int kScales = 128 / FLUSH, kScaleLoads = FLUSH == 32 ? 2 : 1;
    StepWeights weights[P][RT];
    int32_t scales[P][RT][kScaleLoads];
    uint64_t inputs[kOwn][8];
    auto load_rows = [&](uint32_t first) {                    // of the block that begins with step `first`
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const uint32_t piece = wave * kOwn + i, step = first + piece / TM, row = row0 + piece % TM;
            if (step < steps) load_inputs(a, row, kLinearStep * step, lane, kLinearStep * (step + 1) <= a.in && row < a.rows, inputs[i]);
        }
    };
    // whether no weight of the step lies behind the last row
    auto weights_there = [&](uint32_t step) { return last_row + kLinearStep * step / 2 + 128 <= a.weight_bytes; };
    auto load_step = [&](uint32_t step, int p) {
        const uint32_t k = kLinearStep * step;
        if (weights_there(step)) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const uint8_t *from = weight_row[t] + k / 2;
                weights[p][t].w[0] = *reinterpret_cast<const u32x4_any_t *>(from);
                weights[p][t].w[1] = *reinterpret_cast<const u32x4_any_t *>(from + eight_rows[t]);
            }
        }
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            const uint32_t piece = FLUSH == 128 ? q % 2 : q + 4 * i;
            uint32_t group = (uint32_t)(((k + FLUSH * piece) * a.group_inverse) >> 40);
            group = group < a.groups ? group : a.groups - 1;
#pragma unroll
            for (int t = 0; t < RT; ++t) scales[p][t][i] = scale_row[t][group];
        }
    };
    load_rows(0);
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (p * WK + wk < steps) load_step(p * WK + wk, p);
    }
    uint32_t buffer = 0;
    for (uint32_t first = 0; first < steps; first += kSteps) {
        uint8_t *block = lds + buffer * kBlockBytes;
        uint32_t l = lane;
        if constexpr (kWaves == 16 || (FLUSH == 32 && TM * RT <= 4)) settle(l);      // (what follows from it would be kept in registers: 128 are all)
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const uint32_t piece = wave * kOwn + i;
            if (first + piece / TM < steps) store_digits(block + piece * kPieceBytes, l, inputs[i]);
        }
        load_rows(first + kSteps);
        if constexpr (kShared) __syncthreads();
        else wave_exchange();
        if constexpr (kShared) buffer ^= 1;                   // the next block's digits go to the other one
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const uint32_t step = first + p * WK + wk;
            if (step >= steps) break;
            if (p > 0) wave_exchange();                       // the weights before have been read
            int32_t now[RT][kScaleLoads];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (weights_there(step)) store_weights(my_weights + 2048 * t, l, weights[p][t]);
                else store_weights_end(my_weights + 2048 * t, lane, weight_row[t] + kLinearStep * step / 2, eight_rows[t], a.weight + a.weight_bytes - 1);
#pragma unroll
                for (int i = 0; i < kScaleLoads; ++i) now[t][i] = scales[p][t][i];
            }
            wave_exchange();
            if (step + kSteps < steps) load_step(step + kSteps, p);
            // inputs 16 j .. of this lane's digit, j = c + what lane quarter q adds
            const uint8_t *digits_here = block + (p * WK + wk) * (TM * kPieceBytes);
            const uint32_t of_q = FLUSH == 128 ? 2 * q : FLUSH == 64 ? q : q / 2, lane_at = 256 * of_q + 16 * (lane % 16 ^ of_q);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                int w[RT][8];
                int32_t scale[RT][kScales];
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    uint32_t packed[4];
                    half_weights<FLUSH>(my_weights + 2048 * t, l, half, packed);
#pragma unroll
                    for (int i = 0; i < 4; ++i) unpack_weights(packed[i], w[t][2 * i], w[t][2 * i + 1]);
#pragma unroll
                    for (int f = 0; f < kScales; ++f) {
                        const int piece = kScales * half + f;
                        scale[t][f] = __builtin_amdgcn_ds_bpermute(4 * (16 * (piece % 4) + l % 16), now[t][piece / 4]);
                    }
                }
#pragma unroll
                for (int f = 0; f < kScales; ++f) {
                    // A row's sums are scaled while the next one's are under way.
                    i32x4_t part[2][RT];
                    auto scaled = [&](int m) {
#pragma unroll
                        for (int t = 0; t < RT; ++t) {
                            const i32x4_t &s = part[m % 2][t];
                            const int low = (s[0] >> 4) + s[1] * 16, high = s[2] + s[3] * 256;
                            sum[m][t][0] += (uint64_t)((int64_t)low * scale[t][f]);
                            sum[m][t][1] += (uint64_t)((int64_t)high * scale[t][f]);
                        }
                    };
#pragma unroll
                    for (int m = 0; m < TM; ++m) {
                        auto digits_at = [&](uint32_t c) { return digits_here + m * kPieceBytes + (lane_at ^ (16 * c)) + 256 * c; };
                        const i32x4_t zero{0, 0, 0, 0};
                        if constexpr (FLUSH == 32) {
                            const i32x2_t digits = *reinterpret_cast<const i32x2_t *>(digits_at(8 * half + 2 * f) + 8 * (q % 2));
#pragma unroll
                            for (int t = 0; t < RT; ++t) part[m % 2][t] = mfma_16x16x32(digits, i32x2_t{w[t][2 * f], w[t][2 * f + 1]}, zero);
                        } else {
#pragma unroll
                            for (int h = 0; h < FLUSH / 64; ++h) {
                                const int at = FLUSH == 128 ? h : f;
                                const i32x4_t digits = *reinterpret_cast<const i32x4_t *>(digits_at(8 * half + (FLUSH == 128 ? h : 4 * f)));
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
    }
    // A lane's four digits of party q / 2, upper or lower half; then the other half's and the other wavefronts'.
    __syncthreads();
    uint64_t *sums = reinterpret_cast<uint64_t *>(lds);       // [wk][row][tile of the workgroup][party][16]
    constexpr int kSums = TM * RT * WN * 32;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            uint64_t y = sum[m][t][0] + (sum[m][t][1] >> 4 << 16);
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
