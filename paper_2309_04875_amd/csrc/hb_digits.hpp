// Sums of products on Z_2^64 by the matrix cores: numbers of the ring as eight digits of eight bits.
//
// x = sum over i of s_i 2^(8i) mod 2^64 with signed digits -128 .. 127, one for each multiplicand of an int8 matrix instruction, whose int32 sums
// are exact: the bytes of x + 0x8080808080808080, each less 128 (the addition carries what a digit of 128 and more owes to the next; the
// last carry leaves the ring).  Less 128 is the top bit flipped, for a byte read as signed.
#pragma once

#include "hb_fixed.hpp"

namespace hb {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));

constexpr uint64_t kDigitBias = 0x8080808080808080ull;
constexpr uint32_t kDigitFlip = 0x80808080u;

// The 4 x 4 bytes of four words turned: word j gets byte j of each.
__device__ __forceinline__ void turn_bytes(const uint32_t (&w)[4], uint32_t *out)
{
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// Numbers in halves, the bytes' top bits flipped: x - 0x8080808080808080 in digits, one addition less for each number where sums of such digits with a
// vector are owed 0x8080808080808080 times the vector's sum, once for all of them.
template <int N>
struct Flipped {
    uint32_t low[N], high[N];
};

// Dealer words of N states, flipped: the last xor of the generator takes the flip along.  (Halves, for a register each: as 64-bit numbers they would be moved to
// where four of a half lie side by side, an instruction and a half a word.)
template <int N>
__device__ __forceinline__ void mix_flipped(uint64_t (&z)[N], Flipped<N> &out)         // (in step: as in mix_words)
{
    settle(z);
    priority<true, kElsewhere>();
    xor_shift(z, 30);
    settle(z);
    priority<true, kElsewhere>();
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] *= 0xBF58476D1CE4E5B9ull;
    xor_shift(z, 27);
    settle(z);
    priority<true, kElsewhere>();
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] *= 0x94D049BB133111EBull;
    uint64_t t[N];
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = z[i] >> 31;
    settle(t);
    priority<true, kXorRuns>();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        out.low[i] = bitop3<kTtXor3>((uint32_t)z[i], (uint32_t)t[i], kDigitFlip);
        out.high[i] = bitop3<kTtXor3>((uint32_t)(z[i] >> 32), (uint32_t)(t[i] >> 32), kDigitFlip);
    }
    settle(out.low);
    settle(out.high);
    priority<true, kElsewhere>();
}

// Digits of four numbers: out[i] holds digit i of v[0] .. v[3], one byte each.
__device__ __forceinline__ void digits_of(const uint64_t (&v)[4], uint32_t (&out)[8])
{
    uint32_t low[4], high[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint64_t x = v[j] + kDigitBias;
        low[j] = (uint32_t)x;
        high[j] = (uint32_t)(x >> 32);
    }
    turn_bytes(low, out);
    turn_bytes(high, out + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] ^= kDigitFlip;
}

// The same turn of bytes across four neighbouring lanes, of a word each: the word of lane j (mod 4) becomes byte j of the four.  All four lanes run.
struct QuadTurn {
    uint32_t first, second;     // this lane's byte selectors
    __device__ __forceinline__ explicit QuadTurn(uint32_t lane)
        : first(lane & 1 ? 0x03070105u : 0x06020400u), second(lane & 2 ? 0x03020706u : 0x05040100u) {}
    __device__ __forceinline__ uint32_t operator()(uint32_t w) const
    {
        const uint32_t next = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0xB1, 0xF, 0xF, true);       // of lane ^ 1
        w = __builtin_amdgcn_perm(next, w, first);
        const uint32_t far = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x4E, 0xF, 0xF, true);        // of lane ^ 2
        return __builtin_amdgcn_perm(far, w, second);
    }
};
// Sum over four neighbouring lanes, in all of them.
__device__ __forceinline__ uint64_t quad_sum(uint64_t v)
{
    const uint32_t l1 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, 0xB1, 0xF, 0xF, true);
    const uint32_t h1 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), 0xB1, 0xF, 0xF, true);
    v += (uint64_t)h1 << 32 | l1;
    const uint32_t l2 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, 0x4E, 0xF, 0xF, true);
    const uint32_t h2 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), 0x4E, 0xF, 0xF, true);
    return v + ((uint64_t)h2 << 32 | l2);
}

// v of the lane whose number differs by X < 32.
template <int X>
__device__ __forceinline__ uint64_t across(uint64_t v)
{
    const uint32_t low = (uint32_t)__builtin_amdgcn_ds_swizzle((int)(uint32_t)v, X << 10 | 0x1F);
    const uint32_t high = (uint32_t)__builtin_amdgcn_ds_swizzle((int)(uint32_t)(v >> 32), X << 10 | 0x1F);
    return (uint64_t)high << 32 | low;
}

// c + A B of 16 x 64 by 64 x 16 int8.  Lane l holds 16 numbers of row (A) or column (B) l mod 16 in each of its four registers' bytes, those of
// the same 16 places of the sum in A and B (lanes l with the same l / 16 share them); which places is the caller's choice.  The result's lane l
// holds rows 4 (l / 16) .. + 3 of column l mod 16.
__device__ __forceinline__ i32x4_t mfma_16x16x64(i32x4_t a, i32x4_t b, i32x4_t c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
// The same of 32 places, eight a lane.
__device__ __forceinline__ i32x4_t mfma_16x16x32(i32x2_t a, i32x2_t b, i32x4_t c)
{
    return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), c, 0, 0, 0);
}

// What a lane has written to LDS and other lanes of its wavefront read.
__device__ __forceinline__ void wave_exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

}  // namespace hb
