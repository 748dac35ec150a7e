// Fixed point after a product: shares of y / 2^f from shares of y, as the protocol's linear layers and attention need it.
#pragma once

#include "hb_protocol.hpp"

namespace hb {

// Truncation.  y = y_0 + y_1 mod 2^64, read as signed, -2^62 <= y < 2^62; f in 1 .. 62; v: the element's four dealer words.  With
// u = y + 2^62 < 2^63 and the mask r = v_0 + v_1 the parties open c = u + r.  Both are numbers of 63 bits and one: the lower 63 bits of u + r carry
// exactly when the top bits of c and r differ, so
//     u = c' - r' + 2^63 (c_m xor r_m),      c' = c mod 2^63, c_m = c >> 63, and the same of r,
// and dividing each term by 2^f leaves floor(u / 2^f) or one more (where the lower f bits of u and r carry).  The dealer hands out shares of
// r' >> f (v_2 and the rest) and of r_m (v_3 and the rest); c_m xor r_m = c_m + (1 - 2 c_m) r_m is linear in them.
// Shifting each share on its own, which needs no dealer, is wrong by 2^(64-f) with probability |y| / 2^63: 2^-28 an element for products at
// 2^32 that reach 8, several times in a long decode.
constexpr int kTruncateWords = 4;

__device__ __forceinline__ Pair truncate(Pair y, int f, const uint64_t *v)
{
    const uint64_t low = ~0ull >> 1;
    const uint64_t r = v[0] + v[1];                                       // the dealer's mask
    const uint64_t c = (y.p0 + v[0]) + (y.p1 + v[1]) + (1ull << 62);      // opened
    const uint64_t cm = c >> 63, minus = 0 - cm;                          // minus: all ones where c_m = 1
    const uint64_t rh1 = ((r & low) >> f) - v[2], rm1 = (r >> 63) - v[3];
    const int up = 63 - f;
    // +- 2^(63-f) times a share of r_m, the sign being 1 - 2 c_m
    const uint64_t m0 = ((v[3] << up) ^ minus) + cm, m1 = ((rm1 << up) ^ minus) + cm;
    return Pair{((c & low) >> f) + (cm << up) - (1ull << (62 - f)) - v[2] + m0, m1 - rh1};
}

// The four words from generator state z on (state of word v_0).
__device__ __forceinline__ Pair truncate_drawn(Pair y, int f, uint64_t z)
{
    uint64_t v[kTruncateWords];
#pragma unroll
    for (int j = 0; j < kTruncateWords; ++j) v[j] = mix64(z + (uint64_t)j * kGamma);
    return truncate(y, f, v);
}

// State of word j of the generator started at s: mix64 of it is the word.
__device__ __forceinline__ uint64_t state_of(uint64_t s, uint64_t j) { return s + (j + 1) * kGamma; }

}  // namespace hb
