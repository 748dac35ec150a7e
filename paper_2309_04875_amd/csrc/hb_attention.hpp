// Attention of one new token over a paged cache of masked numbers, with the reduced-ring ReLU between its two products.
#pragma once

#include "hb_cache.hpp"

namespace hb {

struct AttentionArgs {
    CacheView cache;
    const uint64_t *q[2];                 // [batch][q_heads][dim]
    uint64_t *out[2];
    uint64_t *scores[2];                  // [batch][q_heads][max_len], workspace
    uint64_t *parts;                      // [splits][batch][q_heads][dim][2], workspace
    const int32_t *table, *lens;          // [batch][table_width], [batch]
    uint64_t table_width;
    uint64_t seed_q, seed_s, seed_p, seed_o;
    uint32_t batch, q_heads, max_len, splits, per_split;
};

__device__ __forceinline__ uint32_t length_of(const AttentionArgs &a, uint32_t b)
{
    const int32_t n = a.lens[b];
    return n < 0 ? 0 : ((uint32_t)n > a.max_len ? a.max_len : (uint32_t)n);
}

constexpr int kAttentionBlock = 256;

// Scores: one wavefront per (sequence, query head, position), lanes over the dimensions.
__global__ void __launch_bounds__(kAttentionBlock)
attention_scores_kernel(AttentionArgs a)
{
    const CacheView &c = a.cache;
    const uint64_t j = (uint64_t)blockIdx.x * (kAttentionBlock / 64) + threadIdx.x / 64;
    if (j >= (uint64_t)a.batch * a.q_heads * a.max_len) return;
    const uint32_t lane = threadIdx.x % 64, t = (uint32_t)(j % a.max_len);
    const uint64_t row = j / a.max_len;
    const uint32_t b = (uint32_t)(row / a.q_heads), head = (uint32_t)(row % a.q_heads) / (a.q_heads / c.heads);
    const int64_t page = t < length_of(a, b) ? a.table[b * a.table_width + t / c.page] : -1;
    Pair s{0, 0};
    if (page >= 0 && page < c.pages) {
        const uint64_t masks = stream_word(c.page_seeds[page], 0);
        const uint64_t *keys = c.keys + page * page_numbers(c);
        uint64_t c1 = 0;
        for (uint32_t d = lane; d < c.dim; d += 64) {
            const uint64_t i = row * c.dim + d, e = place_in_page(c, head, t % c.page, d);
            const uint64_t a0 = stream_word(a.seed_q, 2 * i), a1 = stream_word(a.seed_q, 2 * i + 1);
            const uint64_t eps = (a.q[0][i] - a0) + (a.q[1][i] - a1);                              // opened
            const uint64_t b0 = stream_word(masks, 2 * e), b1 = stream_word(masks, 2 * e + 1), del = keys[e];
            s.p0 += eps * (b0 + del) + del * a0;
            s.p1 += eps * b1 + del * a1;
            c1 += (a0 + a1) * (b0 + b1);                                                         // the dealer's triple
        }
        const uint64_t z = state_of(a.seed_s, 5 * j), c0 = mix64(z);
        s.p0 = wave_sum(s.p0) + c0;
        s.p1 = wave_sum(s.p1 + c1) - c0;
        s = truncate_drawn(s, 16, z + kGamma);
    }
    if (lane == 0) {
        a.scores[0][j] = s.p0;
        a.scores[1][j] = s.p1;
    }
}

// The product with the values: one thread per (split, sequence, query head, dimension).
__global__ void __launch_bounds__(kAttentionBlock)
attention_values_kernel(AttentionArgs a)
{
    const CacheView &c = a.cache;
    const uint64_t i = (uint64_t)blockIdx.x * kAttentionBlock + threadIdx.x;
    const uint64_t rows = (uint64_t)a.batch * a.q_heads, numbers = rows * c.dim;
    if (i >= numbers) return;
    const uint32_t d = (uint32_t)(i % c.dim);
    const uint64_t row = i / c.dim;
    const uint32_t b = (uint32_t)(row / a.q_heads), head = (uint32_t)(row % a.q_heads) / (a.q_heads / c.heads);
    const uint32_t length = length_of(a, b), first = blockIdx.y * a.per_split;
    const uint32_t last = first + a.per_split < length ? first + a.per_split : length;
    Pair o{0, 0};
    for (uint32_t t = first; t < last; ++t) {
        const int64_t page = a.table[b * a.table_width + t / c.page];
        if (page < 0 || page >= c.pages) continue;
        const uint64_t masks = stream_word(c.page_seeds[page], 1), j = row * a.max_len + t, e = place_in_page(c, head, t % c.page, d);
        const uint64_t a0 = stream_word(a.seed_p, 2 * j), a1 = stream_word(a.seed_p, 2 * j + 1);
        const uint64_t eps = (a.scores[0][j] - a0) + (a.scores[1][j] - a1);                          // opened
        const uint64_t b0 = stream_word(masks, 2 * e), b1 = stream_word(masks, 2 * e + 1), del = c.values[page * page_numbers(c) + e];
        o.p0 += eps * (b0 + del) + del * a0;
        o.p1 += eps * b1 + del * a1 + (a0 + a1) * (b0 + b1);
    }
    uint64_t *to = a.parts + 2 * (blockIdx.y * numbers + i);
    to[0] = o.p0;
    to[1] = o.p1;
}

// Joins the splits and divides by the length: a truncation by its whole bits, a factor in (1/2, 1] for the rest.
__global__ void __launch_bounds__(kAttentionBlock)
attention_join_kernel(AttentionArgs a)
{
    const uint64_t per = (uint64_t)a.q_heads * a.cache.dim;
    const uint32_t b = blockIdx.y, at = blockIdx.x * kAttentionBlock + threadIdx.x;
    if (at >= per) return;
    const uint64_t i = b * per + at, numbers = a.batch * per;
    const uint32_t length = __builtin_amdgcn_readfirstlane(length_of(a, b));
    Pair o{0, 0};
    if (length != 0) {
        const uint64_t z = state_of(a.seed_o, 9 * i), c0 = mix64(z);
        o = Pair{c0, 0 - c0};
        for (uint32_t s = 0; s < a.splits; ++s) {
            o.p0 += a.parts[2 * (s * numbers + i)];
            o.p1 += a.parts[2 * (s * numbers + i) + 1];
        }
        const int whole = 31 - __builtin_clz(length);
        const uint64_t factor = ((1ull << (16 + whole)) + length / 2) / length;
        o = truncate_drawn(o, 16 + whole, z + kGamma);
        o = truncate_drawn(Pair{o.p0 * factor, o.p1 * factor}, 16, z + 5 * kGamma);
    }
    a.out[0][i] = o.p0;
    a.out[1][i] = o.p1;
}

}  // namespace hb
