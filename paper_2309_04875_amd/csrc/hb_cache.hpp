// Keys and values of secret-shared tokens in a paged cache of masked numbers, with the position rotation on the way.
#pragma once

#include "hb_fixed.hpp"

namespace hb {

// A cache as kernels see it: number (page, head, offset, d) of the keys or values is what both parties know, x - b.
struct CacheView {
    uint64_t *keys, *values;        // [pages][heads][page][dim]
    const uint64_t *page_seeds;     // [pages]
    uint32_t pages, heads, page, dim;
};

// Place of the number (head, offset, d) within its page, and what words of the page's masks belong to it: 2 place, 2 place + 1.
__device__ __forceinline__ uint64_t place_in_page(const CacheView &c, uint32_t head, uint32_t offset, uint32_t d)
{
    return ((uint64_t)head * c.page + offset) * c.dim + d;
}
__device__ __forceinline__ uint64_t page_numbers(const CacheView &c) { return (uint64_t)c.heads * c.page * c.dim; }

struct AppendArgs {
    CacheView cache;
    const uint64_t *k[2], *v[2], *q[2];   // [tokens][heads][dim], q: [tokens][q_heads][dim]
    uint64_t *qo[2];
    const int64_t *slots;
    const int32_t *positions, *cos, *sin; // cos, sin: [table_rows][rot / 2]
    uint64_t tokens, table_rows, seedA;
    uint32_t q_heads, rot;
    int frac;
    int32_t q_mul;
};

constexpr int kAppendBlock = 256;

// A thread takes a pair of numbers of one token: dimensions d and d + rot/2 of a rotated pair, two neighbours elsewhere.
__global__ void __launch_bounds__(kAppendBlock)
cache_append_kernel(AppendArgs a)
{
    const CacheView &c = a.cache;
    const uint32_t half = a.rot / 2, pairs = c.dim / 2;
    const uint32_t items = (2 * c.heads + a.q_heads) * pairs;
    const uint64_t i = (uint64_t)blockIdx.x * kAppendBlock + threadIdx.x;
    const uint64_t token = i / items;
    if (token >= a.tokens) return;
    const uint32_t item = (uint32_t)(i % items), pair = item % pairs;
    uint32_t head = item / pairs;
    const int64_t slot = a.slots[token];
    if (slot < 0 || (uint64_t)slot >= (uint64_t)c.pages * c.page) return;
    int64_t position = 0;
    if (half != 0) {
        position = a.positions[token];
        if (position < 0 || (uint64_t)position >= a.table_rows) return;
    }
    const bool is_key = head < c.heads, is_query = head >= 2 * c.heads, turned = !is_query && !is_key ? false : pair < half;
    if (!is_key) head -= is_query ? 2 * c.heads : c.heads;
    const uint32_t d0 = pair < half && turned ? pair : (turned || !(is_key || is_query) ? 2 * pair : a.rot + 2 * (pair - half));
    const uint32_t d1 = turned ? d0 + half : d0 + 1;
    const uint64_t *const *x = is_query ? a.q : is_key ? a.k : a.v;
    const uint64_t row = (token * (is_query ? a.q_heads : c.heads) + head) * c.dim;
    Pair y0{x[0][row + d0], x[1][row + d0]}, y1{x[0][row + d1], x[1][row + d1]};
    if (turned || is_query) {
        uint64_t co = 1ull << a.frac, si = 0;
        if (turned) {
            co = (uint64_t)(int64_t)a.cos[position * half + pair];
            si = (uint64_t)(int64_t)a.sin[position * half + pair];
        }
        if (is_query) {                              // the public factor goes into the table, rounded to its precision
            const int64_t round = (int64_t)1 << (a.frac - 1);
            co = (uint64_t)(((int64_t)co * a.q_mul + round) >> a.frac);
            si = (uint64_t)(((int64_t)si * a.q_mul + round) >> a.frac);
        }
        const uint64_t base = is_query ? a.tokens * c.heads * c.dim : 0;
        const Pair t0{y0.p0 * co - y1.p0 * si, y0.p1 * co - y1.p1 * si}, t1{y1.p0 * co + y0.p0 * si, y1.p1 * co + y0.p1 * si};
        y0 = truncate_drawn(t0, a.frac, state_of(a.seedA, kTruncateWords * (base + row + d0)));
        y1 = truncate_drawn(t1, a.frac, state_of(a.seedA, kTruncateWords * (base + row + d1)));
    }
    if (is_query) {
        a.qo[0][row + d0] = y0.p0;
        a.qo[1][row + d0] = y0.p1;
        a.qo[0][row + d1] = y1.p0;
        a.qo[1][row + d1] = y1.p1;
        return;
    }
    const uint32_t page = (uint32_t)((uint64_t)slot / c.page), offset = (uint32_t)((uint64_t)slot % c.page);
    const uint64_t masks = stream_word(c.page_seeds[page], is_key ? 0 : 1);
    uint64_t *to = (is_key ? c.keys : c.values) + page * page_numbers(c);
    const uint64_t e0 = place_in_page(c, head, offset, d0), e1 = place_in_page(c, head, offset, d1);
    to[e0] = (y0.p0 - stream_word(masks, 2 * e0)) + (y0.p1 - stream_word(masks, 2 * e0 + 1));      // opened
    to[e1] = (y1.p0 - stream_word(masks, 2 * e1)) + (y1.p1 - stream_word(masks, 2 * e1 + 1));
}

}  // namespace hb
