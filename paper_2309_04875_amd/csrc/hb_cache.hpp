// Keys and values of secret-shared tokens in a paged cache of masked numbers, with the position rotation on the way.
#pragma once

#include "hb_append_plan.hpp"
#include "hb_fixed.hpp"
#include "hb_kernels.hpp"

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
    uint64_t tokens, table_rows, seedA;   // of this launch, as are the addresses above but for the tables
    uint64_t queries_at;                  // number of the first query, as dealer words count them, beyond that of the first key
    uint32_t q_heads, rot;
    int frac;
    int32_t q_mul;
};

// N neighbouring numbers of both parties.
template <int N>
__device__ __forceinline__ void load_numbers(const uint64_t *const (&x)[2], uint64_t at, Pair (&y)[N])
{
    if constexpr (N == 2) {
        const U64x2 a = load_stream2(x[0] + at), b = load_stream2(x[1] + at);
        y[0] = Pair{a.a, b.a};
        y[1] = Pair{a.b, b.b};
    } else {
        y[0] = Pair{load_stream(x[0] + at), load_stream(x[1] + at)};
    }
}
template <int N>
__device__ __forceinline__ void store_numbers(uint64_t *to, const uint64_t (&v)[N])
{
    if constexpr (N == 2) store_stream2(to, U64x2{v[0], v[1]});
    else store_stream(to, v[0]);
}

// Truncations of N numbers, z: state of the first's first word.
template <int N>
__device__ __forceinline__ void truncate_numbers(Pair (&y)[N], int f, uint64_t z)
{
    uint64_t v[N * kTruncateWords];
#pragma unroll
    for (int j = 0; j < N * kTruncateWords; ++j) v[j] = z + (uint64_t)j * kGamma;
    mix_words<true>(v);
    settle(v);
    priority<true, kElsewhere>();
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = truncate(y[j], f, v + kTruncateWords * j);
}
// What both parties learn of N numbers, z: state of the first's first mask word.
template <int N>
__device__ __forceinline__ void open_numbers(const Pair (&y)[N], uint64_t z, uint64_t *to)
{
    uint64_t b[2 * N], opened[N];
#pragma unroll
    for (int j = 0; j < 2 * N; ++j) b[j] = z + (uint64_t)j * kGamma;
    mix_words<true>(b);
    settle(b);
    priority<true, kElsewhere>();
#pragma unroll
    for (int j = 0; j < N; ++j) opened[j] = (y[j].p0 - b[2 * j]) + (y[j].p1 - b[2 * j + 1]);
    store_numbers<N>(to, opened);
}

// What bounds it: HBM (24 bytes a key or value, 32 a query), and beside it vector-ALU issue: a rotated number takes four dealer words for its
// truncation, and every number of the cache two for its mask, 18 instructions each.  A thread takes N neighbours (dimensions d ..) and the N that
// turn with them (d + rot/2 ..; the next N elsewhere), so that both multiply the same row of the tables and a number's words are drawn in step;
// N = 2 (16-byte accesses, half the addresses) where the rotated part and the rest divide into such groups: 2048 tokens of 8 + 8 + 32 heads of 128,
// 370 MB, in 73 us (5.1 TB/s) instead of 80.  Keys, values and queries have workgroups of their own, whose wavefronts then do the same.  The groups
// of a token are shared out to workgroups, or several tokens with few share one.
template <int N>
__global__ void __launch_bounds__(kAppendBlock)
cache_append_kernel(AppendArgs a, AppendShape stored, AppendShape asked, uint32_t head_inverse)
{
    const CacheView &c = a.cache;
    // Keys, then values, then queries.
    uint32_t block = blockIdx.x;
    const uint32_t kind = block < stored.blocks ? 0 : block < 2 * stored.blocks ? 1 : 2;
    block -= kind * stored.blocks;
    const AppendShape &shape = kind == 2 ? asked : stored;
    const uint32_t heads = kind == 2 ? a.q_heads : c.heads, half = a.rot / 2, groups = c.dim / (2 * N);       // of a head
    uint64_t token;
    uint32_t item;
    if (shape.per_token != 0) {
        token = block / shape.per_token;
        item = block % shape.per_token * kAppendBlock + threadIdx.x;
        if (item >= shape.groups) return;
    } else {
        const uint32_t own = threadIdx.x / shape.groups;
        if (own >= shape.together) return;
        token = (uint64_t)block * shape.together + own;
        item = threadIdx.x % shape.groups;
    }
    if (token >= a.tokens) return;
    const uint32_t head = groups == 1 ? item : __umulhi(item, head_inverse), group = item - head * groups;    // head_inverse: ceil(2^32 / groups)
    const bool turned = kind != 1 && N * group < half;
    const uint32_t d = kind == 1 ? 2 * N * group : turned ? N * group : a.rot + 2 * (N * group - half), apart = turned ? half : N;
    const uint64_t *const x[2] = {kind == 0 ? a.k[0] : kind == 1 ? a.v[0] : a.q[0], kind == 0 ? a.k[1] : kind == 1 ? a.v[1] : a.q[1]};
    const uint64_t at = (token * heads + head) * c.dim + d;
    // All that depends on the token alone is under way before any of it is looked at.
    const int64_t slot = a.slots[token], position = half != 0 ? a.positions[token] : 0;
    Pair y0[N], y1[N];
    load_numbers<N>(x, at, y0);
    load_numbers<N>(x, at + apart, y1);
    if (slot < 0 || (uint64_t)slot >= (uint64_t)c.pages * c.page) return;
    if (half != 0 && (position < 0 || (uint64_t)position >= a.table_rows)) return;
    if (turned || kind == 2) {
        int32_t cos[N] = {}, sin[N] = {};                // both are asked for before either is waited for
        if (turned) {
            const uint64_t from = position * half + N * group;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                cos[j] = a.cos[from + j];
                sin[j] = a.sin[from + j];
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            int64_t co = turned ? cos[j] : (int64_t)1 << a.frac, si = sin[j];
            if (kind == 2) {                         // the public factor goes into the table, rounded to its precision
                const int64_t round = (int64_t)1 << (a.frac - 1);
                co = (co * a.q_mul + round) >> a.frac;
                si = (si * a.q_mul + round) >> a.frac;
            }
            const uint64_t cu = (uint64_t)co, su = (uint64_t)si;
            const Pair u = y0[j], w = y1[j];
            y0[j] = Pair{u.p0 * cu - w.p0 * su, u.p1 * cu - w.p1 * su};
            y1[j] = Pair{w.p0 * cu + u.p0 * su, w.p1 * cu + u.p1 * su};
        }
        const uint64_t z = state_of(a.seedA, kTruncateWords * ((kind == 2 ? a.queries_at : 0) + at));
        truncate_numbers<N>(y0, a.frac, z);
        truncate_numbers<N>(y1, a.frac, z + (uint64_t)(kTruncateWords * apart) * kGamma);
    }
    if (kind == 2) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            uint64_t v0[N], v1[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v0[j] = p == 0 ? y0[j].p0 : y0[j].p1;
                v1[j] = p == 0 ? y1[j].p0 : y1[j].p1;
            }
            store_numbers<N>(a.qo[p] + at, v0);
            store_numbers<N>(a.qo[p] + at + apart, v1);
        }
        return;
    }
    const uint32_t page = (uint32_t)((uint64_t)slot / c.page), offset = (uint32_t)((uint64_t)slot % c.page);
    const uint64_t e = place_in_page(c, head, offset, d), z = state_of(stream_word(c.page_seeds[page], kind), 2 * e);
    uint64_t *to = (kind == 0 ? c.keys : c.values) + page * page_numbers(c) + e;
    open_numbers<N>(y0, z, to);
    open_numbers<N>(y1, z + (uint64_t)(2 * apart) * kGamma, to + apart);
}

}  // namespace hb
