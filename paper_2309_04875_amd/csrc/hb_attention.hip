// C ABI of the paged cache and its attention: argument checks, launches on the caller's stream.
#include "hb_attention.hpp"
#include "hb_check.hpp"
#include "hb_launch.hpp"

#include <algorithm>
#include <type_traits>

namespace {

// What a cache has to be, whatever is done with it.
int check_cache(const hb_cache *cache)
{
    if (cache == nullptr) return HB_EINVAL;
    if (cache->heads < 1 || cache->heads > 4096 || cache->page < 1 || cache->page > 65536 || cache->dim < 2 || cache->dim > HB_CACHE_MAX_DIM ||
        cache->dim % 2 != 0)
        return HB_EINVAL;
    if (cache->pages > ((size_t)1 << 31) - 1) return HB_EINVAL;
    const size_t tokens = cache->pages * (size_t)cache->page;             // below 2^48
    return tokens * (size_t)cache->heads <= HB_MAX_ELEMENTS / (size_t)cache->dim ? HB_OK : HB_EINVAL;
}

size_t cache_bytes(const hb_cache *cache) { return 8 * cache->pages * (size_t)cache->heads * (size_t)cache->page * (size_t)cache->dim; }

hb::CacheView view_of(const hb_cache *cache)
{
    hb::CacheView c = {};
    c.keys = (uint64_t *)cache->keys;
    c.values = (uint64_t *)cache->values;
    c.page_seeds = cache->page_seeds;
    c.pages = (uint32_t)cache->pages;
    c.heads = (uint32_t)cache->heads;
    c.page = (uint32_t)cache->page;
    c.dim = (uint32_t)cache->dim;
    return c;
}

size_t round_up(size_t n) { return (n + 255) & ~(size_t)255; }

// Workspace of hb_attention: shares of the scores, then the pieces' partial sums.  Smaller batches are cut into more pieces, so that the call itself would need
// more room for 127 sequences than for 128: what is asked for, `bytes`, is enough for every smaller batch and max_len too.
struct AttentionLayout {
    size_t scores1, parts, bytes;
    size_t score_pieces, value_pieces;                        // grids: pieces of a head, of all sequences (together != 0) or of the longest
    uint32_t least_scores, least_values, together, waves;     // as in AttentionArgs; wavefronts of a workgroup of the scores
    bool single;
};

bool attention_sizes(const hb_cache *cache, size_t batch, int q_heads, size_t max_len)
{
    return check_cache(cache) == HB_OK && q_heads >= cache->heads && q_heads <= 65536 && q_heads % cache->heads == 0 && batch <= 65535 &&
           max_len <= HB_ATTENTION_MAX_LEN && batch * q_heads * max_len <= HB_MAX_ELEMENTS;
}

// Query heads that a workgroup takes together, a power of two up to eight, and how many such chunks a head of the cache has.
int heads_together(const hb_cache *cache, int q_heads)
{
    const int group = q_heads / cache->heads, chunks = (group + 7) / 8, each = (group + chunks - 1) / chunks;
    return each <= 1 ? 1 : each <= 2 ? 2 : each <= 4 ? 4 : 8;
}
size_t head_chunks(const hb_cache *cache, int q_heads)
{
    const int group = q_heads / cache->heads, together = heads_together(cache, q_heads);
    return (size_t)((group + together - 1) / together);
}

// Wavefronts of a workgroup with so many tiles: four at least, which make the vectors faster (scores of 16 positions of one head of 80, four and
// zeros written 16 bytes at a time: 11.4 -> 8.0 us).
unsigned waves(size_t tiles) { return tiles > (size_t) hb::kAttentionWaves ? hb::kAttentionWaves : tiles < 4 ? 4 : (unsigned)tiles; }

AttentionLayout attention_layout(const hb_cache *cache, size_t batch, int q_heads, size_t max_len)
{
    AttentionLayout lay = {};
    const size_t scores = round_up(8 * batch * q_heads * max_len), numbers = q_heads * cache->dim;
    // Workgroups: two at a time for every compute unit, 512, if that gives every sequence two pieces or more (32768 positions of one sequence 183 us, with
    // 1024 194, with 256 205).  Otherwise pieces of one size, 1024 workgroups or more (64 sequences of none to 1000, four heads, cut so: 104 us, with
    // 512 116, with 2048 100, but eight of 4096 each 202 then, 190 with 1024).
    // No fewer positions than make the vectors of a workgroup's heads, which are the same for 16 positions and for 1000, worth their time (eight heads, 2048
    // positions of four sequences 48 us with 128 at least, 73 with 32; 1000 of one 33 with 64, 40 with 128, 63 with 256).
    const size_t some = batch != 0 ? batch : 1, heads = cache->heads * head_chunks(cache, q_heads), groups = some * heads;
    const int query_heads = heads_together(cache, q_heads);
    const size_t worth = query_heads < 8 ? 16 * query_heads : groups * ((max_len + 63) / 64) <= 256 ? 64 : 128;
    auto units = [](size_t n, size_t unit) { return (n + unit - 1) / unit; };
    auto size = [&](size_t workgroups) {                      // of a piece, where all sequences are of the greatest length
        const size_t each = units(max_len, units(workgroups, groups));
        return each < worth ? worth : each > hb::kMostPlaces ? hb::kMostPlaces : each;
    };
    // Up to 128 positions the values take whole sequences, and nothing is joined, where two heads make the vectors of 128 at a time (128 of one sequence, 8 heads
    // of 64, 18.3 us for 19.0; four query heads to a head 26.6 for 24.6) or where sequences are many (32 of none to 128, four to a head, 32.6 for 37.9).
    const bool joined = max_len > (query_heads <= 2 || groups >= 256 ? 128 : hb::kValueUnit * units(worth, hb::kValueUnit));
    const bool together = joined && batch <= 64 && 512 / heads >= 2 * some;
    const size_t least = together ? worth : size(1024);
    lay.least_scores = (uint32_t)units(least, hb::kScoreUnit);
    lay.least_values = (uint32_t)units(joined ? least : std::max<size_t>(max_len, 1), hb::kValueUnit);
    lay.together = together ? (uint32_t)(512 / heads) : 0;
    lay.waves = waves(units(size(512), 16));
    lay.score_pieces = units(max_len, hb::kScoreUnit * lay.least_scores);
    lay.value_pieces = units(max_len, hb::kValueUnit * lay.least_values);
    lay.single = lay.value_pieces <= 1;
    if (together) {
        // as many as are meant to be, or as one sum's most places make
        const size_t most = batch * units(max_len, hb::kMostPlaces);
        lay.score_pieces = std::min<size_t>(lay.together, batch * lay.score_pieces);
        lay.value_pieces = std::min(std::max<size_t>(lay.together, most), batch * lay.value_pieces);
    }
    lay.scores1 = scores;
    lay.parts = 2 * scores;
    // Pieces of all sequences at most, also of fewer and shorter ones: as many as are cut together (512 / heads), or 1024 / heads and one more a sequence, or as
    // one sum's most places make; a unit each at least.
    const size_t pieces = std::max(batch + units(1024, heads), batch * units(max_len, hb::kMostPlaces));
    lay.bytes = 2 * scores + round_up(16 * numbers * std::min(pieces, batch * units(max_len, hb::kValueUnit)));
    return lay;
}

// body(std::integral_constant<int, GT>) for the number of query heads a workgroup takes.
template <class Body>
void with_heads(int together, const Body &body)
{
    switch (together) {
    case 1: return body(std::integral_constant<int, 1>{});
    case 2: return body(std::integral_constant<int, 2>{});
    case 4: return body(std::integral_constant<int, 4>{});
    default: return body(std::integral_constant<int, 8>{});
    }
}

// Grids: heads of the cache (with their chunks of query heads); pieces, or sequences and pieces of each.
dim3 grid_of(size_t heads, const AttentionLayout &lay, size_t batch, size_t pieces)
{
    if (lay.together == 0) return dim3((unsigned)heads, (unsigned)batch, (unsigned)pieces);
    const size_t y = std::min<size_t>(pieces, 32768);
    return dim3((unsigned)heads, (unsigned)y, (unsigned)((pieces + y - 1) / y));
}

void launch_scores(const hb::AttentionArgs &a, int together, dim3 grid, dim3 block, hipStream_t stream)
{
    with_heads(together, [&](auto heads) {
        constexpr int GT = decltype(heads)::value;
        switch ((a.cache.dim + 63) / 64) {
        case 1: hipLaunchKernelGGL((hb::attention_scores_kernel<GT, 1>), grid, block, 0, stream, a); break;
        case 2: hipLaunchKernelGGL((hb::attention_scores_kernel<GT, 2>), grid, block, 0, stream, a); break;
        case 3: hipLaunchKernelGGL((hb::attention_scores_kernel<GT, 3>), grid, block, 0, stream, a); break;
        default: hipLaunchKernelGGL((hb::attention_scores_kernel<GT, 4>), grid, block, 0, stream, a); break;
        }
    });
}

void launch_values(const hb::AttentionArgs &a, int together, dim3 grid, hipStream_t stream)
{
    const unsigned tiles = (a.cache.dim + 15) / 16;
    grid.x *= (tiles + hb::kAttentionWaves - 1) / hb::kAttentionWaves;
    const dim3 block(64 * waves(tiles));
    with_heads(together, [&](auto heads) {
        constexpr int GT = decltype(heads)::value;
        if (GT >= 4 || a.least_values == 1) hipLaunchKernelGGL((hb::attention_values_kernel<GT, 64>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((hb::attention_values_kernel<GT, GT >= 4 ? 64 : 128>), grid, block, 0, stream, a);
    });
}

}  // namespace

extern "C" {

int hb_cache_append(const hb_cache *cache, const int64_t *k0, const int64_t *k1, const int64_t *v0, const int64_t *v1, size_t tokens,
                    const int64_t *slots, const int32_t *positions, const int32_t *cos, const int32_t *sin, size_t table_rows, int rot, int frac,
                    const int64_t *q0, const int64_t *q1, int q_heads, int32_t q_mul, uint64_t seed, int64_t *q_out0, int64_t *q_out1,
                    uint64_t *opened_bits, void *stream)
{
    int st = check_cache(cache);
    if (st != HB_OK) return st;
    if (rot < 0 || rot > cache->dim || rot % 2 != 0 || frac < 1 || frac > 30 || q_heads < 0 || q_heads > 65536) return HB_EINVAL;
    if (tokens > HB_LINEAR_MAX || table_rows > ((size_t)1 << 31) - 1) return HB_EINVAL;
    const size_t row = 8 * tokens * (size_t)cache->dim, kv = row * cache->heads, q = row * q_heads, table = 4 * table_rows * (size_t)(rot / 2);
    if (tokens != 0) {
        if (rot != 0 && table_rows == 0) return HB_EINVAL;
        const size_t store = cache_bytes(cache);
        const void *ptrs[15] = {cache->keys, cache->values, q_out0, q_out1, cache->page_seeds, k0, k1, v0, v1, slots, positions, cos, sin, q0, q1};
        const size_t sizes[15] = {store, store, q, q, 8 * cache->pages, kv, kv, kv, kv, 8 * tokens, rot != 0 ? 4 * tokens : 0, table, table, q, q};
        const unsigned align[15] = {8, 8, 8, 8, 8, 8, 8, 8, 8, 8, 4, 4, 4, 8, 8};
        st = hb::check_buffers(ptrs, sizes, align, 15);
        if (st != HB_OK) return st;
        // the rotated queries may replace the queries; every other overlap of what is written is refused
        if (!hb::outputs_disjoint(ptrs, sizes, 13, 0, 4)) return HB_EINVAL;
        for (int o = 0; o < 4 && q != 0; ++o) {
            for (int i = 13; i < 15; ++i) {
                const hb::Range a{(uintptr_t)ptrs[o], (uintptr_t)ptrs[o] + sizes[o]}, b{(uintptr_t)ptrs[i], (uintptr_t)ptrs[i] + sizes[i]};
                if (sizes[o] != 0 && !hb::disjoint(a, b) && !(o >= 2 && hb::same(a, b))) return HB_EINVAL;
            }
        }
        hb::AppendArgs a = {};
        a.cache = view_of(cache);
        a.cos = cos;
        a.sin = sin;
        a.table_rows = table_rows;
        a.q_heads = (uint32_t)q_heads;
        a.rot = (uint32_t)rot;
        a.frac = frac;
        a.q_mul = q_mul;
        // N = 2 from a workgroup for each compute unit on: below it a thread's time is the launch's (8 tokens of 48 heads of 128 4.1 us with N = 1, 4.6
        // with 2; 128 of them 8.4 and 7.8; 333 of 36 heads of 80 10.4 and 9.1).
        const uint64_t numbers = (uint64_t)tokens * (2 * (uint64_t)cache->heads + q_heads) * cache->dim;
        const int n = rot % 4 == 0 && cache->dim % 4 == 0 && numbers >= 4ull * 256 * hb::kAppendBlock ? 2 : 1, groups = cache->dim / (2 * n);      // of a head
        const uint64_t of_each = (uint64_t)cache->heads * groups, of_queries = (uint64_t)q_heads * groups, most = hb::append_launch_tokens(of_each, of_queries);
        const uint32_t head_inverse = groups == 1 ? 0 : (uint32_t)(((1ull << 32) + groups - 1) / groups);
        for (uint64_t first = 0; first < tokens; first += most) {
            const uint64_t here = std::min<uint64_t>(tokens - first, most), keys = first * cache->heads * cache->dim, queries = first * q_heads * cache->dim;
            const int64_t *const in[4] = {k0, k1, v0, v1};
            for (int p = 0; p < 2; ++p) {
                a.k[p] = (const uint64_t *)in[p] + keys;
                a.v[p] = (const uint64_t *)in[2 + p] + keys;
            }
            if (q_heads != 0) {
                a.q[0] = (const uint64_t *)q0 + queries;
                a.q[1] = (const uint64_t *)q1 + queries;
                a.qo[0] = (uint64_t *)q_out0 + queries;
                a.qo[1] = (uint64_t *)q_out1 + queries;
            }
            a.slots = slots + first;
            a.positions = rot != 0 ? positions + first : nullptr;
            a.tokens = here;
            a.seedA = hb::stream_word(seed, 1) + hb::kTruncateWords * keys * hb::kGamma;          // the state `keys` numbers on
            a.queries_at = (uint64_t)tokens * cache->heads * cache->dim + queries - keys;
            const hb::AppendShape stored = hb::append_shape(here, of_each), asked = hb::append_shape(here, of_queries);
            const dim3 grid(2 * stored.blocks + asked.blocks), block(hb::kAppendBlock);
            if (n == 2) hipLaunchKernelGGL(hb::cache_append_kernel<2>, grid, block, 0, (hipStream_t)stream, a, stored, asked, head_inverse);
            else hipLaunchKernelGGL(hb::cache_append_kernel<1>, grid, block, 0, (hipStream_t)stream, a, stored, asked, head_inverse);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return hb::fail_hip(e, "kernel launch");
        }
    }
    if (opened_bits) *opened_bits = 64ull * tokens * ((uint64_t)cache->heads * (rot + 2 * cache->dim) + (uint64_t)q_heads * cache->dim);
    return HB_OK;
}

size_t hb_attention_workspace_bytes(const hb_cache *cache, size_t batch, int q_heads, size_t max_len)
{
    return attention_sizes(cache, batch, q_heads, max_len) ? attention_layout(cache, batch, q_heads, max_len).bytes : 0;
}

int hb_attention(const hb_cache *cache, const int64_t *q0, const int64_t *q1, size_t batch, int q_heads, const int32_t *page_table,
                 size_t table_width, const int32_t *lens, size_t max_len, int k, int m, uint64_t seed, int64_t *out0, int64_t *out1,
                 void *workspace, size_t workspace_bytes, uint64_t *opened_bits, void *stream)
{
    if (!attention_sizes(cache, batch, q_heads, max_len) || !(k >= 0 && m > k && m <= 64)) return HB_EINVAL;
    if (table_width > ((size_t)1 << 31) - 1 || table_width * cache->page < max_len) return HB_EINVAL;
    const size_t scores = batch * q_heads * max_len;
    const uint64_t bits = 64ull * batch * q_heads * cache->dim * 3 + hb_opened_bits(1, k, m, scores) + 128ull * scores;
    if (batch != 0) {
        const AttentionLayout lay = attention_layout(cache, batch, q_heads, max_len);
        if (workspace_bytes < lay.bytes) return HB_EINVAL;
        const size_t q = 8 * batch * q_heads * cache->dim, store = max_len != 0 ? cache_bytes(cache) : 0;
        const void *ptrs[10] = {out0, out1, workspace, q0, q1, cache->keys, cache->values, cache->page_seeds, page_table, lens};
        const size_t sizes[10] = {q, q, lay.bytes, q, q, store, store, max_len != 0 ? 8 * cache->pages : 0, 4 * batch * table_width, 4 * batch};
        const unsigned align[10] = {8, 8, 256, 8, 8, 8, 8, 8, 4, 4};
        const int st = hb::check_buffers(ptrs, sizes, align, 10);
        if (st != HB_OK) return st;
        if (!hb::outputs_disjoint(ptrs, sizes, 10, 0, 3)) return HB_EINVAL;
        hb::AttentionArgs a = {};
        a.cache = view_of(cache);
        a.q[0] = (const uint64_t *)q0;
        a.q[1] = (const uint64_t *)q1;
        a.out[0] = (uint64_t *)out0;
        a.out[1] = (uint64_t *)out1;
        char *base = (char *)workspace;
        a.scores[0] = (uint64_t *)base;
        a.scores[1] = (uint64_t *)(base + lay.scores1);
        a.parts = (uint64_t *)(base + lay.parts);
        a.table = page_table;
        a.lens = lens;
        a.table_width = table_width;
        a.seed_q = hb_tensor_seed(seed, 0);
        a.seed_s = hb_tensor_seed(seed, 1);
        const uint64_t seed_relu = hb_tensor_seed(seed, 2);
        a.seed_p = hb_tensor_seed(seed, 3);
        a.seed_o = hb_tensor_seed(seed, 4);
        a.batch = (uint32_t)batch;
        a.q_heads = (uint32_t)q_heads;
        a.max_len = (uint32_t)max_len;
        a.least_scores = lay.least_scores;
        a.least_values = lay.least_values;
        a.together = lay.together;
        a.single = lay.single;
        const hb::GroupLauncher relu = hb::launcher_table().f[hb::kRelu][m - k - 1];
        if (relu == nullptr) return hb::fail_hip(hipErrorInvalidDeviceFunction, "no kernel was built for this slice width");
        hipError_t e = hipSuccess;
        if (max_len != 0) {
            const int together = heads_together(cache, q_heads);
            const size_t heads = cache->heads * head_chunks(cache, q_heads);                 // 2^14 at most
            launch_scores(a, together, grid_of(heads, lay, batch, lay.score_pieces), dim3(64 * lay.waves), (hipStream_t)stream);
            e = hipGetLastError();
            if (e == hipSuccess) {
                e = relu(a.scores[0], a.scores[1], scores, k, hb::stream_word(seed_relu, 0), hb::stream_word(seed_relu, 1), a.scores[0], a.scores[1],
                         (hipStream_t)stream);
            }
            if (e == hipSuccess) {
                launch_values(a, together, grid_of(heads, lay, batch, lay.value_pieces), (hipStream_t)stream);
                e = hipGetLastError();
            }
        }
        if (e == hipSuccess && !(lay.single && max_len != 0)) {
            const unsigned over = (unsigned)(((uint64_t)q_heads * cache->dim + hb::kJoinNumbers - 1) / hb::kJoinNumbers);
            hipLaunchKernelGGL(hb::attention_join_kernel, dim3(over, (unsigned)batch), dim3(hb::kJoinBlock), 0, (hipStream_t)stream, a);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return hb::fail_hip(e, "kernel launch");
    }
    if (opened_bits) *opened_bits = bits;
    return HB_OK;
}

}  // extern "C"
