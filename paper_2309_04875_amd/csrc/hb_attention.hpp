// Attention of one new token over a paged cache of masked numbers, with the reduced-ring ReLU between its two products.
#pragma once

#include "hb_cache.hpp"
#include "hb_digits.hpp"
#include "hb_kernels.hpp"

namespace hb {

struct AttentionArgs {
    CacheView cache;
    const uint64_t *q[2];                 // [batch][q_heads][dim]
    uint64_t *out[2];
    uint64_t *scores[2];                  // [batch][q_heads][max_len], workspace
    uint64_t *parts;                      // [pieces of the values][2][q_heads][dim], workspace
    const int32_t *table, *lens;          // [batch][table_width], [batch]
    uint64_t table_width;
    uint64_t seed_q, seed_s, seed_p, seed_o;
    uint32_t batch, q_heads, max_len;
    // A piece is the positions that a workgroup has: `least` units or more.  together: how many pieces all sequences are cut into; 0: every sequence by itself
    // into pieces of the least size.  single: no sequence has more than one piece of the values.
    uint32_t least_scores, least_values, together, single;
};

__device__ __forceinline__ uint32_t length_of(const AttentionArgs &a, uint32_t b)
{
    const int32_t n = a.lens[b];
    return n < 0 ? 0 : ((uint32_t)n > a.max_len ? a.max_len : (uint32_t)n);
}

// How the sequences are cut.  Their lengths are the device's alone, and max_len may be far above them: each workgroup works out for itself, a sequence a lane (64
// at most), the smallest size of a piece that makes no more than a.together pieces, and which piece is its own.  That number is what the card holds at a
// time: eight sequences of none to 4096 of 128, 32 query heads on 8, 117 us; 145 cut after max_len, where 67 pieces a head came and 64 fit (16 of two
// heads of 128 94 and 105; 128 positions of one 19.7 and 19.1: the cutting itself).  Where sequences and heads are too many, pieces are of one size, and
// begin with another sequence for every piece of the length: with the same order the longest would meet in a part of the card, since workgroups go to the
// dies and their parts in turn (sixteen sequences, two heads, 122 us, 104 so).
constexpr uint32_t kScoreUnit = 16, kValueUnit = 64;
constexpr uint32_t kMostPlaces = 1 << 12;                     // positions that one sum takes (below)

struct Cut {
    uint32_t length, upto, pieces, size;                      // a sequence's length, its pieces, and those up to and with it; positions of a piece
};
// Inclusive sums over a row of 16 lanes.
__device__ __forceinline__ uint32_t row_scan(uint32_t v)
{
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, true);       // from one lane below, two, four, eight
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, true);
    return v + __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, true);
}
template <uint32_t UNIT>
__device__ __forceinline__ Cut cut_sequences(const AttentionArgs &a, uint32_t lane, uint32_t least)
{
    const uint32_t length = lane < a.batch ? length_of(a, lane) : 0, units = (length + UNIT - 1) / UNIT;
    uint32_t pieces = units, scan = row_scan(units), each = least;
    auto row = [&](int r) { return (uint32_t)__builtin_amdgcn_readlane(scan, 16 * r + 15); };
    const uint32_t all = row(0) + row(1) + row(2) + row(3);
    if (all > each * a.together) each = __builtin_amdgcn_readfirstlane((all + a.together - 1) / a.together);
    for (;; each += each / 16 + 1) {
        const bool most = UNIT == kValueUnit && each >= kMostPlaces / UNIT;
        if (most) each = kMostPlaces / UNIT;
        if (each != 1) {
            pieces = (units + each - 1) / each;
            scan = row_scan(pieces);
        }
        const uint32_t r0 = row(0), r1 = r0 + row(1), r2 = r1 + row(2);
        if (r2 + row(3) <= a.together || most) return Cut{length, scan + (lane < 16 ? 0 : lane < 32 ? r0 : lane < 48 ? r1 : r2), pieces, each * UNIT};
    }
}

// The piece of this workgroup: positions first to end (none: nothing to do) of sequence b.  part: its number among all.
struct Piece {
    uint32_t b, length, first, end, part;
};
template <uint32_t UNIT>
__device__ __forceinline__ Piece piece_of(const AttentionArgs &a, uint32_t lane, uint32_t least)
{
    uint32_t b, length, split, size, part;
    if (a.together == 0) {
        b = (blockIdx.y + blockIdx.z) % a.batch;
        length = __builtin_amdgcn_readfirstlane(length_of(a, b));
        split = blockIdx.z;
        size = least * UNIT;
        part = split * a.batch + b;
    } else {
        const Cut cut = cut_sequences<UNIT>(a, lane, least);
        part = blockIdx.y + blockIdx.z * gridDim.y;
        b = __builtin_popcountll(__ballot(cut.upto <= part));
        if (b >= a.batch) return Piece{0, 0, 0, 0, 0};
        length = __builtin_amdgcn_readlane(cut.length, b);
        split = part - (__builtin_amdgcn_readlane(cut.upto, b) - __builtin_amdgcn_readlane(cut.pieces, b));
        size = __builtin_amdgcn_readfirstlane(cut.size);
    }
    const uint32_t first = split * size, left = first < length ? length - first : 0;
    return Piece{b, length, first, first + (left < size ? left : size), part};
}

constexpr int kAttentionBlock = 512, kAttentionWaves = kAttentionBlock / 64, kJoinBlock = 256;

// Both products of attention are sums of Beaver products of few fresh vectors with many masked numbers D = x - b of the cache.  With a = a_0 + a_1 and
// eps = (q or p) - a the two parties' sums are, their terms collected by what is read from the cache or drawn for it,
//   party 0:  sum eps (b_0 + D) + D a_0              = sum b_0 eps + D (eps + a_0)
//   party 1:  sum eps b_1 + D a_1 + (b_0 + b_1) a    = sum b_0 a   + b_1 (a + eps) + D a_1      (the last term: the dealer's triple)
// so three matrices, b_0, b_1 and D, meet two vectors for each query head, one for each party: b_0 {eps, a}, b_1 {0, a + eps}, D {eps + a_0, a_1}.
//
// In digits: sum over s of 2^(8s) of sum over i <= s of (digit i of the matrix) (digit s - i of the vectors).  Matrices are the left operands, 16
// rows a tile; the right operand has a column (s, v) for every weight 2^(8s) and vector v = party * GT + head: 16 GT columns, GT tiles.  int32 sums
// hold up to 8 x 2^14 a place and matrix: 2^12 places at most go into one.
//
// The matrices' words go in with their bytes' top bits flipped, which is a number less 0x80..80: every vector's result is owed that constant times the sum of
// its entries over the three matrices (owed[v]).
//
// Two forms.  WHOLE: a left operand is the lower (or upper) halves of four numbers as they are, four digits each, and a column holds for a number the
// digits s, s-1, s-2, s-3 of its vector (for the upper halves s-4 ..: the columns of weight 2^(8(s-4))), zeros below digit 0: planes [s][v] of four
// bytes a place.  Otherwise digit i of 16 numbers is an operand, their bytes turned before (12 instructions a number of the cache and its two
// masks, of 51), and a column holds digit s - i: planes [digit][v] of a byte a place, the columns of digit i being the planes 2 GT i further up,
// planes of zeros before the first, and tiles whose columns all have s < i left out.  WHOLE has fewer instructions, but four times the planes to
// write and to hold: it is for one or two heads at a time (32 heads of 4096 positions of 128, one query head each, 85 -> 78 us; 8192 of 8 heads 53 -> 49; eight
// sequences of none to 4096 with two 126 -> 117) and, 64 positions at a time, for the values of four (2 x 4096 of 192 110 -> 104, 4 x 1000 of 128 40 -> 39; their
// scores stay as they were, or with few positions lose: 39 -> 46).
static_assert(3ll * 8 * 128 * 128 * kMostPlaces < 1ll << 31, "sums of digit products");

template <int GT, bool WHOLE, int PLACES>
struct Planes {
    static constexpr int nv = 2 * GT, zeros = WHOLE ? GT == 1 : 16, rows = zeros + 8 * nv;          // of one matrix
    static constexpr uint32_t stride = (WHOLE ? 4 : 1) * PLACES + 16;         // (16 more: rows of 16 fall into different banks)
    static constexpr uint32_t matrix = rows * stride, bytes = 3 * matrix;
    // A lane's part of the columns: of every 64 places lane quarter g has 16 g .. 16 g + 15.
    static constexpr uint32_t per_64 = WHOLE ? 256 : 64;
    struct Column {
        const uint8_t *at, *high;             // high: for GT = 1, the column of four weights less, or zeros
        __device__ __forceinline__ Column operator+(uint32_t bytes) const { return Column{at + bytes, high + bytes}; }
    };
    static __device__ __forceinline__ Column column(const uint8_t *lds, uint32_t lane)
    {
        const uint32_t c = lane % 16, part = lane / 16 * (per_64 / 4);
        return Column{lds + c * stride + part, lds + (c < 8 ? 0 : c - 7) * stride + part};
    }

    // Place i of vector v.  Four lanes side by side have places 4 n .. 4 n + 3.
    static __device__ __forceinline__ void store(uint8_t *planes, const QuadTurn &turn, uint32_t i, uint32_t v, uint64_t x)
    {
        x += kDigitBias;
        if constexpr (WHOLE) {
            // the digits from the highest on: bytes 7 - s .. 10 - s of these eight and zeros
            const uint32_t high = __builtin_bswap32((uint32_t)(x >> 32) ^ kDigitFlip), low = __builtin_bswap32((uint32_t)x ^ kDigitFlip);
            uint8_t *to = planes + (zeros + v) * stride + 4 * i;
            const uint32_t w[8] = {low >> 24, low >> 16, low >> 8, low, __builtin_amdgcn_alignbyte(low, high, 3), __builtin_amdgcn_alignbyte(low, high, 2),
                                   __builtin_amdgcn_alignbyte(low, high, 1), high};
#pragma unroll
            for (int s = 0; s < 8; ++s) *reinterpret_cast<uint32_t *>(to + s * nv * stride) = w[s];
        } else {
            const uint32_t j = i % 4;                         // this lane writes digits j and 4 + j of all four
            uint8_t *to = planes + (zeros + j * nv + v) * stride + i - j;
            *reinterpret_cast<uint32_t *>(to) = turn((uint32_t)x) ^ kDigitFlip;
            *reinterpret_cast<uint32_t *>(to + 4 * nv * stride) = turn((uint32_t)(x >> 32)) ^ kDigitFlip;
        }
    }

    // The vectors of one query head for the three matrices, place i; what is not there is zeros.
    static __device__ __forceinline__ void store_vectors(uint8_t *lds, const QuadTurn &turn, uint32_t i, uint32_t head, uint64_t eps, uint64_t a0, uint64_t a1,
                                                         unsigned long long *owed)
    {
        store(lds, turn, i, head, eps);
        store(lds, turn, i, GT + head, a0 + a1);
        store(lds + matrix, turn, i, GT + head, a0 + a1 + eps);
        store(lds + 2 * matrix, turn, i, head, eps + a0);
        store(lds + 2 * matrix, turn, i, GT + head, a1);
        const uint64_t owed0 = quad_sum(2 * eps + a0), owed1 = quad_sum(2 * a0 + 3 * a1 + eps);
        if (i % 4 < 2) atomicAdd(&owed[i % 4 * GT + head], (unsigned long long)(kDigitBias * (i % 4 == 0 ? owed0 : owed1)));
    }

    // Zeros where no vector is: before the planes, and party 0's vectors for b_1.
    static __device__ __forceinline__ void clear(uint8_t *lds, unsigned long long *owed, uint32_t threads)
    {
        if (threadIdx.x < nv) owed[threadIdx.x] = 0;
        constexpr uint32_t row = stride / 16, before = zeros * row;
        const i32x4_t none{};
        if constexpr (zeros != 0) {
            for (uint32_t i = threadIdx.x; i < 3 * before; i += threads) *reinterpret_cast<i32x4_t *>(lds + i / before * matrix + i % before * 16) = none;
        }
        for (uint32_t i = threadIdx.x; i < 8 * GT * row; i += threads) {
            const uint32_t plane = i / row;
            *reinterpret_cast<i32x4_t *>(lds + matrix + (zeros + plane / GT * nv + plane % GT) * stride + i % row * 16) = none;
        }
    }

    typedef Flipped<4> Numbers4;
    typedef uint32_t Digits[8][4];            // otherwise: a lane's 16 numbers of a row: digit, four numbers a word

    static __device__ __forceinline__ i32x4_t operand(const uint8_t *at) { return *reinterpret_cast<const i32x4_t *>(at); }
    // sums += numbers 4 s .. 4 s + 3 (bytes flipped) of one matrix times its vectors.
    static __device__ __forceinline__ void multiply(i32x4_t (&sums)[GT], const Numbers4 &z, int s, const Column &column)
    {
        const i32x4_t low{(int)z.low[0], (int)z.low[1], (int)z.low[2], (int)z.low[3]}, high{(int)z.high[0], (int)z.high[1], (int)z.high[2], (int)z.high[3]};
        i32x4_t right[GT];
#pragma unroll
        for (int tile = 0; tile < GT; ++tile) {
            right[tile] = operand(column.at + (zeros + 16 * tile) * stride + 16 * s);
            sums[tile] = mfma_16x16x64(low, right[tile], sums[tile]);
        }
        // the upper halves meet the columns of four weights less
        if constexpr (GT == 1) {
            sums[0] = mfma_16x16x64(high, operand(column.high + 16 * s), sums[0]);
        } else {
#pragma unroll
            for (int tile = GT / 2; tile < GT; ++tile) sums[tile] = mfma_16x16x64(high, right[tile - GT / 2], sums[tile]);
        }
    }
    // The same of digits of all 16.
    static __device__ __forceinline__ void multiply(i32x4_t (&sums)[GT], const Digits &d, const Column &column)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const i32x4_t left{(int)d[i][0], (int)d[i][1], (int)d[i][2], (int)d[i][3]};
#pragma unroll
            for (int tile = 0; tile < GT; ++tile) {
                if (i * nv > 16 * tile + 15) continue;
                sums[tile] = mfma_16x16x64(left, operand(column.at + (zeros + 16 * tile - i * nv) * stride), sums[tile]);
            }
        }
    }
    static __device__ __forceinline__ void digits_at(Digits &d, int s, const Numbers4 &z)
    {
        uint32_t w[8];
        turn_bytes(z.low, w);
        turn_bytes(z.high, w + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i][s] = w[i];
    }

    // sums += the three matrices, 16 numbers a lane each, times their vectors: numbers(x) loads D, state(start, j), start being start_of(p), is that of the
    // word for number j of b_p.  both: not all of the second eight numbers meet zeros; else their words are not drawn
    // (WHOLE only; scores of 80 and 96 dimensions, calls 3 % shorter, of 32 8 %.  For the ends of sequences in the values it costs more than it saves.)
    // Words are drawn eight in step (four: 1 to 4 % slower; 16: as fast).  The loads are under way while words are drawn, but for GT = 8, where the
    // 32 registers that they hold would be the fifth wavefront's on a SIMD.
    template <class Numbers, class Start, class State>
    static __device__ __forceinline__ void multiply_three(i32x4_t (&sums)[GT], const Column &column, const Numbers &numbers, const Start &start_of,
                                                          const State &state, bool both)
    {
        uint64_t delta[16];
        Digits d;
        auto masked = [&] {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                Numbers4 z;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    z.low[j] = (uint32_t)delta[4 * s + j] ^ kDigitFlip;
                    z.high[j] = (uint32_t)(delta[4 * s + j] >> 32) ^ kDigitFlip;
                }
                if constexpr (WHOLE) multiply(sums, z, s, column + 2 * matrix);
                else digits_at(d, s, z);
            }
            if constexpr (!WHOLE) multiply(sums, d, column + 2 * matrix);
        };
        numbers(delta);
        if constexpr (GT == 8) {
            masked();
            __builtin_amdgcn_sched_barrier(0);                // D leaves its registers before words are drawn
        }
#pragma unroll 1
        for (int p = 0; p < 2; ++p) {
            uint64_t start = start_of(p);
            settle(start);                                    // (else p gamma is a product for every word)
#pragma unroll
            for (int s = 0; s < 4; s += 2) {
                if (WHOLE && s == 2 && !both) break;
                uint64_t z[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = state(start, 4 * s + j);
                Flipped<8> words;
                mix_flipped(z, words);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    Numbers4 four;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        four.low[j] = words.low[4 * x + j];
                        four.high[j] = words.high[4 * x + j];
                    }
                    if constexpr (WHOLE) multiply(sums, four, s + x, column + p * matrix);
                    else digits_at(d, s + x, four);
                }
            }
            if constexpr (!WHOLE) multiply(sums, d, column + p * matrix);
        }
        if constexpr (GT != 8) masked();
    }
};

// The weights 2^(8s) put together: value[r] of vector v = lane mod 2 GT and row 4 (lane / 16) + r, in all lanes with that v.
template <int GT>
__device__ __forceinline__ void join_digits(const i32x4_t (&sums)[GT], uint32_t lane, const unsigned long long *owed, uint64_t (&value)[4])
{
    constexpr int kPer = 16 / (2 * GT);                 // values of s in a tile
    // 2^(8 s') of this lane's s' = s mod kPer
    uint64_t weight = 1;
#pragma unroll
    for (int s = 1; s < kPer; ++s) weight = lane % 16 / (2 * GT) == s ? 1ull << (8 * s) : weight;
    if constexpr (kPer > 1) settle(weight);             // (the product does not become a shift by an amount in a vector register)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        uint64_t y = 0;
#pragma unroll
        for (int tile = 0; tile < GT; ++tile) y += (uint64_t)(int64_t)sums[tile][r] << (8 * kPer * tile);
        if constexpr (kPer > 1) y *= weight;
        if constexpr (GT <= 1) y += across<2>(y);
        if constexpr (GT <= 2) y += across<4>(y);
        if constexpr (GT <= 4) y += across<8>(y);
        value[r] = y + owed[lane % (2 * GT)];
    }
}

// After join_digits the lanes of a head, 16 / GT by four rows, hold all its rows: each takes one of them (two where there are only two lanes, GT = 8).
template <int GT>
struct RowShare {
    static constexpr int kRows = GT == 8 ? 2 : 1;
    uint32_t part;
    bool any, party1;
    __device__ __forceinline__ explicit RowShare(uint32_t lane) : part(lane % 16 / GT), any(lane % 16 / GT * kRows < 4), party1((lane & GT) != 0) {}
    __device__ __forceinline__ uint32_t row(int x) const { return part * kRows + x; }
    // mine: the values of this lane's party, other: those of the other one's
    __device__ __forceinline__ Pair pick(int x, const uint64_t (&mine)[4], const uint64_t (&other)[4]) const
    {
        const uint32_t at = row(x);
        const Pair y{at == 0 ? mine[0] : at == 1 ? mine[1] : at == 2 ? mine[2] : mine[3],
                     at == 0 ? other[0] : at == 1 ? other[1] : at == 2 ? other[2] : other[3]};
        return party1 ? Pair{y.p1, y.p0} : y;
    }
};

// An output's sum divided by the length (the same for the whole wavefront): a truncation by its whole bits, a factor in (1/2, 1] for the rest.
__device__ __forceinline__ Pair finish_output(const AttentionArgs &a, uint64_t i, uint32_t length, Pair sum)
{
    if (length == 0) return Pair{0, 0};
    const uint64_t z = state_of(a.seed_o, 9 * i), c0 = mix64(z);
    const int whole = 31 - __builtin_clz(length);
    const uint64_t factor = ((1ull << (16 + whole)) + length / 2) / length;
    const Pair o = truncate_drawn(Pair{sum.p0 + c0, sum.p1 - c0}, 16 + whole, z + kGamma);
    return truncate_drawn(Pair{o.p0 * factor, o.p1 * factor}, 16, z + 5 * kGamma);
}

// Where a position of a sequence lies: its page, or -1 for one behind the end and for a hole.
__device__ __forceinline__ int64_t page_of(const AttentionArgs &a, uint32_t b, uint32_t t, uint32_t length)
{
    if (t >= length) return -1;
    const int64_t page = a.table[b * a.table_width + t / a.cache.page];
    return page < (int64_t)a.cache.pages ? page : -1;
}

// What a workgroup works on beside its piece: a head of the cache and up to GT of its query heads.
struct HeadChunk {
    uint32_t head, first, count;          // query heads first .. first + count - 1
};
template <int GT>
__device__ __forceinline__ HeadChunk head_chunk(const AttentionArgs &a, uint32_t index)
{
    const uint32_t group = a.q_heads / a.cache.heads, chunks = (group + GT - 1) / GT;
    const uint32_t chunk = index % chunks, head = index / chunks, left = group - chunk * GT;
    return HeadChunk{head, head * group + chunk * GT, left < GT ? left : GT};
}

// Scores.  A wavefront takes 16 positions at a time: a row of its tile is a key, lane l has row l mod 16 and of every 64 dimensions the pairs
// 8 j + 2 (l / 16), j = 0 .. 7 (the lanes of a row read 64 bytes side by side).
// What bounds it: vector-ALU issue, and the matrix instructions, which overlap little with it: of a key's number 34 instructions are its two dealer words, and a
// score takes five more.  32768 positions of 8 heads of 128, four query heads each, 268 MB: 81 us; 81 also with all loads from one row.
template <int GT, int ND>
__global__ void __launch_bounds__(kAttentionBlock, 4)
attention_scores_kernel(AttentionArgs a)
{
    using P = Planes<GT, (GT <= 2 && GT * ND < 8), 64 * ND>;     // two workgroups' on a compute unit
    __shared__ __align__(16) uint8_t lds[P::bytes];
    __shared__ unsigned long long owed[2 * GT];
    const CacheView &c = a.cache;
    const HeadChunk h = head_chunk<GT>(a, blockIdx.x);
    const uint32_t threads = blockDim.x;                      // from 256 to kAttentionBlock
    const uint32_t lane = threadIdx.x % 64, g = lane / 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Piece piece = piece_of<kScoreUnit>(a, lane, a.least_scores);
    const uint32_t first = piece.first, end = piece.end;
    if (first >= end || c.pages == 0) return;                 // (no score of a position without a key is used)
    const uint64_t row0 = (uint64_t)piece.b * a.q_heads + h.first;
    // The queries' numbers, one a thread, in the order of their bytes in the planes: four consecutive ones are two pairs of dimensions.  A thread's first
    // is under way before anything is waited for.
    constexpr uint32_t kNumbers = GT * ND * 64;
    uint64_t q0, q1;
    auto head_of = [](uint32_t i) { return i / (ND * 64); };
    auto dimension = [](uint32_t i) { return i / 16 % (4 * ND) * 16 + i / 4 % 4 * 2 + 8 * (i / 2 % 2) + i % 2; };
    auto asked = [&](uint32_t i) { return head_of(i) < h.count && dimension(i) < c.dim; };
    auto load_number = [&](uint32_t i) {
        const uint64_t at = asked(i) ? (row0 + head_of(i)) * c.dim + dimension(i) : 0;
        q0 = a.q[0][at];
        q1 = a.q[1][at];
    };
    load_number(threadIdx.x < kNumbers ? threadIdx.x : 0);
    // The keys of 16 positions, a row each.  One without a key reads the first one's: its score is not used.
    uint64_t there = 0, seed = 0, place = 0;
    const uint64_t *keys = nullptr;
    auto look_up = [&](uint32_t t0) {
        const int64_t page = page_of(a, piece.b, t0 + lane % 16, end);
        there = __ballot(page >= 0);
        place = page >= 0 ? place_in_page(c, h.head, (t0 + lane % 16) % c.page, 0) : 0;
        keys = c.keys + (page >= 0 ? page : 0) * page_numbers(c) + place;
        seed = c.page_seeds[page >= 0 ? page : 0];
    };
    if (first + 16 * wave < end) look_up(first + 16 * wave);
    P::clear(lds, owed, threads);
    __syncthreads();
    const QuadTurn turn(lane);
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < kNumbers; i += threads) {
        if (i >= threads) load_number(i);
        uint64_t w[2] = {state_of(a.seed_q, 2 * ((row0 + head_of(i)) * c.dim + dimension(i)))};
        w[1] = w[0] + kGamma;
        w[0] = asked(i) ? mix64(w[0]) : 0;
        w[1] = asked(i) ? mix64(w[1]) : 0;
        const uint64_t eps = asked(i) ? (q0 - w[0]) + (q1 - w[1]) : 0;                     // opened
        P::store_vectors(lds, turn, i / 64 % ND * 64 + i / 4 % 4 * 16 + i / 16 % 4 * 4 + i % 4, head_of(i), eps, w[0], w[1], owed);
    }
    __syncthreads();
    const typename P::Column column = P::column(lds, lane);
    const uint32_t chunks = (c.dim + 63) / 64;
    for (uint32_t t0 = first + 16 * wave; t0 < end; t0 += threads / 4) {
        if (t0 != first + 16 * wave) look_up(t0);
        uint64_t z0 = state_of(stream_word(seed, 0), 2 * (place + 2 * g));
        i32x4_t sums[GT] = {};
        typename P::Column at = column;
#pragma unroll 1
        for (uint32_t chunk = 0; chunk < chunks; ++chunk) {
            auto numbers = [&](uint64_t (&delta)[16]) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint32_t dim = 64 * chunk + 8 * j + 2 * g;
                    dim = dim < c.dim ? dim : c.dim - 2;          // behind the last dimension the vectors are zeros
                    const U64x2 v = load_stream2(keys + dim);
                    delta[2 * j] = v.a;
                    delta[2 * j + 1] = v.b;
                }
            };
            auto start_of = [&](int p) { return p == 0 ? z0 : z0 + kGamma; };
            auto state = [&](uint64_t start, int j) { return start + (uint64_t)(2 * (8 * (j / 2) + j % 2)) * kGamma; };
            P::multiply_three(sums, at, numbers, start_of, state, 64 * chunk + 32 < c.dim);
            z0 += 128 * kGamma;
            at = at + P::per_64;
        }
        uint64_t mine[4], other[4];
        join_digits<GT>(sums, lane, owed, mine);
#pragma unroll
        for (int r = 0; r < 4; ++r) other[r] = across<GT>(mine[r]);
        uint32_t l = lane;
        settle(l);                                            // (nothing of this stays in registers from tile to tile)
        const uint32_t head = l % GT;
        const RowShare<GT> own(l);
        if (!own.any || head >= h.count) continue;
#pragma unroll
        for (int x = 0; x < RowShare<GT>::kRows; ++x) {
            const uint32_t at = t0 + 4 * (l / 16) + own.row(x);
            if (at >= end) continue;
            const uint64_t j = (row0 + head) * a.max_len + at;
            Pair score{0, 0};
            if ((uint32_t)there >> (at - t0) & 1) {
                const Pair y = own.pick(x, mine, other);
                const uint64_t z = state_of(a.seed_s, 5 * j), c0 = mix64(z);
                score = truncate_drawn(Pair{y.p0 + c0, y.p1 - c0}, 16, z + kGamma);
            }
            a.scores[0][j] = score.p0;
            a.scores[1][j] = score.p1;
        }
    }
}

// The product with the values.  A wavefront has 16 dimensions, the rows of its tile, and lane l takes 16 of every 64 positions; the workgroup, up to 128 dimensions,
// makes the weights' vectors of CHUNK positions at a time.
// What bounds it: as above, without the five words and the turned bytes (WHOLE); the same 32768 positions 81 us, 74 with all loads from one row.
template <int GT, int CHUNK>
__global__ void __launch_bounds__(kAttentionBlock, 4)
attention_values_kernel(AttentionArgs a)
{
    const uint32_t threads = blockDim.x;                      // 64 for every 16 dimensions, 256 at least
    using P = Planes<GT, (GT <= 4), CHUNK>;
    __shared__ __align__(16) uint8_t lds[P::bytes];
    __shared__ unsigned long long owed[2 * GT];
    __shared__ uint64_t row_at[CHUNK], row_state[CHUNK];      // a position's numbers and masks
    const CacheView &c = a.cache;
    const uint32_t halves = (c.dim + kAttentionWaves * 16 - 1) / (kAttentionWaves * 16);       // a workgroup each
    const HeadChunk h = head_chunk<GT>(a, blockIdx.x / halves);
    const uint32_t lane = threadIdx.x % 64, g = lane / 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Piece piece = piece_of<kValueUnit>(a, lane, a.least_values);
    const uint32_t first = piece.first, end = piece.end;
    if (first >= end && (piece.length != 0 || !a.single)) return;          // the join does not read it
    const uint64_t row0 = (uint64_t)piece.b * a.q_heads + h.first;
    const uint32_t dim0 = blockIdx.x % halves * (kAttentionWaves * 16) + 16 * wave, dim = dim0 + lane % 16 < c.dim ? dim0 + lane % 16 : 0;
    const typename P::Column column = P::column(lds, lane);
    P::clear(lds, owed, threads);
    __syncthreads();
    const uint64_t z = (uint64_t)(2 * dim) * kGamma;
    const QuadTurn turn(lane);
    i32x4_t sums[GT] = {};
    // What a thread needs for the next chunk's vectors is under way while this one's are multiplied: the weight's shares, the position's page, that page's
    // seed, and the page of the chunk after it.  (For GT = 8 there are no registers for that.)
    constexpr bool kEarly = GT < 8;
    const uint32_t my_place = threadIdx.x % CHUNK;            // the place in the chunk of every number that this thread makes
    int32_t page = -1, next_page = -1;
    uint64_t p0 = 0, p1 = 0, seed = 0;
    auto find = [&](uint32_t t0) { return (int32_t)page_of(a, piece.b, t0 + my_place, end); };
    auto weight_at = [&](uint32_t i, uint32_t t0) {
        const bool asked = i / CHUNK < h.count && t0 + my_place < end;
        return (row0 + (asked ? i / CHUNK : 0)) * a.max_len + (asked ? t0 + my_place : first);
    };
    auto load_weight = [&](uint32_t i, uint32_t t0) {
        const uint64_t n = weight_at(i, t0);
        p0 = a.scores[0][n];
        p1 = a.scores[1][n];
    };
    auto load_seed = [&] {
        if (threadIdx.x < CHUNK && page >= 0) seed = c.page_seeds[page];
    };
    page = find(first);
    if constexpr (kEarly) {
        load_weight(threadIdx.x, first);
        next_page = find(first + CHUNK);
    }
    load_seed();
    for (uint32_t t0 = first; t0 < end; t0 += CHUNK) {
        uint32_t thread = threadIdx.x;
        settle(thread);                                       // what follows from it is not kept in registers from chunk to chunk
#pragma unroll 1
        for (uint32_t i = thread; i < GT * CHUNK; i += threads) {
            if (!kEarly || i >= threads) load_weight(i, t0);
            const bool there = page >= 0 && i / CHUNK < h.count;
            const uint64_t s = state_of(a.seed_p, 2 * weight_at(i, t0)), a0 = there ? mix64(s) : 0, a1 = there ? mix64(s + kGamma) : 0;
            const uint64_t eps = there ? (p0 - a0) + (p1 - a1) : 0;                        // opened
            P::store_vectors(lds, turn, i % CHUNK, i / CHUNK, eps, a0, a1, owed);
        }
        if (thread < CHUNK) {
            const uint64_t place = place_in_page(c, h.head, (t0 + thread) % c.page, 0);
            row_at[thread] = page >= 0 ? page * page_numbers(c) + place : 0;  // without a value: the first one's, times zeros
            row_state[thread] = page >= 0 ? state_of(stream_word(seed, 1), 2 * place) : 0;
        }
        if (t0 + CHUNK < end) {
            if constexpr (kEarly) {
                page = next_page;
                load_weight(thread, t0 + CHUNK);
                next_page = find(t0 + 2 * CHUNK);
            } else {
                page = find(t0 + CHUNK);
            }
            load_seed();
        }
        __syncthreads();
        for (uint32_t block = 0; block < CHUNK / 64 && t0 + 64 * block < end && c.pages != 0 && dim0 < c.dim; ++block) {
            auto numbers = [&](uint64_t (&delta)[16]) {
#pragma unroll
                for (int j = 0; j < 16; ++j) delta[j] = load_stream(c.values + row_at[64 * block + 16 * g + j] + dim);
            };
            auto start_of = [&](int p) { return p == 0 ? z : z + kGamma; };
            auto state = [&](uint64_t start, int j) { return row_state[64 * block + 16 * g + j] + start; };
            P::multiply_three(sums, column + P::per_64 * block, numbers, start_of, state, true);
        }
        __syncthreads();
    }
    // Of each number and party one partial sum, or the result where there is one split.
    uint32_t l = lane;
    settle(l);
    const uint32_t head = l % GT;
    const bool party1 = (l & GT) != 0;
    uint64_t y[4];
    join_digits<GT>(sums, lane, owed, y);
    if (!a.single) {
        if (l % 16 >= (2 * GT) || head >= h.count) return;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t to = dim0 + 4 * (l / 16) + r;
            if (to < c.dim) a.parts[((2 * (uint64_t)piece.part + party1) * a.q_heads + h.first + head) * c.dim + to] = y[r];
        }
        return;
    }
    uint64_t other[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) other[r] = across<GT>(y[r]);
    const RowShare<GT> mine(l);
    if (!mine.any || head >= h.count) return;
#pragma unroll
    for (int x = 0; x < RowShare<GT>::kRows; ++x) {
        const Pair sum = mine.pick(x, y, other);
        const uint32_t to = dim0 + 4 * (l / 16) + mine.row(x);
        if (to >= c.dim) continue;
        const uint64_t i = (row0 + head) * c.dim + to;
        const Pair o = finish_output(a, i, piece.length, sum);
        a.out[0][i] = o.p0;
        a.out[1][i] = o.p1;
    }
}

// Joins a sequence's pieces and divides by the length.  32 numbers a workgroup, whose pieces eight threads each share out: a launch and one chain of loads, 4 to 5 us.
constexpr int kJoinNumbers = 32, kJoinShares = kJoinBlock / kJoinNumbers;

__global__ void __launch_bounds__(kJoinBlock)
attention_join_kernel(AttentionArgs a)
{
    __shared__ uint64_t partial[2][kJoinShares][kJoinNumbers];
    const uint64_t per = (uint64_t)a.q_heads * a.cache.dim;
    const uint32_t b = blockIdx.y, x = threadIdx.x % kJoinNumbers, share = threadIdx.x / kJoinNumbers, at = blockIdx.x * kJoinNumbers + x;
    const uint64_t i = b * per + at;
    uint32_t length, pieces, from, step;                      // the sequence's pieces: from, from + step, ..
    if (a.together == 0) {
        const uint32_t size = a.least_values * kValueUnit;
        length = __builtin_amdgcn_readfirstlane(length_of(a, b));
        pieces = (length + size - 1) / size;
        from = b;
        step = a.batch;
    } else {
        const Cut cut = cut_sequences<kValueUnit>(a, threadIdx.x % 64, a.least_values);
        length = __builtin_amdgcn_readlane(cut.length, b);
        pieces = __builtin_amdgcn_readlane(cut.pieces, b);
        from = __builtin_amdgcn_readlane(cut.upto, b) - pieces;
        step = 1;
    }
    Pair o{0, 0};
    if (at < per) {
        for (uint32_t s = share; s < pieces; s += kJoinShares) {
            const uint64_t part = 2 * (uint64_t)(from + s * step) * per + at;
            o.p0 += a.parts[part];
            o.p1 += a.parts[part + per];
        }
    }
    partial[0][share][x] = o.p0;
    partial[1][share][x] = o.p1;
    __syncthreads();
    if (share != 0 || at >= per) return;
    o = Pair{0, 0};
#pragma unroll
    for (int s = 0; s < kJoinShares; ++s) {
        o.p0 += partial[0][s][x];
        o.p1 += partial[1][s][x];
    }
    o = finish_output(a, i, length, o);
    a.out[0][i] = o.p0;
    a.out[1][i] = o.p1;
}

}  // namespace hb
