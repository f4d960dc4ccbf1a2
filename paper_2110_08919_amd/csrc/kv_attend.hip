// Attention of new tokens over a key-value cache held as codes: o = sum_j softmax_j(scale q . x^_j) y^_j over the tokens
// of all pages of a sequence, or of listed ones.
//
// Mathematics.  A key reads back as x^_i = k_i + (c_i + 1/2) s_i, so q . x^ = sum_i (q_i s_i) c_i + sum_i q_i (k_i + s_i / 2).
// The second sum is the same for every token and drops out of the softmax: the query takes the steps, and the codes enter
// the products as the integers they are.  Likewise o_i = k_i + s_i (1/2 + sum_j p_j c_ji / sum_j p_j).
//
// Scores on the int8 matrix instruction (16x16x64), so that key codes need no conversion: a row of q' = q s is rounded to
// Q = rint(q' Qmax / max |q'|) and split into signed digits of 8 bits, one product each, summed exactly in int32: two digits for
// bfloat16, three for float16, four for float32, so that features far below the row's largest keep the bits their type has
// (query_digits).
// Weights exp2(t - m) are rounded to fp16 (float32 calls: two fp16 terms) and multiply the value codes, which fp16 holds
// exactly, on the fp16 matrix instruction with float32 sums.  To float16 results that is an error like that of their own rounding, 1.3e-4 of the
// root mean square at most beside 2.1e-4; two terms would take 3 to 15 % more time wherever the vector pipe is the bound (8 heads
// of 128 on 4-bit codes, 32 float16 rows each: 222 us for 191).  The sum of weights is taken of the rounded ones, as their product
// with ones: a sixteenth of what it takes the vector pipe.  m is a
// maximum that may lag behind by 2 (weights are lifted by 2^13, reach 2^15, and are rounded to 2^-24 at the small end, 2^-37 of
// the largest token's): it moves, and the sums are rescaled, only in tiles where a score passes it by more.
//
// Layout.  Tokens are the rows of the first product (S^T = K Q^T) and the summed index of the second (O^T = V^T P^T), so
// the registers that hold scores of a token group are the operand of the second product as they are: register j of lane
// (n, g) holds query row n and token 4 g + j of its group of 16, and the second product takes its 8 tokens per lane as
// 4 g .. 4 g + 3 of two groups.  A lane owns dpad / 16 neighbouring features of the values: it loads them from the rows
// of its 8 tokens and gathers the operand of each with byte permutes.  Nothing goes through LDS until the end.  Each wave
// walks its own tiles of 32 or 64 tokens with the next tile's loads in flight.
//
// Bound by reading keys and values once.  Measured, heads of 128, bfloat16: 64 sequences of 32 000 to 56 000 tokens, 8 heads of 8
// query rows (5.75 GB): 967 us, 5.95 TB/s where a plain streaming read has 6.16; 32 of 1000 to 8000, 8 heads of 4 rows (298 MB): 59 us,
// 5.0 TB/s.  Many query rows, float32 queries and packed codes are bound by the vector pipe (scores to weights, codes to fp16): 48
// bfloat16 rows on 3 heads of 128 at 4 bits, 32 sequences of 15 000 to 32 000 tokens: 128 us where reading takes 48.  Small calls are round trips to memory one behind the
// other, with few tiles to a wave between them: arguments, lengths, page numbers, keys, and at the end LDS, the part or the output, and the
// join (4 to 6 us): 64 chosen pages of 64 tokens, 8 heads: 9.4 us; 4 sequences of up to 300 tokens, 12 heads of 64: 8.6; 48 float32 rows on
// one head of 192, 4 bits, 8 sequences of 3500 to 9000 tokens: 18.8; 256 pages of 32, 4 bits, 16 sequences of 4 heads of 96, 6 float16 rows
// each: 21.2.
#include <algorithm>
#include <type_traits>

#include "kv_internal.h"
#include "wave_ops.h"

namespace lpq {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int THREADS = 256, WAVES = 4;
constexpr float NEG = -INFINITY;
// Not more, also where it would take less time (bfloat16 rows with a mask by 6, so to 2^-33: 32 trees on 96 rows a head 161 us by 2, 154 by 6): what a token
// sees does not say how exact its weights are.
constexpr float HEADROOM = 2.0f;     // how far scores may pass the maximum before it moves (powers of two)
constexpr float LIFT = 13.0f;        // weights are exp2(t - m + LIFT): at most 2^15, and fp16 holds them to 2^-37 of the largest
constexpr float FAR = 1024.0f;       // maxima beyond it are subtracted from the scores before these are multiplied by their scale
constexpr float MAXIMUM = 0x1p-48f;  // maxima that go from wave to wave and from part to part are times this: finite for any query and scale
__device__ __forceinline__ float lag(float m, float top) { return top == NEG ? 1.0f : __builtin_amdgcn_exp2f((m - top) * (1.0f / MAXIMUM)); }

// Digits of 8 bits that hold a row of queries.  Rounded to 2^-16 of the row's largest q' a bfloat16 value keeps its 8 bits down to 2^-8 of the
// largest, to 2^-24 a float16 value its 11 down to 2^-13, to 2^-32 a float32 value its 24 down to 2^-8.  Keys of 128 features, one of them 20 (100)
// times as wide, scores of standard deviation 8, error of the result before it is rounded, of its root mean square: float16 in two digits
// 4.1e-4 (5.6e-4), in three 0.7e-4 (0.8e-4), all of it the weights' (its own rounding: 2.1e-4); bfloat16 in two 3.1e-4 (4.6e-4; 1.6e-3); float32 in
// three up to 1.5 times that of scores in float32, in four below it.  Time, 16 conversations of 32 000 to 56 000 tokens, 8 heads of 128: up to 16 rows
// the same, bound by memory; 32 float32 rows on 4-bit codes 220 us in three digits, 237 in four, in heads of 256 on 8-bit codes 577, 670;
// 32 float16 rows on 4-bit codes, for which registers then do not hold two row tiles, 152 in two, 191 in three.
__host__ __device__ constexpr int query_digits(int type) { return type == LPQ_TYPE_BF16 ? 2 : type == LPQ_TYPE_F16 ? 3 : 4; }
// Tokens a wave has in registers: 64 where a row of codes has at
// most 64 bytes, else 32.
__host__ __device__ constexpr int tile_tokens(int dpad, bool packed) { return (packed ? dpad / 2 : dpad) <= 64 ? 64 : 32; }
// Whether there is a kernel that takes more than 16 query rows through a tile of tokens 32 at a time: codes are unpacked and made fp16 once
// for 32 rows.  16 conversations of 32 000 to 56 000 tokens, 8 heads of 128, 32 rows each, 32 against 16 at a time, us: bfloat16 161, 200 on
// 4-bit codes, 274, 322 on 8-bit codes, float32 287, 343 on 8-bit codes; heads of 256, bfloat16 511, 594.  Not so for 4-bit codes in heads of
// 192 (298, 273), whose 32 rows leave one workgroup to a CU, and where three or four digits leave too few registers: 4-bit codes in heads of
// more than 64 (float16 rows of 256: 453, 457), float32 rows in heads of 192 (470, 448) and 256.
// Nor for trees, float16 in heads of 256 on 8-bit codes: 32 rows would have 10 registers in scratch.
__host__ __device__ constexpr bool two_row_tiles(int dpad, bool packed, int type, bool tree)
{
    if (tree && dpad == 256 && !packed && type == LPQ_TYPE_F16) return false;
    if (packed) return dpad == 64 || (type == LPQ_TYPE_BF16 && dpad != 192);
    return dpad < 192 || type != LPQ_TYPE_F32;
}
// Whether a call is long enough for it, in tokens of all (sequence, head) as the table has room for.  One tile is twice the time then, which
// short calls wait for: 8 heads of 128, 32 bfloat16 rows, 4000 to 8000 tokens, 32 against 16 at a time, us: 1 conversation 16.5, 14.0, 4 20.9,
// 20.6, 8 27.3, 28.2, 16 47, 54; on 4-bit codes 15.1, 12.7, 21.0, 19.2, 26.7, 24.4, 36, 38; heads of 256 22, 17, 33, 28, 52, 52, 100, 105.
constexpr int64_t TWO_ROW_TOKENS = int64_t(1) << 19;
// Workgroups of four waves that a CU's registers hold.  Compiled so, no kernel has vector registers in scratch (three go to accumulation
// registers where 32 rows of 256 bfloat16 features are taken); 47 to 83 scalar registers live in lanes of vector registers, nearly all of them what
// is the same for a whole run, outside the loop over tiles.
// With a window, four workgroups of bfloat16 rows of 128 features would have 3 registers in scratch.
__host__ __device__ constexpr int blocks_per_cu(int dpad, bool packed, int rt, int type, bool window)
{
    if (window && dpad == 128 && !packed && rt == 1) return 3;
    if (dpad > 128) return rt == 1 && !(dpad > 192 && type == LPQ_TYPE_F32) ? 2 : 1;
    if (rt > 1) return 2;
    if (type == LPQ_TYPE_F32) return 3;
    return dpad > 64 && (packed || type == LPQ_TYPE_F16) ? 3 : 4;
}

// Positions of sequence b that exist, and tiles of tokens a call goes through for it: at least one, so that a sequence
// without tokens has its zeros written too.
__device__ __forceinline__ int length_of(const KvView &kv, const KvAttend &a, int len)
{
    const int room = a.table_pages << kv.page_shift;       // below 2^31
    return len < 0 ? 0 : (len > room ? room : len);
}
__device__ __forceinline__ int tiles_of(const KvView &kv, const KvAttend &a, int given, int tile)
{
    int len = length_of(kv, a, given);
    if (a.chosen && len > 0) len = a.n_select << kv.page_shift;
    const int tiles = (int)(((unsigned)len + tile - 1) / tile);
    return tiles < 1 ? 1 : tiles;
}

// With a window: what the rows of one row tile, new tokens [from, to], can see of a sequence, in groups of 16 positions: the first
// `sink` groups, then those from `low` on, `groups` in all.
struct RowTokens {
    int from, to;
};
struct Span {
    int sink, low, groups;
};
__device__ __forceinline__ RowTokens row_tokens(const KvQueries &q, int row0, int tile_rows)
{
    const int rows = q.new_tokens * q.group, end = row0 + tile_rows < rows ? row0 + tile_rows : rows;
    return {__builtin_amdgcn_readfirstlane(row0 / q.group), __builtin_amdgcn_readfirstlane((end - 1) / q.group)};
}
// The first position that a token at position `me` has in its window.
__device__ __forceinline__ int window_from(const KvWindow &a, int me)
{
    const int first = me < 0 ? 0 : me + 1 - a.window;
    return first < 0 ? 0 : first;
}
__device__ __forceinline__ Span span_of(const KvWindow &a, const KvQueries &q, RowTokens t, int len)
{
    const int end = len - q.new_tokens + t.to + 1, above = end < 0 ? 0 : end;
    Span s;
    s.low = window_from(a, len - q.new_tokens + t.from) >> 4;
    const int sinks = a.sinks < above ? a.sinks : above;
    s.sink = (int)(((unsigned)sinks + 15) >> 4);
    if (s.sink > s.low) s.sink = s.low;
    s.groups = above ? s.sink + (int)(((unsigned)above + 15) >> 4) - s.low : 0;
    return s;
}
template <typename CALL>
__device__ __forceinline__ int tiles_seen(const KvView &kv, const KvQueries &q, const CALL &a, RowTokens t, int given, int tile)
{
    if constexpr (std::is_same<CALL, KvWindow>::value) {
        if (!a.chosen) {
            const int per = tile >> 4, tiles = (span_of(a, q, t, length_of(kv, a, given)).groups + per - 1) / per;
            return tiles < 1 ? 1 : tiles;
        }
    }
    return tiles_of(kv, a, given, tile);
}

// How the tiles of all (sequence, head), of all pairs for short, are dealt to the workgroups.  Where a head's rows take several
// row tiles, as many workgroups have the same share, next to each other on one XCD (workgroups are dealt to the 8 of them in
// turn), so that what one of them reads the others find in its L2.
//   Long calls: one behind the other in equal runs.  A run ends where it ends: what a workgroup has of a pair that began before
//   its run or goes on after it is a part, at most two per workgroup.
//   Short calls (runs below CROSSING tiles), where going over to another pair costs as much as the run itself: a workgroup
//   has one pair or an even part of one.
// kv_join_kernel joins a pair's parts.  Fewer than 2^31 tiles (kv_attend_plan).
// CROSSING: attention and join, equal runs against even parts, us, 8 heads of 128, 8 bfloat16 rows each, tables of 32 000 to 56 000 tokens:
// 4 conversations (runs of 43 tiles) 80, 76, 8 (86) 141, 137, 16 (172) 263, 262, 24 (258) 384, 386, 32 (344) 505, 517, 64 (690) 962, 1028; of 900 to
// 8000 tokens, 4 rows: 64 (71) 118, 114; of 4000 to 32 000: 48 (211) 310, 313, 96 (422) 608, 633.
constexpr unsigned CROSSING = 200;
struct Place {
    int b, pair, tile, tiles;      // sequence, head, tile of it, tiles of the sequence
    int run;                       // tiles of the workgroup
    int whole;                     // tiles of every workgroup that has a part of this pair, but the last
};
// Where a pair's parts are, with r row tiles: part 0 of row tile t in slot 2 (first r + t) + 1, part u > 0 in 2 ((first + u) r + t).
struct Parts {
    int first, count;
};
// Every wave for itself: a lane adds up some neighbouring sequences, the lanes' sums are scanned, the lane whose sequences
// hold the workgroup's first tile (or part) finds it.
template <typename CALL>
__device__ __forceinline__ bool first_place(const KvView &kv, const KvQueries &q, const CALL &a, RowTokens rows, unsigned me, unsigned of, int tile,
                                            int least, unsigned crossing, Place &out)
{
    auto tiles_of = [&](int b) { return tiles_seen(kv, q, a, rows, a.lengths[b], tile); };
    const int lane = threadIdx.x & 63, pairs = kv.heads;      // of a sequence
    const int per = (a.nseq + 63) / 64, b0 = lane * per, b1 = b0 + per < a.nseq ? b0 + per : a.nseq;
    unsigned mine = 0;
#pragma unroll 4
    for (int b = b0; b < b1; ++b) mine += (unsigned)tiles_of(b);
    unsigned upto = wave_scan(mine);
    const unsigned total = (unsigned)__builtin_amdgcn_readlane((int)upto, 63) * pairs, all_pairs = (unsigned)a.nseq * pairs;
    unsigned run = (total + of - 1) / of;
    const bool apart = run < crossing && all_pairs < of;
    if (apart) {
        // The smallest run whose parts fit the grid, or nearly: at least total / of, and every pair rounds its number of parts up
        // by less than one, so that total / (of - all_pairs) is enough.
        unsigned enough = (total + of - all_pairs - 1) / (of - all_pairs);
        for (int i = 0; i < 4 && run + 1 < enough; ++i) {
            const unsigned mid = (run + enough) / 2;
            unsigned parts = 0;
            for (int b = b0; b < b1; ++b) parts += ((unsigned)tiles_of(b) + mid - 1) / mid;
            if ((unsigned)__builtin_amdgcn_readlane((int)wave_scan(parts), 63) * pairs <= of) enough = mid;
            else run = mid + 1;
        }
        run = enough;
    }
    if (run < (unsigned)least) run = least;
    run = __builtin_amdgcn_readfirstlane((int)run);
    auto weight = [&](unsigned tiles) { return apart ? (tiles + run - 1) / run : tiles; };
    if (apart) {
        mine = 0;
        for (int b = b0; b < b1; ++b) mine += weight((unsigned)tiles_of(b));
        upto = wave_scan(mine);
    }
    const uint64_t from64 = apart ? (uint64_t)me : (uint64_t)run * me;
    if (from64 >= (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)upto, 63) * pairs) return false;
    const unsigned from = (unsigned)from64;
    const int who = __ffsll((unsigned long long)__ballot(from < upto * pairs)) - 1;      // the first lane that reaches beyond it
    unsigned left = from - (upto - mine) * pairs;
    int b = b0, tiles = 1;
    if (lane == who) {
        for (; b < b1; ++b) {
            tiles = tiles_of(b);
            const unsigned w = weight((unsigned)tiles) * pairs;
            if (left < w) break;
            left -= w;
        }
    }
    out.b = __builtin_amdgcn_readlane(b, who);
    out.tiles = __builtin_amdgcn_readlane(tiles, who);
    left = __builtin_amdgcn_readlane((int)left, who);
    // (divisions leave their results in vector registers)
    const unsigned each = __builtin_amdgcn_readfirstlane((int)weight((unsigned)out.tiles));
    out.pair = __builtin_amdgcn_readfirstlane((int)(left / each));
    out.tile = (int)(left - out.pair * each);
    out.run = out.whole = (int)run;
    if (apart) {
        out.whole = __builtin_amdgcn_readfirstlane((int)((out.tiles + each - 1) / each));      // even parts
        out.tile *= out.whole;
        out.run = out.whole < out.tiles - out.tile ? out.whole : out.tiles - out.tile;
    }
    return true;
}

// A stretch of memory: what lies beyond its end reads as 0 and is not fetched.
typedef __amdgpu_buffer_rsrc_t Stretch;
__device__ __forceinline__ Stretch stretch(const uint8_t *p, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p), 0, bytes, 0x00027000);
}

typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v3u __attribute__((ext_vector_type(3)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// Feature number f (0 .. dpad / 16 - 1) of a lane's share of a value row: neighbours, or, where that would be 6 bytes, 8 (4 bytes)
// from the first 128 features and 4 (2 bytes) from the others.
template <int DP, bool PACKED>
__device__ __forceinline__ constexpr int feature_of(int lane16, int f)
{
    constexpr int NT = DP / 16;
    if (PACKED && NT == 12) return f < 8 ? lane16 * 8 + f : 128 + lane16 * 4 + f - 8;
    return lane16 * NT + f;
}
// Bytes of that share, of the row that begins at `at` of the stretch.
template <int DP, bool PACKED>
__device__ __forceinline__ void load_share(Stretch s, unsigned at, int lane16, uint32_t *w)
{
    constexpr int BYTES = PACKED ? DP / 32 : DP / 16;
    if constexpr (BYTES == 16) {
        const v4u t = __builtin_amdgcn_raw_buffer_load_b128(s, at + lane16 * 16, 0, 0);
        w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w;
    } else if constexpr (BYTES == 12) {
        const v3u t = __builtin_amdgcn_raw_buffer_load_b96(s, at + lane16 * 12, 0, 0);
        w[0] = t.x; w[1] = t.y; w[2] = t.z;
    } else if constexpr (BYTES == 8) {
        const v2u t = __builtin_amdgcn_raw_buffer_load_b64(s, at + lane16 * 8, 0, 0);
        w[0] = t.x; w[1] = t.y;
    } else if constexpr (BYTES == 6) {
        w[0] = __builtin_amdgcn_raw_buffer_load_b32(s, at + lane16 * 4, 0, 0);
        w[1] = __builtin_amdgcn_raw_buffer_load_b16(s, at + 64 + lane16 * 2, 0, 0);
    } else if constexpr (BYTES == 4) {
        w[0] = __builtin_amdgcn_raw_buffer_load_b32(s, at + lane16 * 4, 0, 0);
    } else {
        w[0] = __builtin_amdgcn_raw_buffer_load_b16(s, at + lane16 * 2, 0, 0);
    }
}

// One tile of tokens in registers: the keys, and the values of a lane's features.
template <int DP, bool PACKED>
struct Tile {
    static constexpr int TG = tile_tokens(DP, PACKED) / 16, NS = DP / 64, NT = DP / 16;
    static constexpr int VW = ((PACKED ? NT / 2 : NT) + 3) / 4;
    uint32_t k[TG][NS][PACKED ? 2 : 4];
    uint32_t v[TG / 2][8][VW];
};

// Halves [features t of token e | of token e + 1] as fp16 c 2^-9, exactly, from the two tokens' shares of a row.  A byte alone in a half
// is the fp16 number u 2^-24 (c + 128, packed: c + 8 or 16 c + 128, below 2^10): one multiplication by 2^15 or 2^11 and an addition.
constexpr float VALUE_SCALE = 512.0f;
template <bool PACKED>
__device__ __forceinline__ uint32_t value_pair(uint32_t w0, uint32_t w1, int t, v2h off)
{
    const int byte = PACKED ? (t >> 1) & 3 : t & 3;
    uint32_t x = __builtin_amdgcn_perm(w1, w0, 0x0c000c00u | (uint32_t)byte | (uint32_t)(4 + byte) << 16);
    const _Float16 up = (_Float16)(PACKED && (t & 1) ? 2048.0f : 32768.0f);
    if (PACKED) x &= t & 1 ? 0x00f000f0u : 0x000f000fu;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(v2h, x), v2h{up, up}, off));
}
__device__ __forceinline__ uint32_t value_word(bool packed, uint32_t w) { return packed ? w : w ^ 0x80808080u; }

// Workspace: sums [2 grid][rows of a tile][DP], then maximum and sum of weights [2 grid][rows of a tile][2], then Parts per pair.
struct Workspace {
    float *sums, *ml;
    Parts *parts;
};
__host__ __device__ __forceinline__ Workspace workspace(float *p, int64_t slots, int tile_rows, int dpad)
{
    Workspace w;
    w.sums = p;
    w.ml = p + slots * tile_rows * dpad;
    w.parts = reinterpret_cast<Parts *>(w.ml + slots * tile_rows * 2);
    return w;
}

// Over the 8, 16 or 32 neighbouring lanes of a row, in all of them.
template <int LR>
__device__ __forceinline__ float row_max(float v)
{
    auto with = [&](int t) { v = fmaxf(v, __builtin_bit_cast(float, t)); };
    with(dpp_move<DPP_XOR1>(__builtin_bit_cast(int, v)));
    with(dpp_move<DPP_XOR2>(__builtin_bit_cast(int, v)));
    with(dpp_move<DPP_HALF_MIRROR>(__builtin_bit_cast(int, v)));
    if (LR >= 16) with(dpp_move<DPP_ROW_MIRROR>(__builtin_bit_cast(int, v)));
    if (LR >= 32) v = fmaxf(v, __shfl_xor(v, 16, 64));
    return v;
}
template <int LR>
__device__ __forceinline__ int row_sum_of(int v)
{
    v += dpp_move<DPP_XOR1>(v);
    v += dpp_move<DPP_XOR2>(v);
    v += dpp_move<DPP_HALF_MIRROR>(v);
    if (LR >= 16) v += dpp_move<DPP_ROW_MIRROR>(v);
    if (LR >= 32) v += __shfl_xor(v, 16, 64);
    return v;
}

// A row of queries, 8 features a lane, LR lanes.
//   What every token's score has: sum q (k + s / 2) scale.
template <int LR>
__device__ __forceinline__ float query_offset(const float *v, const float *step, const float *k, float scale)
{
    float offset = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) offset += v[e] * scale * (k[e] + 0.5f * step[e]);
#pragma unroll
    for (int o = 1; o < LR; o <<= 1) offset += __shfl_xor(offset, o, 64);
    return offset;
}
//   x = q s in place, times 1 / back^2 where that leaves binary32's middle range (rare); returns its largest magnitude, infinite if one is not finite.
template <int LR>
__device__ __forceinline__ float query_steps(float *x, const float *step, float *back)
{
    float v[8], most;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[e];
    auto with_steps = [&](float by) {
        most = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = v[e] * by * by * step[e];
            const float size = fabsf(x[e]);
            most = fmaxf(most, size <= 3.402823466e38f ? size : INFINITY);     // a NaN counts as infinite
        }
        most = row_max<LR>(most);
    };
    with_steps(1.0f);
    *back = 1.0f;
    if (__any(most == INFINITY || (most > 0.0f && most <= 1e-30f))) {
        *back = most == INFINITY ? 0x1p64f : most > 0.0f && most <= 1e-30f ? 0x1p-64f : 1.0f;
        with_steps(1.0f / *back);
    }
    return most;
}
//   Rounded to most / QMAX, of the sign of the scores' scale, in ND signed digits, `apart` bytes from one to the next.
template <int ND, bool PACKED>
__device__ __forceinline__ void query_digits8(const float *x, float most, float scale, float qmax, int8_t *row, int apart, int qc)
{
    const bool use = most != INFINITY && most > 1e-30f;          // below 1e-30 now: scores are 0 at any scale
    const float f = use ? __uint_as_float(__float_as_uint(qmax / most) | (__float_as_uint(scale) & 0x80000000u)) : 0.0f;
    int8_t d[ND][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        // packed rows have the even features of 16 first (low nibbles of 8 bytes), then the odd ones
        const int to = PACKED ? (e >> 1) + 4 * (e & 1) : e;
        int z = use ? (int)rintf(x[e] * f) : 0;
#pragma unroll
        for (int dd = ND - 1; dd > 0; --dd) {
            const int up = (z + 128) >> 8;
            d[dd][to] = (int8_t)(z - (up << 8));                 // -128 .. 127
            z = up;
        }
        d[0][to] = (int8_t)z;
    }
#pragma unroll
    for (int dd = 0; dd < ND; ++dd) {
        uint32_t w[2];
        __builtin_memcpy(w, d[dd], 8);
        int8_t *const to = row + dd * apart;
        if (PACKED) {
            *reinterpret_cast<uint32_t *>(to + 16 * (qc >> 1) + 4 * (qc & 1)) = w[0];
            *reinterpret_cast<uint32_t *>(to + 16 * (qc >> 1) + 8 + 4 * (qc & 1)) = w[1];
        } else {
            *reinterpret_cast<uint2 *>(to + 8 * qc) = make_uint2(w[0], w[1]);
        }
    }
}
//   What the integer scores are multiplied by, above 0 and finite.
template <bool PACKED>
__device__ __forceinline__ float score_scale(float most, float qmax, float back, float scale)
{
    const float by = most / qmax * (PACKED ? 1.44269504088896f / 16.0f : 1.44269504088896f) * back * fabsf(scale) * back;
    return fminf(fmaxf(by, 1e-30f), 3.402823466e38f);
}
// The digits' products put together.
template <int ND>
__device__ __forceinline__ float score_of(const v4i *sum, int j)
{
    const float low = (float)(sum[ND - 2][j] * 256 + sum[ND - 1][j]);
    if constexpr (ND == 4) return __builtin_fmaf((float)(sum[0][j] * 256 + sum[1][j]), 65536.0f, low);
    else if constexpr (ND == 3) return __builtin_fmaf((float)sum[0][j], 65536.0f, low);
    else return low;
}
// The same without conversions, which take four times an addition's time: a sum that begins at the bits of 1.5 x 2^23 has, read as binary32, that much more
// than its value (sums of a digit's products stay within 2^22).  The score comes out SCORE_SHIFT too large, which drops out of the softmax.
constexpr float SCORE_SHIFT = 12582912.0f;
constexpr int INT_AS_FLOAT = 0x4b400000;
template <int ND>
__device__ __forceinline__ float shifted_score(const v4i *sum, int j)
{
    auto of = [&](int dd) { const int bits = sum[dd][j]; return __builtin_bit_cast(float, bits); };
    const float low = __builtin_fmaf(of(ND - 2) - SCORE_SHIFT, 256.0f, of(ND - 1));
    if constexpr (ND == 4) return __builtin_fmaf(__builtin_fmaf(of(0) - SCORE_SHIFT, 256.0f, of(1) - SCORE_SHIFT), 65536.0f, low);
    else if constexpr (ND == 3) return __builtin_fmaf(of(0) - SCORE_SHIFT, 65536.0f, low);
    else return low;
}
// Orders what the lanes of one wave write to and read from LDS.
__device__ __forceinline__ void wave_order()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);        // lgkmcnt(0)
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}

template <int DP, bool PACKED, int RT, int TYPE, typename CALL>
__global__ __launch_bounds__(THREADS, blocks_per_cu(DP, PACKED, RT, TYPE, std::is_same<CALL, KvWindow>::value)) void kv_attend_kernel(KvView kv, KvQueries q, CALL a, int row_tiles,
                                                                                       int least)
{
    typedef Tile<DP, PACKED> T;
    constexpr bool WINDOW = std::is_same<CALL, KvWindow>::value, TREE = std::is_same<CALL, KvTree>::value, MASKED = WINDOW || TREE;
    constexpr int TG = T::TG, NS = T::NS, NT = T::NT, TOK = 16 * TG;
    constexpr int ND = query_digits(TYPE), NP = TYPE == LPQ_TYPE_F32 ? 2 : 1, RB = PACKED ? DP / 2 : DP;
    // what ND digits hold, less a rounding
    constexpr float QMAX = ND == 4 ? 2139061888.0f : ND == 3 ? 8355600.0f : 32639.0f;
    __shared__ float red_m[WAVES][16 * RT], red_l[WAVES][16 * RT];
    __shared__ __align__(16) float sums[WAVES][16][DP + 4];
    __shared__ __align__(16) int8_t digits[ND][16 * RT][DP + 16];
    __shared__ float row_scale[16 * RT], row_shift[16 * RT];
    __shared__ int4 row_sees[MASKED ? 16 * RT : 1];

    const int lane0 = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = q.new_tokens * q.group;
    const int64_t head_bytes = (int64_t)kv.page * RB;
    const Workspace ws = workspace(a.part, 2 * (int64_t)gridDim.x, 16 * RT, DP);
    Place at;
    int row_tile;
    unsigned share;                // of the tiles
    if (least == 0) {              // a workgroup per pair and row tile
        const int pair = __builtin_amdgcn_readfirstlane(blockIdx.x / row_tiles);
        row_tile = blockIdx.x - pair * row_tiles;
        share = pair;
        at.b = __builtin_amdgcn_readfirstlane(pair / kv.heads);
        at.pair = pair - at.b * kv.heads;
        at.tile = 0;
        at.tiles = tiles_seen(kv, q, a, row_tokens(q, row_tile * 16 * RT, 16 * RT), kv_uniform(a.lengths)[at.b], TOK);
        at.run = at.whole = at.tiles;
    } else {
        const unsigned eights = __builtin_amdgcn_readfirstlane(blockIdx.x / (8 * row_tiles)), in = blockIdx.x - eights * 8 * row_tiles;
        row_tile = in >> 3;
        share = eights * 8 + (in & 7);
        if (!first_place(kv, q, a, row_tokens(q, row_tile * 16 * RT, 16 * RT), share, gridDim.x / row_tiles, TOK, least, CROSSING, at)) return;
    }
    const int row0 = row_tile * 16 * RT;
    int left = at.run, b = at.b, pair = at.pair, start = at.tile, tiles = at.tiles;

    for (;;) {
        // ---- tiles [start, end) of a pair; all lanes have the same, and scalar registers hold it
        b = __builtin_amdgcn_readfirstlane(b);
        pair = __builtin_amdgcn_readfirstlane(pair);
        start = __builtin_amdgcn_readfirstlane(start);
        tiles = __builtin_amdgcn_readfirstlane(tiles);
        left = __builtin_amdgcn_readfirstlane(left);
        const int h = pair;
        const int end = left < tiles - start ? start + left : tiles;
        const int len = length_of(kv, a, kv_uniform(a.lengths)[b]);
        const int32_t *table = a.table + (int64_t)b * a.ld_table, *chosen = a.chosen + ((int64_t)b * kv.heads + h) * a.n_select;
        int lane = lane0, tid = threadIdx.x;
        asm volatile("" : "+v"(lane), "+v"(tid));      // nothing that depends on it is worth registers over all of a run
        const int n = lane & 15, g = lane >> 4;

        // Pages.  A lane looks up the page of the pool and the position of one group of 16 tokens, those of the wave's next
        // PER tiles at once, and again while these are gone through; a tile's come out by lane number.  Position INT32_MAX:
        // there is none.
        constexpr int PER = 64 / TG;
        // Positions between the sinks' groups and the windows' are left out.  (The loop over tiles has the two numbers from LDS: registers.)
        struct Gap {
            int from, width;
        };
        Gap gap = {0, 0};
        if constexpr (WINDOW) {
            if (!a.chosen) {
                const Span span = span_of(a, q, row_tokens(q, row0, 16 * RT), len);
                gap = {16 * span.sink, 16 * (span.low - span.sink)};
            }
        }
        const int columns = a.chosen ? a.n_select : a.table_pages, pool_pages = (int)kv.pages;      // below 2^31
        const int first_tile = start + wave;
        auto look_up = [&](int turn, int &page, int &pos, Gap gap) {
            unsigned token = 16u * ((first_tile + (turn + lane / TG) * WAVES) * TG + lane % TG);
            if constexpr (WINDOW) {
                if (token >= (unsigned)gap.from) token += gap.width;      // (the last tile may reach beyond what the rows see)
            }
            const int want = (int)(token >> kv.page_shift), inside = (int)token & (kv.page - 1);
            bool there = want < columns;
            int column = there ? want : columns - 1;
            if (a.chosen) {
                column = chosen[column];
                there = there && (unsigned)column < (unsigned)a.table_pages;
                column = there ? column : 0;
            }
            const int p = (column << kv.page_shift) + inside, id = table[column];
            there = there && p < len && (unsigned)id < (unsigned)pool_pages;
            page = there ? id : 0;
            pos = there ? p : INT32_MAX;
        };
        const int turns = first_tile < end ? (end - first_tile + WAVES - 1) / WAVES : 0;
        int page_now, pos_now, page_then = 0, pos_then = INT32_MAX;
        struct Where { int64_t base[TG]; int pos[TG]; };
        auto find = [&](int turn, Where &w) {
#pragma unroll
            for (int tg = 0; tg < TG; ++tg) {
                const int from = (turn % PER) * TG + tg, page = __builtin_amdgcn_readlane(page_now, from), pos = __builtin_amdgcn_readlane(pos_now, from);
                w.pos[tg] = turn < turns ? pos : INT32_MAX;
                w.base[tg] = ((int64_t)page * kv.heads + h) * head_bytes + (int64_t)((pos & (kv.page - 1) & ~15) * RB);
            }
        };
        T t;
        auto load_keys = [&](const Where &w) {
#pragma unroll
            for (int tg = 0; tg < TG; ++tg) {
                const Stretch rows16 = stretch(kv.k + w.base[tg], w.pos[tg] == INT32_MAX ? 0 : 16 * RB);
#pragma unroll
                for (int st = 0; st < NS; ++st) {
                    if constexpr (PACKED) {
                        const v2u x = __builtin_amdgcn_raw_buffer_load_b64(rows16, n * RB + g * 8 + 32 * st, 0, 0);
                        t.k[tg][st][0] = x.x; t.k[tg][st][1] = x.y;
                    } else {
                        const v4u x = __builtin_amdgcn_raw_buffer_load_b128(rows16, n * RB + g * 16 + 64 * st, 0, 0);
                        t.k[tg][st][0] = x.x; t.k[tg][st][1] = x.y; t.k[tg][st][2] = x.z; t.k[tg][st][3] = x.w;
                    }
                }
            }
        };
        auto load_values = [&](const Where &w) {
#pragma unroll
            for (int tg = 0; tg < TG; ++tg) {
                const Stretch rows16 = stretch(kv.v + w.base[tg], w.pos[tg] == INT32_MAX ? 0 : 16 * RB);
#pragma unroll
                for (int j = 0; j < 4; ++j) load_share<DP, PACKED>(rows16, (4 * g + j) * RB, n, t.v[tg >> 1][(tg & 1) * 4 + j]);
            }
        };

        // ---- what memory has to bring, asked for before any of it is used: queries (LR lanes per row, 8 features each), the wave's
        // first tile
        constexpr int LR = DP <= 64 ? 8 : DP <= 128 ? 16 : 32, PASS = THREADS / LR, PASSES = (16 * RT + PASS - 1) / PASS;
        const int qc = tid % LR, qc0 = 8 * qc < DP ? 8 * qc : 0;
        auto load_queries = [&](int i) {
            const int r16 = i * PASS + tid / LR, r = row0 + r16;
            const bool on = r16 < 16 * RT && r < rows && 8 * qc < DP;
            const int64_t qat = (int64_t)b * q.ld_seq + (int64_t)(r / q.group) * q.ld_token + (int64_t)(h * q.group + r % q.group) * q.ld_head;
            return kv_load8(q.p, TYPE, qat + qc0, on ? kv.dim - qc0 : 0);
        };
        Raw8 raw = load_queries(0);
        float step[8];
        kv_load_floats8(kv.key.s + h * DP + qc0, step);
        Where now, next;
        look_up(0, page_now, pos_now, gap);
        find(0, now);
        load_keys(now);
        load_values(now);

        // ---- queries: steps folded in, digits (a loop: what runs once per call costs its fetch from memory, not its instructions)
#pragma unroll 1
        for (int i = 0; i < PASSES; ++i) {
            const int r16 = i * PASS + tid / LR;
            float x[8], back;
            kv_floats8(raw, TYPE, kv.dim - qc0, x);
            if (i + 1 < PASSES) raw = load_queries(i + 1);
            if (a.lse) {
                const float offset = query_offset<LR>(x, step, kv.key.k + h * DP + qc0, a.scale);
                if (qc == 0 && r16 < 16 * RT) row_shift[r16] = offset;
            }
            const float most = query_steps<LR>(x, step, &back);
            if (r16 >= 16 * RT) continue;
            if (8 * qc < DP) query_digits8<ND, PACKED>(x, most, a.scale, QMAX, digits[0][r16], 16 * RT * (DP + 16), qc);
            // equal scores stay equal, and -inf in the place of a masked one stays that (below 1e-30 scores are 0 in any case, at the other end the
            // largest take all); negative: the row is not finite
            if (qc == 0) row_scale[r16] = most == INFINITY ? -1.0f : score_scale<PACKED>(most, QMAX, back, a.scale);
        }
        // Of a window: a row sees .x positions from .y on, and those below .z.  Of a tree: positions up to .x (-1: none) that are below .y, or
        // whose bits are set in its token's words, bit p & 31 of word .z + (p >> 5); .y is a multiple of 32 at or ahead of the first new token, so
        // that four neighbours are in one word.  The bits are in the memory that joins the waves at the end.
        uint32_t *tree_bits = reinterpret_cast<uint32_t *>(&sums[0][0][0]);
        if constexpr (WINDOW) {
            if (tid < 16 * RT) {
                const int r = row0 + tid, me = r < rows ? len - q.new_tokens + r / q.group : -1;
                const int first = window_from(a, me), sinks = me < a.sinks ? me + 1 : a.sinks;
                const int kept = tid == 0 ? gap.from : gap.width;
                row_sees[tid] = me < 0 ? make_int4(0, 0, 0, kept) : make_int4(me + 1 - first, first, sinks, kept);
            }
        }
        if constexpr (TREE) {
            static_assert(sizeof(sums) >= 16 * RT * ((KV_MAX_TREE + 31 + 63) / 64) * 8, "a row tile's bits");
            const RowTokens mine = row_tokens(q, row0, 16 * RT);
            const int words = (q.new_tokens + 31 + 63) >> 6, drafts = len - q.new_tokens, begin = drafts & ~31;      // words of 64 positions
            if (tid < 16 * RT) {
                const int r = row0 + tid, token = r / q.group;
                row_sees[tid] = make_int4(r < rows && drafts + token >= 0 ? len - 1 : -1, begin, (token - mine.from) * 2 * words - (begin >> 5), 0);
            }
            const int count = (mine.to - mine.from + 1) * words;
            const uint8_t *mask = a.tree + (int64_t)b * a.ldt_seq;
            for (int i = wave; i < count; i += WAVES) {
                const int token = i / words, to = (i - token * words) * 64 + lane - (drafts - begin);
                bool sees = to < 0;
                if (to >= 0 && to < q.new_tokens) sees = mask[(int64_t)(mine.from + token) * a.ldt_token + to] != 0;
                const uint64_t all = __ballot(sees);
                if (lane == 0) reinterpret_cast<uint64_t *>(tree_bits)[i] = all;
            }
        }
        __syncthreads();
        v4i qd[RT][ND][NS];      // lane (n, g): features 64 st + 16 g .. + 15 of row n
        float rs[RT], m[RT];     // scale of the scores (integers so far) and their maximum, as an integer
        v4f l[RT];               // sums of the weights, four times the same
        v8h ones;
#pragma unroll
        for (int e = 0; e < 8; ++e) ones[e] = (_Float16)1.0f;
        int last[RT];            // last position a row sees
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
            for (int dd = 0; dd < ND; ++dd) {
#pragma unroll
                for (int st = 0; st < NS; ++st) qd[rt][dd][st] = *reinterpret_cast<const v4i *>(&digits[dd][rt * 16 + n][64 * st + 16 * g]);
            }
            rs[rt] = fabsf(row_scale[rt * 16 + n]);
            m[rt] = NEG;
            l[rt] = v4f{0.f, 0.f, 0.f, 0.f};
            if constexpr (!MASKED) {
                const int r = row0 + rt * 16 + n;
                const int see = len - q.new_tokens + r / q.group;
                last[rt] = r < rows ? (see < -1 ? -1 : see) : -1;
            }
        }
        int seen = len - q.new_tokens;       // a tile that ends at or before this position is seen by every row (with a window: where it begins
        int windows = 0;                     // at or behind `windows`; the sinks are few)
        if constexpr (WINDOW) {
            const RowTokens mine = row_tokens(q, row0, 16 * RT);
            windows = window_from(a, seen + mine.to);
            seen += mine.from;
        }
        if constexpr (TREE) --seen;

        v4f acc[RT][NT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[rt][t] = v4f{0.f, 0.f, 0.f, 0.f};

        auto gap_kept = [&]() {
            if constexpr (WINDOW) return Gap{__builtin_amdgcn_readfirstlane(row_sees[0].w), __builtin_amdgcn_readfirstlane(row_sees[1].w)};
            else return Gap{0, 0};
        };
        if (turns > PER) look_up(PER, page_then, pos_then, gap_kept());

        // ---- the wave's tiles: the next tile's keys are asked for as soon as this one's are used up, its values likewise
        // (behind the last tile as well, with nothing to fetch: loads that every turn makes are waited for one kind at a time)
        for (int turn = 0; turn < turns; ++turn) {
            if ((turn + 1) % PER == 0) {
                page_now = page_then;
                pos_now = pos_then;
                if (turns > turn + 1 + PER) look_up(turn + 1 + PER, page_then, pos_then, gap_kept());
            }
            find(turn + 1, next);
            bool part = false;
#pragma unroll
            for (int tg = 0; tg < TG; ++tg) {
                part |= now.pos[tg] > seen - 15;     // also where a group does not count
                if constexpr (WINDOW) part |= now.pos[tg] < windows;
            }
            float s[RT][TG][4];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int tg = 0; tg < TG; ++tg) {
                    v4i sum[ND];
#pragma unroll
                    for (int dd = 0; dd < ND; ++dd) sum[dd] = v4i{0, 0, 0, 0};
#pragma unroll
                    for (int st = 0; st < NS; ++st) {
                        v4i kf;
                        if constexpr (PACKED) {
                            // nibbles c + 8 -> bytes 16 c
                            const uint32_t x = t.k[tg][st][0] ^ 0x88888888u, y = t.k[tg][st][1] ^ 0x88888888u;
                            kf = v4i{(int)((x << 4) & 0xf0f0f0f0u), (int)((y << 4) & 0xf0f0f0f0u), (int)(x & 0xf0f0f0f0u), (int)(y & 0xf0f0f0f0u)};
                        } else {
                            kf = v4i{(int)t.k[tg][st][0], (int)t.k[tg][st][1], (int)t.k[tg][st][2], (int)t.k[tg][st][3]};
                        }
#pragma unroll
                        for (int dd = 0; dd < ND; ++dd) sum[dd] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf, qd[rt][dd][st], sum[dd], 0, 0, 0);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[rt][tg][j] = score_of<ND>(sum, j);
                }
            load_keys(next);
            v2h off = {(_Float16)(PACKED ? -8.0f / VALUE_SCALE : -128.0f / VALUE_SCALE), (_Float16)(PACKED ? -8.0f / VALUE_SCALE : -128.0f / VALUE_SCALE)};
            asm("" : "+v"(off));           // in a vector register: an instruction takes one scalar constant, and that is the other factor
            v8h w[RT][NP][TG / 2];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if (part) {
                    asm volatile("");      // a branch: few tiles need it
                    if constexpr (MASKED) {
                        const int4 row = row_sees[rt * 16 + n];
#pragma unroll
                        for (int tg = 0; tg < TG; ++tg) {
                            uint32_t named = ~0u;
                            if constexpr (TREE) {
                                const int at = now.pos[tg] + 4 * g;
                                if (now.pos[tg] <= row.x && at >= row.y) named = tree_bits[row.z + (at >> 5)] >> (at & 31);
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int e = 4 * g + j;
                                bool sees;
                                if (WINDOW) sees = (unsigned)(now.pos[tg] - row.y) + e < (unsigned)row.x || now.pos[tg] < row.z - e;
                                else sees = now.pos[tg] <= row.x - e && ((named >> j) & 1);
                                if (!sees) s[rt][tg][j] = NEG;
                            }
                        }
                    } else {
#pragma unroll
                        for (int tg = 0; tg < TG; ++tg)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (now.pos[tg] > last[rt] - (4 * g + j)) s[rt][tg][j] = NEG;
                    }
                }
                float top = s[rt][0][0];
#pragma unroll
                for (int tg = 0; tg < TG; ++tg)
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = fmaxf(top, s[rt][tg][j]);
                if (__any((top - m[rt]) * rs[rt] > HEADROOM)) {
                    top = fmaxf(top, __shfl_xor(top, 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    const float next = fmaxf(m[rt], top);
                    const float f = next == NEG ? 1.0f : __builtin_amdgcn_exp2f((m[rt] - next) * rs[rt]);
                    m[rt] = next;
                    l[rt] *= f;
#pragma unroll
                    for (int t_ = 0; t_ < NT; ++t_)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[rt][t_][j] *= f;
                }
                const float most = m[rt] == NEG ? 0.0f : m[rt];
                float up = LIFT - most * rs[rt];
                // A difference of numbers this large keeps too little of it: by 2^27 weights were beyond fp16.  In float32 calls none is taken, so that the
                // largest score's weight is 2^13 to the last bit, and a token that has all the weight comes out as it reads back.
                if (NP == 2 || __any(fabsf(up) > FAR)) {
                    asm volatile("");
#pragma unroll
                    for (int tg = 0; tg < TG; ++tg)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[rt][tg][j] -= most;
                    up = LIFT;
                }
#pragma unroll
                for (int tg = 0; tg < TG; ++tg)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][tg][j], rs[rt], up));
                        const _Float16 p0 = (_Float16)p;
                        w[rt][0][tg >> 1][(tg & 1) * 4 + j] = p0;
                        if constexpr (NP == 2) w[rt][1][tg >> 1][(tg & 1) * 4 + j] = (_Float16)(p - (float)p0);
                    }
#pragma unroll
                for (int half = 0; half < TG / 2; ++half)
#pragma unroll
                    for (int p = 0; p < NP; ++p) l[rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, w[rt][p][half], l[rt], 0, 0, 0);
            }
#pragma unroll
            for (int half = 0; half < TG / 2; ++half) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int i = 0; i < T::VW; ++i) t.v[half][e][i] = value_word(PACKED, t.v[half][e][i]);
#pragma unroll
                for (int f = 0; f < NT; ++f) {
                    const int word = PACKED ? f >> 3 : f >> 2;
                    uint32_t two[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) two[e] = value_pair<PACKED>(t.v[half][2 * e][word], t.v[half][2 * e + 1][word], f, off);
                    v8h vf;
                    __builtin_memcpy(&vf, two, 16);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            acc[rt][f] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, w[rt][p][half], acc[rt][f], 0, 0, 0);
                }
            }
            load_values(next);
            now = next;
        }
        asm volatile("s_nop 15");      // the last matrix results are read in other blocks of code

        // ---- the waves' parts joined
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (g == 0) {
                red_m[wave][rt * 16 + n] = m[rt] * MAXIMUM * rs[rt];
                // a row that is not finite is not a number from the first token on that it sees
                red_l[wave][rt * 16 + n] = row_scale[rt * 16 + n] < 0.0f && l[rt][0] > 0.0f ? NAN : l[rt][0];
            }
        }
        __syncthreads();
        const bool whole = start == 0 && end == tiles;
        const int64_t slot = 2 * ((int64_t)share * row_tiles + row_tile) + (start == 0 ? 1 : 0);
        if (least != 0 && start == 0 && threadIdx.x == 0 && (MASKED || row_tile == 0))
            ws.parts[MASKED ? ((int64_t)b * kv.heads + pair) * row_tiles + row_tile : (int64_t)b * kv.heads + pair] = {(int)share, 1 + (int)(((unsigned)(tiles - end) + at.whole - 1) / at.whole)};
#pragma unroll 1
        for (int rt = 0; rt < RT; ++rt) {
            float top = NEG;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) top = fmaxf(top, red_m[w][rt * 16 + n]);
            const float f = lag(red_m[wave][rt * 16 + n], top);
            if (rt) __syncthreads();
            auto put = [&](const v4f *x) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int t_ = 0; t_ < NT; ++t_) sums[wave][n][feature_of<DP, PACKED>(4 * g + j, t_)] = x[t_][j] * (f * VALUE_SCALE);
            };
            if (RT == 1 || rt == 0) put(acc[0]);
            else put(acc[RT - 1]);
            if (a.lse && start == 0 && wave == 0 && g == 0) {      // of several parts: what every token has, the rest is added when they are joined
                const int r = row0 + rt * 16 + n;
                if (r < rows) {
                    float sum = 0.0f;
#pragma unroll
                    for (int w = 0; w < WAVES; ++w)
                        sum += red_l[w][rt * 16 + n] * lag(red_m[w][rt * 16 + n], top);
                    const int64_t lat = ((int64_t)b * q.new_tokens + r / q.group) * ((int64_t)kv.heads * q.group) + h * q.group + r % q.group;
                    a.lse[lat] = !whole ? row_shift[rt * 16 + n] : sum == 0.0f ? NEG : (top * (1.0f / MAXIMUM) - LIFT + __log2f(sum)) * 0.69314718055994531f + row_shift[rt * 16 + n];
                }
            }
            __syncthreads();
            const int r16 = tid >> 4, r = row0 + rt * 16 + r16;
            if (r < rows) {
                float mm = NEG, ll = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) mm = fmaxf(mm, red_m[w][rt * 16 + r16]);
#pragma unroll
                for (int w = 0; w < WAVES; ++w)
                    ll += red_l[w][rt * 16 + r16] * lag(red_m[w][rt * 16 + r16], mm);
                const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
                const int64_t row = slot * (16 * RT) + rt * 16 + r16;
                const int64_t out_row = (int64_t)b * a.ldo_seq + (int64_t)(r / q.group) * a.ldo_token + (int64_t)(h * q.group + r % q.group) * a.ldo_head;
#pragma unroll 1
                for (int i = 0; i < NS; ++i) {
                    const int c0 = 4 * ((tid & 15) + 16 * i);
                    float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) {
                        const float4 y = *reinterpret_cast<const float4 *>(&sums[w][r16][c0]);
                        x[0] += y.x; x[1] += y.y; x[2] += y.z; x[3] += y.w;
                    }
                    if (whole) {
                        const float *vs = kv.value.s + h * DP + c0, *vk = kv.value.k + h * DP + c0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = ll == 0.0f ? 0.0f : (x[e] * inv + 0.5f) * vs[e] + vk[e];
                        kv_store<4>(a.out, TYPE, out_row + c0, kv.dim - c0, x);
                    } else {
                        *reinterpret_cast<float4 *>(ws.sums + row * DP + c0) = make_float4(x[0], x[1], x[2], x[3]);
                    }
                }
                if ((tid & 15) == 0 && !whole) {
                    ws.ml[row * 2] = mm;
                    ws.ml[row * 2 + 1] = ll;
                }
            }
        }

        // ---- on to what follows in the workgroup's run
        left -= end - start;
        if (left <= 0) return;
        if (end == tiles && ++pair == kv.heads) {
            pair = 0;
            if (++b >= a.nseq) return;
            tiles = tiles_seen(kv, q, a, row_tokens(q, row0, 16 * RT), kv_uniform(a.lengths)[b], TOK);
        }
        start = 0;
        __syncthreads();               // LDS is used again
    }
}

// Calls with a window and query rows enough to fill the chip, as the parts of prompts have.  The same mathematics, digits, weights and masks as
// kv_attend_kernel, shared out the other way: a wave has 16 rows of its own, and all eight go through the same tokens, 64 at a time.  Waves 0
// to 3 bring the keys of a group of 16 each into LDS, as the first product's operands, waves 4 to 7 the values, as fp16 in the second's, so that
// codes are fetched, unpacked and made fp16 once for 128 rows; two buffers take turns, with one barrier to a tile, and the next tile's codes are under
// way in registers meanwhile.  No row is another wave's concern: nothing is joined, and what a workgroup costs before its first tile and
// behind its last, 9 us there, is shared by eight times the rows.
// us, kv_attend_kernel and this one: 4 sequences of up to 9000 tokens, windows of 600 for 6000 rows a head, 4 heads of 96 on 4-bit codes, float16 113, 70; 8 of
// 128 on 8-bit codes, bfloat16 265, 144, windows of 4000 1114, 515; 2800 float32 rows, windows of 1000, heads of 128 224, 150, of 256 575, 271; 128
// sequences, 48 rows, windows of 1000 141, 103.  Where its workgroups do not fill the chip it loses: 32 sequences of 96 rows, windows of 2000, 87, 89,
// 720 float32 rows on one head of 192 25, 41.  Bound by the chain of a wave, which goes from scores over maximum, exponentials and roundings to sums with
// nothing of the next tokens beside it, and by how the last workgroups fill the chip: the first call's 752 stand on 512 places, so that 2.8 of 4 waves
// are on a SIMD on average, the vector pipe is busy 61 % of the time (16 scores a lane of 64 tokens, each joined from its digits, compared, scaled,
// raised and rounded) and the matrix pipe 23 %.
constexpr int ROWS_TOKENS = 64, ROWS_WAVES = 8, ROWS_THREADS = 64 * ROWS_WAVES, ROWS_TILE = 16 * ROWS_WAVES;
__host__ __device__ constexpr int rows_digits(int type, int dpad) { return query_digits(type) * 8 * (dpad + 16); }      // bytes, of 8 rows
__host__ __device__ constexpr int rows_stage(int dpad) { return ROWS_TOKENS * dpad * 3; }
__host__ __device__ constexpr int rows_blocks_per_cu(int dpad) { return dpad <= 128 ? 2 : 1; }

template <int DP, bool PACKED, int TYPE>
__global__ __launch_bounds__(ROWS_THREADS, 2 * rows_blocks_per_cu(DP)) void kv_rows_kernel(KvView kv, KvQueries q, KvWindow a, int row_tiles)
{
    constexpr int NS = DP / 64, NT = DP / 16, RB = PACKED ? DP / 2 : DP, VW = ((PACKED ? NT / 2 : NT) + 3) / 4;
    constexpr int ND = query_digits(TYPE), NP = TYPE == LPQ_TYPE_F32 ? 2 : 1, TILE_ROWS = ROWS_TILE;
    constexpr float QMAX = ND == 4 ? 2139061888.0f : ND == 3 ? 8355600.0f : 32639.0f;
    constexpr int KEYS = ROWS_TOKENS * DP, STAGE = rows_stage(DP);      // bytes: keys, keys and values
    static_assert(ROWS_WAVES * rows_digits(TYPE, DP) <= 2 * STAGE, "the queries' digits go through the buffers' memory");
    __shared__ __align__(16) char stage[2 * STAGE];
    __shared__ int group_at[2][4];
    __shared__ int4 row_sees[TILE_ROWS];
    __shared__ float row_scale[TILE_ROWS], row_shift[TILE_ROWS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int rows = q.new_tokens * q.group;
    const int64_t head_bytes = (int64_t)kv.page * RB;
    // Neighbouring row tiles of a pair, which see nearly the same tokens, on one XCD.
    const int work = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);      // (the grid: a multiple of 8)
    if (work >= a.nseq * kv.heads * row_tiles) return;
    const int pair = __builtin_amdgcn_readfirstlane(work / row_tiles), row_tile = work - pair * row_tiles;
    const int b = __builtin_amdgcn_readfirstlane(pair / kv.heads), h = pair - b * kv.heads;
    const int group = wave & 3;
    const bool brings_keys = wave < 4;
    const int tile0 = row_tile * TILE_ROWS, row0 = tile0 + 16 * wave;
    const RowTokens tile_rows = row_tokens(q, tile0, TILE_ROWS);
    const bool working = row0 < rows;      // a wave behind the last row brings tokens in, and has none of its own to see
    const int len = length_of(kv, a, kv_uniform(a.lengths)[b]);
    const int32_t *table = a.table + (int64_t)b * a.ld_table, *chosen = a.chosen + ((int64_t)b * kv.heads + h) * a.n_select;

    // Pages, as in kv_attend_kernel: a lane looks up the wave's group of one of the next 64 tiles.
    int gap_from = 0, gap_width = 0;
    if (!a.chosen) {
        const Span span = span_of(a, q, tile_rows, len);
        gap_from = 16 * span.sink;
        gap_width = 16 * (span.low - span.sink);
    }
    const int columns = a.chosen ? a.n_select : a.table_pages, pool_pages = (int)kv.pages, turns = tiles_seen(kv, q, a, tile_rows, kv_uniform(a.lengths)[b], ROWS_TOKENS);
    int pages, positions;
    auto look_up = [&](int turn) {
        unsigned token = 64u * (unsigned)(turn + lane) + 16u * group;
        if (token >= (unsigned)gap_from) token += gap_width;      // (the last tile may reach beyond what the rows see)
        const int want = (int)(token >> kv.page_shift), inside = (int)token & (kv.page - 1);
        bool there = turn + lane < turns && want < columns;
        int column = there ? want : 0;
        if (a.chosen) {
            column = chosen[column];
            there = there && (unsigned)column < (unsigned)a.table_pages;
            column = there ? column : 0;
        }
        const int p = (column << kv.page_shift) + inside, id = table[column];
        there = there && p < len && (unsigned)id < (unsigned)pool_pages;
        pages = there ? id : 0;
        positions = there ? p : INT32_MAX;
    };
    constexpr int KW = NS * (PACKED ? 2 : 4);
    uint32_t raw_codes[KW > 4 * VW ? KW : 4 * VW];
    int position;
    auto load = [&](int turn) {
        const int page = __builtin_amdgcn_readlane(pages, turn & 63);
        position = __builtin_amdgcn_readlane(positions, turn & 63);
        const int64_t base = ((int64_t)page * kv.heads + h) * head_bytes + (int64_t)((position & (kv.page - 1) & ~15) * RB);
        const Stretch rows16 = stretch((brings_keys ? kv.k : kv.v) + base, position == INT32_MAX ? 0 : 16 * RB);
        if (brings_keys) {
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                if constexpr (PACKED) {
                    const v2u x = __builtin_amdgcn_raw_buffer_load_b64(rows16, n * RB + g * 8 + 32 * st, 0, 0);
                    raw_codes[2 * st] = x.x; raw_codes[2 * st + 1] = x.y;
                } else {
                    const v4u x = __builtin_amdgcn_raw_buffer_load_b128(rows16, n * RB + g * 16 + 64 * st, 0, 0);
                    raw_codes[4 * st] = x.x; raw_codes[4 * st + 1] = x.y; raw_codes[4 * st + 2] = x.z; raw_codes[4 * st + 3] = x.w;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t w[VW];
                load_share<DP, PACKED>(rows16, (4 * g + j) * RB, n, w);
                asm volatile("");          // (else the compiler makes one store of both branches' and keeps the array in memory)
#pragma unroll
                for (int i = 0; i < VW; ++i) raw_codes[j * VW + i] = w[i];
            }
        }
    };
    // Keys [group][64 features][lane] 16 bytes, values [two groups][feature of a lane's][lane] 8 tokens, of which this wave has 4.
    auto keep = [&](int buffer) {
        char *const to = stage + buffer * STAGE;
        if (brings_keys) {
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                uint4 x;
                if constexpr (PACKED) {       // nibbles c + 8 -> bytes 16 c
                    const uint32_t u = raw_codes[2 * st] ^ 0x88888888u, w = raw_codes[2 * st + 1] ^ 0x88888888u;
                    x = make_uint4(u << 4 & 0xf0f0f0f0u, w << 4 & 0xf0f0f0f0u, u & 0xf0f0f0f0u, w & 0xf0f0f0f0u);
                } else {
                    x = make_uint4(raw_codes[4 * st], raw_codes[4 * st + 1], raw_codes[4 * st + 2], raw_codes[4 * st + 3]);
                }
                *reinterpret_cast<uint4 *>(to + ((group * NS + st) * 64 + lane) * 16) = x;
            }
            if (lane == 0) group_at[buffer][group] = position;
            return;
        }
        v2h off = {(_Float16)(PACKED ? -8.0f / VALUE_SCALE : -128.0f / VALUE_SCALE), (_Float16)(PACKED ? -8.0f / VALUE_SCALE : -128.0f / VALUE_SCALE)};
        asm("" : "+v"(off));
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < VW; ++i) raw_codes[j * VW + i] = value_word(PACKED, raw_codes[j * VW + i]);
#pragma unroll
        for (int f = 0; f < NT; ++f) {
            const int word = PACKED ? f >> 3 : f >> 2;
            *reinterpret_cast<uint2 *>(to + KEYS + (((group >> 1) * NT + f) * 64 + lane) * 16 + 8 * (group & 1)) =
                make_uint2(value_pair<PACKED>(raw_codes[word], raw_codes[VW + word], f, off),
                           value_pair<PACKED>(raw_codes[2 * VW + word], raw_codes[3 * VW + word], f, off));
        }
    };

    look_up(0);
    load(0);

    // ---- queries: steps folded in, digits, 8 rows at a time through memory of the wave's own
    constexpr int LR = DP <= 64 ? 8 : DP <= 128 ? 16 : 32, PASS = 64 / LR, PASSES = 16 / PASS;
    const int qc = lane % LR, qc0 = 8 * qc < DP ? 8 * qc : 0;
    int8_t *const digits = reinterpret_cast<int8_t *>(stage) + wave * rows_digits(TYPE, DP);
    float step[8];
    kv_load_floats8(kv.key.s + h * DP + qc0, step);
    auto load_queries = [&](int i) {
        const int r = row0 + i * PASS + lane / LR;
        const bool on = i < PASSES && r < rows && 8 * qc < DP;
        const int64_t qat = (int64_t)b * q.ld_seq + (int64_t)(r / q.group) * q.ld_token + (int64_t)(h * q.group + r % q.group) * q.ld_head;
        return kv_load8(q.p, TYPE, qat + qc0, on ? kv.dim - qc0 : 0);
    };
    v4i qd[ND][NS];          // lane (n, g): features 64 st + 16 g .. + 15 of row n
    Raw8 raw = load_queries(0);
#pragma unroll
    for (int eight = 0; eight < 2; ++eight) {
#pragma unroll 1
        for (int i = eight * PASSES / 2; i < (eight + 1) * PASSES / 2; ++i) {
            const int r16 = i * PASS + lane / LR;
            float x[8], back;
            kv_floats8(raw, TYPE, kv.dim - qc0, x);
            raw = load_queries(i + 1);
            if (a.lse) {
                const float offset = query_offset<LR>(x, step, kv.key.k + h * DP + qc0, a.scale);
                if (qc == 0) row_shift[16 * wave + r16] = offset;
            }
            const float most = query_steps<LR>(x, step, &back);
            if (8 * qc < DP) query_digits8<ND, PACKED>(x, most, a.scale, QMAX, digits + (r16 & 7) * (DP + 16), 8 * (DP + 16), qc);
            if (qc == 0) row_scale[16 * wave + r16] = most == INFINITY ? -1.0f : score_scale<PACKED>(most, QMAX, back, a.scale);
        }
        wave_order();
        if (n >> 3 == eight) {
#pragma unroll
            for (int dd = 0; dd < ND; ++dd)
#pragma unroll
                for (int st = 0; st < NS; ++st) qd[dd][st] = *reinterpret_cast<const v4i *>(digits + (dd * 8 + (n & 7)) * (DP + 16) + 64 * st + 16 * g);
        }
        wave_order();
    }
    const float rs = row_scale[16 * wave + n], scale = fabsf(rs);      // of the scores (integers so far)
    float m = NEG;           // their maximum, as an integer
    // What rows see: .x positions from .y on, and those below .z.
    if (threadIdx.x < TILE_ROWS) {
        const int r = tile0 + threadIdx.x, me = r < rows ? len - q.new_tokens + r / q.group : -1;
        const int first = window_from(a, me), sinks = me < a.sinks ? me + 1 : a.sinks;
        row_sees[threadIdx.x] = me < 0 ? make_int4(0, 0, 0, 0) : make_int4(me + 1 - first, first, sinks, 0);
    }
    // A group that ends at or before `seen` and begins at or behind `windows` is seen by all of the wave's rows.
    const RowTokens mine = row_tokens(q, working ? row0 : tile0, 16);
    const int seen = len - q.new_tokens + mine.from, windows = window_from(a, len - q.new_tokens + mine.to);

    v4f l = {0.f, 0.f, 0.f, 0.f}, acc[NT];
    v8h ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (_Float16)1.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = v4f{0.f, 0.f, 0.f, 0.f};
    __syncthreads();               // the digits are read: the buffers are free
    keep(0);
    if (turns > 1) load(1);
    __syncthreads();

    for (int turn = 0; turn < turns; ++turn) {
        const char *const here = stage + (turn & 1) * STAGE;
        if (working) {
            int pos[4];
            {
                const int4 p = *reinterpret_cast<const int4 *>(group_at[turn & 1]);
                pos[0] = __builtin_amdgcn_readfirstlane(p.x); pos[1] = __builtin_amdgcn_readfirstlane(p.y);
                pos[2] = __builtin_amdgcn_readfirstlane(p.z); pos[3] = __builtin_amdgcn_readfirstlane(p.w);
            }
            // 32 tokens at a time
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                const int first = half ? pos[2] : pos[0], second = half ? pos[3] : pos[1];
                const bool part = first > seen - 15 || second > seen - 15 || first < windows || second < windows;
                float s[2][4];
#pragma unroll
                for (int tg = 0; tg < 2; ++tg) {
                    v4i sum[ND];
#pragma unroll
                    for (int dd = 0; dd < ND; ++dd) sum[dd] = v4i{INT_AS_FLOAT, INT_AS_FLOAT, INT_AS_FLOAT, INT_AS_FLOAT};
#pragma unroll
                    for (int st = 0; st < NS; ++st) {
                        const v4i kf = *reinterpret_cast<const v4i *>(here + (((2 * half + tg) * NS + st) * 64 + lane) * 16);
#pragma unroll
                        for (int dd = 0; dd < ND; ++dd) sum[dd] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf, qd[dd][st], sum[dd], 0, 0, 0);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[tg][j] = shifted_score<ND>(sum, j);
                }
                if (part) {
                    asm volatile("");      // a branch: few tiles need it
                    const int4 row = row_sees[16 * wave + n];
#pragma unroll
                    for (int tg = 0; tg < 2; ++tg) {
                        const int at16 = tg ? second : first;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int e = 4 * g + j;
                            const bool sees = (unsigned)(at16 - row.y) + e < (unsigned)row.x || at16 < row.z - e;
                            if (!sees) s[tg][j] = NEG;
                        }
                    }
                }
                float top = s[0][0];
#pragma unroll
                for (int tg = 0; tg < 2; ++tg)
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = fmaxf(top, s[tg][j]);
                if (__any((top - m) * scale > HEADROOM)) {
                    top = fmaxf(top, __shfl_xor(top, 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    const float next = fmaxf(m, top);
                    const float f = next == NEG ? 1.0f : __builtin_amdgcn_exp2f((m - next) * scale);
                    m = next;
                    l *= f;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[t][j] *= f;
                }
                const float most = m == NEG ? 0.0f : m;
                float up = LIFT - most * scale;
                if (NP == 2 || __any(fabsf(up) > FAR)) {       // a difference of numbers this large keeps too little of it
                    asm volatile("");
#pragma unroll
                    for (int tg = 0; tg < 2; ++tg)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[tg][j] -= most;
                    up = LIFT;
                }
                v8h w[NP];
#pragma unroll
                for (int tg = 0; tg < 2; ++tg)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tg][j], scale, up));
                        const _Float16 p0 = (_Float16)p;
                        w[0][tg * 4 + j] = p0;
                        if constexpr (NP == 2) w[1][tg * 4 + j] = (_Float16)(p - (float)p0);
                    }
#pragma unroll
                for (int p = 0; p < NP; ++p) l = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, w[p], l, 0, 0, 0);
#pragma unroll
                for (int f = 0; f < NT; ++f) {
                    const v8h vf = *reinterpret_cast<const v8h *>(here + KEYS + ((half * NT + f) * 64 + lane) * 16);
#pragma unroll
                    for (int p = 0; p < NP; ++p) acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, w[p], acc[f], 0, 0, 0);
                }
            }
        }
        if (turn + 1 < turns) {
            keep((turn + 1) & 1);
            if (((turn + 2) & 63) == 0) look_up(turn + 2);
            if (turn + 2 < turns) load(turn + 2);
        }
        __syncthreads();
    }
    asm volatile("s_nop 15");      // the last matrix results are read in other blocks of code

    // ---- results
    const int r = row0 + n;
    if (r >= rows) return;
    // a row that is not finite is not a number from the first token on that it sees
    const float sum = rs < 0.0f && l[0] > 0.0f ? NAN : l[0], inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int64_t out_row = (int64_t)b * a.ldo_seq + (int64_t)(r / q.group) * a.ldo_token + (int64_t)(h * q.group + r % q.group) * a.ldo_head;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int f = 0; f < NT; f += 4) {
            const int c0 = feature_of<DP, PACKED>(4 * g + j, f);
            const float4 vs = *reinterpret_cast<const float4 *>(kv.value.s + h * DP + c0), vk = *reinterpret_cast<const float4 *>(kv.value.k + h * DP + c0);
            const float by[4] = {vs.x, vs.y, vs.z, vs.w}, from[4] = {vk.x, vk.y, vk.z, vk.w};
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = sum == 0.0f ? 0.0f : (acc[f + e][j] * VALUE_SCALE * inv + 0.5f) * by[e] + from[e];
            kv_store<4>(a.out, TYPE, out_row + c0, kv.dim - c0, x);
        }
    if (a.lse && g == 0) {
        const int64_t at = ((int64_t)b * q.new_tokens + r / q.group) * ((int64_t)kv.heads * q.group) + h * q.group + r % q.group;
        a.lse[at] = sum == 0.0f ? NEG : ((m - SCORE_SHIFT) * scale - LIFT + __log2f(sum)) * 0.69314718055994531f + row_shift[16 * wave + n];
    }
}

// Parts of a row joined, o = sum_u o_u 2^(m_u - m) / sum_u l_u 2^(m_u - m): a workgroup of NT threads per row, dpad / 4 of them side by
// side per part.  Bound by two round trips to memory (which parts, then the parts, all asked for at once up to 4 per thread): 1024 rows
// of 2 to 8 parts 4.7 us, 4096 rows 6.4, 32 rows of 32 parts 4.0.
template <int NT, bool MASKED>
__global__ __launch_bounds__(NT) void kv_join_kernel(KvView kv, KvQueries q, KvAttend a, int row_tiles, int tile_rows, int grid)
{
    __shared__ float4 sums[NT];
    __shared__ float weight[KV_ATTEND_SHARES];
    __shared__ float red[NT / 64], redl[NT / 64];
    const int rows = q.new_tokens * q.group;
    const int r = blockIdx.x % rows, bh = blockIdx.x / rows, h = bh % kv.heads, b = bh / kv.heads;
    const Workspace ws = workspace(a.part, 2 * (int64_t)grid, tile_rows, kv.dpad);
    const Parts parts = ws.parts[MASKED ? (int64_t)bh * row_tiles + r / tile_rows : bh];
    if (parts.count <= 1) return;
    const int cols = kv.dpad >> 2, groups = NT / cols;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row_tile = r / tile_rows, inside = r - row_tile * tile_rows;
    auto row_of = [&](int u) { return (2 * (((int64_t)parts.first + u) * row_tiles + row_tile) + (u == 0 ? 1 : 0)) * tile_rows + inside; };
    const int col = tid % cols, grp = tid / cols;
    // the first parts' sums are under way while the weights are made
    auto sums_of = [&](int u) { return *reinterpret_cast<const float4 *>(ws.sums + row_of(u < parts.count ? u : 0) * kv.dpad + 4 * col); };
    constexpr int AHEAD = 4;
    float4 ahead[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ahead[i] = sums_of(grp + i * groups);
    float top = NEG;
    for (int u = tid; u < parts.count; u += NT) {
        const float m = ws.ml[row_of(u) * 2];
        weight[u] = m;
        top = fmaxf(top, m);
    }
    top = __uint_as_float(wave_all(__float_as_uint(top), [](uint32_t x, uint32_t y) { return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y))); }));
    if (lane == 0) red[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) top = fmaxf(top, red[w]);
    float l = 0.0f;
    for (int u = tid; u < parts.count; u += NT) {
        const float f = lag(weight[u], top);
        weight[u] = f;
        l += ws.ml[row_of(u) * 2 + 1] * f;
    }
    l = __uint_as_float(wave_all(__float_as_uint(l), [](uint32_t x, uint32_t y) { return __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); }));
    if (lane == 0) redl[wave] = l;
    __syncthreads();
    l = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) l += redl[w];
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (grp < groups) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float f = grp + i * groups < parts.count ? weight[grp + i * groups] : 0.0f;
            const float4 y = ahead[i];
            if (f != 0.0f) { x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f; }
        }
#pragma unroll 4
        for (int u = grp + AHEAD * groups; u < parts.count; u += groups) {
            const float f = weight[u];
            const float4 y = sums_of(u);
            x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
        }
        sums[tid] = x;
    }
    __syncthreads();
    if (grp) return;
    for (int o = 1; o < groups; ++o) {
        const float4 y = sums[o * cols + col];
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    }
    const int c0 = 4 * col;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const float *vs = kv.value.s + h * kv.dpad + c0, *vk = kv.value.k + h * kv.dpad + c0;
    float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = l == 0.0f ? 0.0f : (v[e] * inv + 0.5f) * vs[e] + vk[e];
    const int64_t out_row = (int64_t)b * a.ldo_seq + (int64_t)(r / q.group) * a.ldo_token + (int64_t)(h * q.group + r % q.group) * a.ldo_head;
    kv_store<4>(a.out, q.type, out_row + c0, kv.dim - c0, v);
    if (a.lse && col == 0) {
        const int64_t lat = ((int64_t)b * q.new_tokens + r / q.group) * ((int64_t)kv.heads * q.group) + h * q.group + r % q.group;
        a.lse[lat] = l == 0.0f ? NEG : (top * (1.0f / MAXIMUM) - LIFT + __log2f(l)) * 0.69314718055994531f + a.lse[lat];
    }
}

template <int DP, bool PACKED, int TYPE, typename CALL>
void launch_rows(const KvView &kv, const KvQueries &q, const CALL &a, const KvAttendPlan &p, hipStream_t st)
{
    if constexpr (std::is_same<CALL, KvWindow>::value) {
        if (p.rows == ROWS_TILE) {
            kv_rows_kernel<DP, PACKED, TYPE><<<p.grid, ROWS_THREADS, 0, st>>>(kv, q, a, p.row_tiles);
            return;
        }
    }
    if constexpr (two_row_tiles(DP, PACKED, TYPE, std::is_same<CALL, KvTree>::value)) {
        if (p.rows == 32) {
            kv_attend_kernel<DP, PACKED, 2, TYPE><<<p.grid, THREADS, 0, st>>>(kv, q, a, p.row_tiles, p.least);
            return;
        }
    }
    kv_attend_kernel<DP, PACKED, 1, TYPE><<<p.grid, THREADS, 0, st>>>(kv, q, a, p.row_tiles, p.least);
}

template <int DP, int TYPE, typename CALL>
void launch_codes(const KvView &kv, const KvQueries &q, const CALL &a, const KvAttendPlan &p, hipStream_t st)
{
    if (kv.packed) launch_rows<DP, true, TYPE>(kv, q, a, p, st);
    else launch_rows<DP, false, TYPE>(kv, q, a, p, st);
}

template <int DP, typename CALL>
void launch_dim(const KvView &kv, const KvQueries &q, const CALL &a, const KvAttendPlan &p, hipStream_t st)
{
    if (q.type == LPQ_TYPE_F32) launch_codes<DP, LPQ_TYPE_F32>(kv, q, a, p, st);
    else if (q.type == LPQ_TYPE_F16) launch_codes<DP, LPQ_TYPE_F16>(kv, q, a, p, st);
    else launch_codes<DP, LPQ_TYPE_BF16>(kv, q, a, p, st);
}

template <typename CALL>
hipError_t launch_all(const KvView &kv, const KvQueries &q, const CALL &a, const KvAttendPlan &p, hipStream_t st)
{
    switch (kv.dpad) {
    case 64: launch_dim<64>(kv, q, a, p, st); break;
    case 128: launch_dim<128>(kv, q, a, p, st); break;
    case 192: launch_dim<192>(kv, q, a, p, st); break;
    default: launch_dim<256>(kv, q, a, p, st); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.least == 0) return e;
    const unsigned rows = (unsigned)((int64_t)a.nseq * kv.heads * q.new_tokens * q.group);
    constexpr bool MASKED = !std::is_same<CALL, KvAttend>::value;
    // Many rows fill the chip with a wave each, few rows of many parts want more.
    if (rows >= 1024) kv_join_kernel<64, MASKED><<<rows, 64, 0, st>>>(kv, q, a, p.row_tiles, p.rows, (int)p.grid);
    else kv_join_kernel<256, MASKED><<<rows, 256, 0, st>>>(kv, q, a, p.row_tiles, p.rows, (int)p.grid);
    return hipGetLastError();
}

}  // namespace

// Short sequences get a workgroup per pair and row tile: joining parts would cost more than it gives.  Otherwise as many workgroups as
// the chip holds at once, and no fewer than 4 tiles each.  Short is up to 1024 tokens, of more than 128 features fewer where workgroups are
// few: 16 pairs, whole against split and joined, us: 1000 tokens of 64 features 10.9, 12.8, of 128 13.6, 13.5, of 256 19.6, 17.2; 500 of 256
// 15.6, 16.1.  512 pairs of 128, 1000 tokens: 24.4, 31.3.  Nor are sequences split where a pair's row tiles fill the chip by themselves: 16 384
// bfloat16 rows on one head of 128, 2000 tokens 69 us, split into 8 shares and joined 135, 50 000 tokens 1123, 1168 (and 136 MB of parts).
KvAttendPlan kv_attend_plan(const KvView &kv, int64_t nseq, int new_tokens, int group, int64_t tokens, int type, const KvMask &mask)
{
    KvAttendPlan p;
    const int64_t rows = (int64_t)new_tokens * group;
    const int64_t pairs = nseq * kv.heads;
    // What a row tile has to go through at most, of tokens that lie side by side: the sinks, and the windows of its new tokens.
    if (mask.window) tokens = std::min<int64_t>(tokens, round_up((int64_t)mask.sinks, 16) + mask.window + std::min<int64_t>(new_tokens, 128 / group + 2) + 30);
    const int64_t row_tiles = ceil_div(rows, (int64_t)ROWS_TILE);
    if (mask.window && rows > 32 && row_tiles * pairs >= 256 * rows_blocks_per_cu(kv.dpad)) return {(int)row_tiles, ROWS_TILE, 0, (unsigned)round_up(row_tiles * pairs, 8), 0};
    p.rows = rows > 16 && pairs * tokens > TWO_ROW_TOKENS && two_row_tiles(kv.dpad, kv.packed, type, mask.tree != nullptr) ? 32 : 16;
    p.row_tiles = (int)ceil_div(rows, (int64_t)p.rows);
    const int64_t tile = tile_tokens(kv.dpad, kv.packed);
    p.least = 0;
    p.grid = (unsigned)(pairs * p.row_tiles);
    p.bytes = 0;
    const int64_t tiles = ceil_div(tokens, tile);
    const bool few = (int64_t)p.grid < 256 && tokens * kv.dpad > 128 * 1024;
    const int64_t chip = std::min<int64_t>(256 * blocks_per_cu(kv.dpad, kv.packed, p.rows / 16, type, mask.window != 0), KV_ATTEND_SHARES);
    if ((tokens > 1024 || few) && p.row_tiles < chip && pairs * tiles < (int64_t(1) << 31)) {      // (beyond that there are pairs enough)
        p.least = 4;
        const int64_t most = ceil_div(tiles, (int64_t)p.least) * pairs;
        const int64_t room = ceil_div(chip, (int64_t)p.row_tiles);
        int64_t shares = most < room ? most : room;
        // Not a workgroup more than the chip holds at once, which would be a second generation of them: 96 bfloat16 rows on 8 heads of 128, 32
        // sequences of 900 to 8000 tokens, 528 workgroups 181 us, 504 161; 720 float32 rows on one of 192 31.6, 25.5.
        if (p.row_tiles > 1) shares = (mask.window || mask.tree) && room > 8 && shares > room / 8 * 8 ? room / 8 * 8 : round_up(shares, 8);
        p.grid = (unsigned)(shares * p.row_tiles);
        p.bytes = ((size_t)2 * p.grid * p.rows * (kv.dpad + 2) + (size_t)2 * pairs * (mask.window || mask.tree ? p.row_tiles : 1)) * sizeof(float);
    }
    return p;
}

hipError_t launch_kv_attend(const KvView &kv, const KvQueries &q, const KvAttend &a, const KvMask &mask, const KvAttendPlan &p, hipStream_t st)
{
    if (a.nseq <= 0) return hipSuccess;
    if (mask.window) return launch_all(kv, q, KvWindow{a, mask.window, mask.sinks}, p, st);
    if (mask.tree) return launch_all(kv, q, KvTree{a, mask.tree, mask.ldt_seq, mask.ldt_token}, p, st);
    return launch_all(kv, q, a, p, st);
}

}  // namespace lpq
