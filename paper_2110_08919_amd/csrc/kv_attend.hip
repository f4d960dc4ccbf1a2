// Attention of new tokens over a key-value cache held as codes: o = sum_j softmax_j(scale q . x^_j) y^_j over the tokens
// of all pages of a sequence, or of listed ones.
//
// Mathematics.  A key reads back as x^_i = k_i + (c_i + 1/2) s_i, so q . x^ = sum_i (q_i s_i) c_i + sum_i q_i (k_i + s_i / 2).
// The second sum is the same for every token and drops out of the softmax: the query takes the steps, and the codes enter
// the products as the integers they are.  Likewise o_i = k_i + s_i (1/2 + sum_j p_j c_ji / sum_j p_j).
//
// Scores on the int8 matrix instruction (16x16x64), so that key codes need no conversion: a row of q' = q s is rounded to
// Q = rint(q' Qmax / max |q'|) and split into signed digits of 7 bits, one product each, summed exactly in int32.  Two
// digits for 16-bit queries (Qmax = 16319: an error of 2^-15 of the row's largest q', where bfloat16 holds 2^-9 of each
// value), three for float32 (Qmax = 2088895, 2^-22).
// Weights exp2(t - m) are rounded to fp16 (float32 calls: two fp16 terms) and multiply the value codes, which fp16 holds
// exactly, on the fp16 matrix instruction with float32 sums.  The sum of weights is taken of the rounded ones.  m is a
// maximum that may lag behind by 2^8 (the weights of a tile reach 2^14 then, and 2^-24 below that the smallest that counts):
// it moves, and the sums are rescaled, only in tiles where a score passes it by more.
//
// Layout.  Tokens are the rows of the first product (S^T = K Q^T) and the summed index of the second (O^T = V^T P^T), so
// the registers that hold scores of a token group are the operand of the second product as they are: register j of lane
// (n, g) holds query row n and token 4 g + j of its group of 16, and the second product takes its 8 tokens per lane as
// 4 g .. 4 g + 3 of two groups.  A lane owns dpad / 16 neighbouring features of the values: it loads them from the rows
// of its 8 tokens and gathers the operand of each with byte permutes.  Nothing goes through LDS until the end.  Each wave
// walks its own tiles of 64 (or 32) tokens with the next tile's loads in flight.
#include "kv_internal.h"

namespace lpq {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int THREADS = 256, WAVES = 4;
constexpr float NEG = -INFINITY;
constexpr float HEADROOM = 8.0f;     // how far scores may pass the maximum before it moves (powers of two)
constexpr float LIFT = 6.0f;         // weights are exp2(t - m + LIFT): at most 2^14, and small ones stay normal fp16

// Tiles of a sequence's tokens, and how they are dealt to the parts of a call.
struct Deal {
    int64_t tokens;
    int tiles, per, used;      // per part; parts that have any
};
__device__ __forceinline__ Deal deal(int64_t tokens, int tile, int splits)
{
    Deal d;
    d.tokens = tokens;
    d.tiles = (int)((tokens + tile - 1) / tile);
    const int even = (d.tiles + splits - 1) / splits;
    d.per = even > WAVES ? even : WAVES;
    d.used = (d.tiles + d.per - 1) / d.per;
    return d;
}

template <int DP>
constexpr int tile_tokens() { return DP <= 128 ? 64 : 32; }

__device__ __forceinline__ int64_t call_tokens(const KvView &kv, const KvAttend &a, int b)
{
    int64_t len = a.lengths[b];
    const int64_t room = (int64_t)a.table_pages << kv.page_shift;
    len = len < 0 ? 0 : (len > room ? room : len);
    if (a.chosen && len > 0) {
        const int64_t listed = (int64_t)a.n_select << kv.page_shift;
        return listed;
    }
    return len;
}

// Bytes of a lane's share of a value row.
template <int BYTES>
__device__ __forceinline__ void load_share(const uint8_t *p, uint32_t *w)
{
    if constexpr (BYTES == 16) {
        const uint4 t = *reinterpret_cast<const uint4 *>(p);
        w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w;
    } else if constexpr (BYTES == 12) {
        const uint3 t = *reinterpret_cast<const uint3 *>(p);
        w[0] = t.x; w[1] = t.y; w[2] = t.z;
    } else if constexpr (BYTES == 8) {
        const uint2 t = *reinterpret_cast<const uint2 *>(p);
        w[0] = t.x; w[1] = t.y;
    } else if constexpr (BYTES == 6) {
        const uint16_t *t = reinterpret_cast<const uint16_t *>(p);
        w[0] = (uint32_t)t[0] | (uint32_t)t[1] << 16;
        w[1] = t[2];
    } else if constexpr (BYTES == 4) {
        w[0] = *reinterpret_cast<const uint32_t *>(p);
    } else {
        w[0] = *reinterpret_cast<const uint16_t *>(p);
    }
}

// One tile in registers.
template <int DP, bool PACKED>
struct Tile {
    static constexpr int TG = tile_tokens<DP>() / 16, NS = DP / 64, NT = DP / 16;
    static constexpr int VB = PACKED ? NT / 2 : NT, VW = (VB + 3) / 4;
    uint32_t k[TG][NS][PACKED ? 2 : 4];
    uint32_t v[TG / 2][8][VW];
    int pos[TG];          // position of a group's first token; INT32_MAX: the group does not count
};

// Halves [features t of token e | of token e + 1] as fp16, from the two tokens' shares of a row.
template <bool PACKED>
__device__ __forceinline__ uint32_t value_pair(uint32_t w0, uint32_t w1, int t)
{
    const int byte = PACKED ? (t >> 1) & 3 : t & 3;
    const uint32_t sel = 0x0c000c00u | (uint32_t)byte | (uint32_t)(4 + byte) << 16;
    const uint32_t x = __builtin_amdgcn_perm(w1, w0, sel);
    if constexpr (!PACKED) {
        const v2h off = {(_Float16)1152.0f, (_Float16)1152.0f};                 // 1024 + 128 + c, less that: exact
        const v2h y = __builtin_bit_cast(v2h, x ^ 0x64806480u) - off;
        return __builtin_bit_cast(uint32_t, y);
    } else if ((t & 1) == 0) {
        const v2h off = {(_Float16)1032.0f, (_Float16)1032.0f};                 // 1024 + 8 + c
        const v2h y = __builtin_bit_cast(v2h, (x & 0x000f000fu) | 0x64006400u) - off;
        return __builtin_bit_cast(uint32_t, y);
    } else {
        const v2h off = {(_Float16)1152.0f, (_Float16)1152.0f}, f = {(_Float16)0.0625f, (_Float16)0.0625f};
        const v2h y = (__builtin_bit_cast(v2h, (x & 0x00f000f0u) | 0x64006400u) - off) * f;    // 1024 + 128 + 16 c
        return __builtin_bit_cast(uint32_t, y);
    }
}

template <int DP, bool PACKED, int RT, bool WIDE>
__global__ __launch_bounds__(THREADS) void kv_attend_kernel(KvView kv, KvQueries q, KvAttend a, int row_tiles, int splits)
{
    typedef Tile<DP, PACKED> T;
    constexpr int TG = T::TG, NS = T::NS, NT = T::NT, VB = T::VB, TOK = 16 * TG;
    constexpr int ND = WIDE ? 3 : 2, NP = WIDE ? 2 : 1, RB = PACKED ? DP / 2 : DP;
    constexpr float QMAX = WIDE ? 2088895.0f : 16319.0f;
    __shared__ float red_m[WAVES][16 * RT], red_l[WAVES][16 * RT];
    __shared__ float sums[WAVES][16][DP + 4];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    int id = blockIdx.x;
    const int h = id % kv.heads;
    id /= kv.heads;
    const int row_tile = id % row_tiles;
    id /= row_tiles;
    const int b = id % a.nseq, split = id / a.nseq;
    const int rows = q.new_tokens * q.group, row0 = row_tile * 16 * RT;
    int64_t len = a.lengths[b];
    {
        const int64_t room = (int64_t)a.table_pages << kv.page_shift;
        len = len < 0 ? 0 : (len > room ? room : len);
    }
    const Deal d = deal(call_tokens(kv, a, b), TOK, splits);
    if (split > 0 && split >= d.used) return;

    // ---- queries: steps folded in, digits; lane (n, g) holds features 64 st + 16 g .. + 15 of row n
    v4i qd[RT][ND][NS];
    v4i q0[RT][ND];          // packed keys hold c + 8: what that adds to each sum is taken off at its start
    float rs[RT], shift[RT], m[RT], l[RT];
    int last[RT];            // last position a row sees
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = row0 + rt * 16 + n;
        const bool on = r < rows;
        const int64_t at = (int64_t)b * q.ld_seq + (int64_t)(r / q.group) * q.ld_token + (int64_t)(h * q.group + r % q.group) * q.ld_head;
        float x[NS][16];
        float most = 0.0f, offset = 0.0f;
        bool bad = false;
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
            for (int e0 = 0; e0 < 16; e0 += 8) {
                const int c0 = 64 * st + 16 * g + e0;
                float *v = &x[st][e0];
                kv_load8(q.p, q.type, on ? at + c0 : 0, on ? kv.dim - c0 : 0, q.vec, v);
                const float *step = kv.key.s + h * DP + c0, *k = kv.key.k + h * DP + c0;
                if (a.lse) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) offset += v[e] * (k[e] + 0.5f * step[e]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] *= step[e];
                    most = fmaxf(most, fabsf(v[e]));
                    bad |= !(fabsf(v[e]) <= 3.402823466e38f);
                }
            }
        most = fmaxf(most, __shfl_xor(most, 16, 64));
        most = fmaxf(most, __shfl_xor(most, 32, 64));
        offset += __shfl_xor(offset, 16, 64);
        offset += __shfl_xor(offset, 32, 64);
        int any = bad;
        any |= __shfl_xor(any, 16, 64);
        any |= __shfl_xor(any, 32, 64);
        const bool use = !any && most > 1e-30f;      // below that QMAX / most leaves the range of binary32, and scores are 0
        const float f = use ? QMAX / most : 0.0f;
        rs[rt] = any ? NAN : (use ? most / QMAX * a.scale * 1.44269504088896f : 0.0f);
        shift[rt] = offset * a.scale;
        int dsum[ND];
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) dsum[dd] = 0;
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            int8_t digit[ND][16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                // packed: low nibbles (even features) first, then the high ones
                const int src = PACKED ? (e < 8 ? 2 * e : 2 * (e - 8) + 1) : e;
                int v = use ? (int)rintf(x[st][src] * f) : 0;
#pragma unroll
                for (int dd = ND - 1; dd > 0; --dd) {
                    const int up = (v + 64) >> 7, low = v - (up << 7);       // low in -64 .. 63
                    digit[dd][e] = (int8_t)low;
                    dsum[dd] += low;
                    v = up;
                }
                digit[0][e] = (int8_t)v;
                dsum[0] += v;
            }
#pragma unroll
            for (int dd = 0; dd < ND; ++dd) __builtin_memcpy(&qd[rt][dd][st], digit[dd], 16);
        }
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) {
            int v = 0;
            if (PACKED) {
                v = dsum[dd];
                v += __shfl_xor(v, 16, 64);
                v += __shfl_xor(v, 32, 64);
                v *= -8;
            }
            q0[rt][dd] = v4i{v, v, v, v};
        }
        m[rt] = NEG;
        l[rt] = 0.0f;
        const int64_t see = len - q.new_tokens + r / q.group;
        last[rt] = on ? (int)(see < -1 ? -1 : see) : -1;
    }
    const int64_t least64 = len - q.new_tokens;      // a tile that ends at or before this position is seen by every row
    const int least = (int)(least64 < -1 ? -1 : least64);

    v4f acc[RT][NT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[rt][t] = v4f{0.f, 0.f, 0.f, 0.f};

    const int32_t *table = a.table + (int64_t)b * a.ld_table;
    const int32_t *chosen = a.chosen ? a.chosen + ((int64_t)b * kv.heads + h) * a.n_select : nullptr;
    const int64_t head_bytes = (int64_t)kv.page * RB;

    // Page of the pool and position of group `grp` of the call's tokens; page -1 where there is none.
    auto place = [&](int64_t grp, int &page, int &pos) {
        const int64_t at = grp * 16;
        int column = (int)(at >> kv.page_shift);
        const int inside = (int)at & (kv.page - 1);
        page = -1;
        pos = INT32_MAX;
        if (chosen) {
            if (column >= a.n_select) return;
            column = chosen[column];
            if (column < 0 || column >= a.table_pages) return;
        }
        const int64_t p = ((int64_t)column << kv.page_shift) + inside;
        if (p >= len) return;
        const int id_ = table[column];
        if (id_ < 0 || id_ >= kv.pages) return;
        page = id_;
        pos = (int)p;
    };
    struct Ids { int page[TG], pos[TG]; };
    auto find = [&](int tile, Ids &i) {
#pragma unroll
        for (int tg = 0; tg < TG; ++tg) place((int64_t)tile * TG + tg, i.page[tg], i.pos[tg]);
    };
    auto load = [&](const Ids &i, T &t) {
#pragma unroll
        for (int tg = 0; tg < TG; ++tg) {
            const int page = i.page[tg] < 0 ? 0 : i.page[tg];
            const int row = i.page[tg] < 0 ? 0 : i.pos[tg] & (kv.page - 1);
            t.pos[tg] = i.pos[tg];
            const int64_t at = ((int64_t)page * kv.heads + h) * head_bytes + (int64_t)row * RB;
            const uint8_t *kp = kv.k + at + n * RB + g * (PACKED ? 8 : 16);
#pragma unroll
            for (int st = 0; st < NS; ++st) {
                if constexpr (PACKED) {
                    const uint2 w = *reinterpret_cast<const uint2 *>(kp + 32 * st);
                    t.k[tg][st][0] = w.x; t.k[tg][st][1] = w.y;
                } else {
                    const uint4 w = *reinterpret_cast<const uint4 *>(kp + 64 * st);
                    t.k[tg][st][0] = w.x; t.k[tg][st][1] = w.y; t.k[tg][st][2] = w.z; t.k[tg][st][3] = w.w;
                }
            }
            const uint8_t *vp = kv.v + at + (4 * g) * RB + n * VB;
#pragma unroll
            for (int j = 0; j < 4; ++j) load_share<VB>(vp + j * RB, t.v[tg >> 1][(tg & 1) * 4 + j]);
        }
    };
    auto compute = [&](const T &t) {
        bool part = false;
#pragma unroll
        for (int tg = 0; tg < TG; ++tg) part |= t.pos[tg] > least - 15;     // also where a group does not count
        v8h w[RT][NP][TG / 2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float s[TG][4];
#pragma unroll
            for (int tg = 0; tg < TG; ++tg) {
                v4i sum[ND];
#pragma unroll
                for (int dd = 0; dd < ND; ++dd) sum[dd] = q0[rt][dd];
#pragma unroll
                for (int st = 0; st < NS; ++st) {
                    v4i kf;
                    if constexpr (PACKED) {
                        const uint32_t x = t.k[tg][st][0], y = t.k[tg][st][1];
                        kf = v4i{(int)(x & 0x0f0f0f0fu), (int)(y & 0x0f0f0f0fu), (int)((x >> 4) & 0x0f0f0f0fu), (int)((y >> 4) & 0x0f0f0f0fu)};
                    } else {
                        kf = v4i{(int)t.k[tg][st][0], (int)t.k[tg][st][1], (int)t.k[tg][st][2], (int)t.k[tg][st][3]};
                    }
#pragma unroll
                    for (int dd = 0; dd < ND; ++dd) sum[dd] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf, qd[rt][dd][st], sum[dd], 0, 0, 0);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (WIDE) s[tg][j] = ((float)sum[0][j] * 16384.0f + (float)(sum[1][j] * 128 + sum[2][j])) * rs[rt];
                    else s[tg][j] = (float)(sum[0][j] * 128 + sum[1][j]) * rs[rt];
                }
            }
            if (part) {
#pragma unroll
                for (int tg = 0; tg < TG; ++tg)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (t.pos[tg] > last[rt] - (4 * g + j)) s[tg][j] = NEG;
            }
            float top = s[0][0];
#pragma unroll
            for (int tg = 0; tg < TG; ++tg)
#pragma unroll
                for (int j = 0; j < 4; ++j) top = fmaxf(top, s[tg][j]);
            if (__any(top > m[rt] + HEADROOM)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float next = fmaxf(m[rt], top);
                const float f = next == NEG ? 1.0f : __builtin_amdgcn_exp2f(m[rt] - next);
                m[rt] = next;
                l[rt] *= f;
#pragma unroll
                for (int t_ = 0; t_ < NT; ++t_)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[rt][t_][j] *= f;
            }
            const float base = (m[rt] == NEG ? 0.0f : m[rt]) - LIFT;
            float add = 0.0f;
#pragma unroll
            for (int tg = 0; tg < TG; ++tg)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p = __builtin_amdgcn_exp2f(s[tg][j] - base);
                    const _Float16 p0 = (_Float16)p;
                    w[rt][0][tg >> 1][(tg & 1) * 4 + j] = p0;
                    add += (float)p0;
                    if constexpr (WIDE) {
                        const _Float16 p1 = (_Float16)(p - (float)p0);
                        w[rt][1][tg >> 1][(tg & 1) * 4 + j] = p1;
                        add += (float)p1;
                    }
                }
            l[rt] += add;
        }
#pragma unroll
        for (int half = 0; half < TG / 2; ++half)
#pragma unroll
            for (int f = 0; f < NT; ++f) {
                const int word = PACKED ? f >> 3 : f >> 2;
                uint32_t pair[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) pair[e] = value_pair<PACKED>(t.v[half][2 * e][word], t.v[half][2 * e + 1][word], f);
                v8h vf;
                __builtin_memcpy(&vf, pair, 16);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        acc[rt][f] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, w[rt][p][half], acc[rt][f], 0, 0, 0);
            }
    };

    // ---- the wave's tiles, one ahead in registers, places of the one after that known
    const int end = (split + 1) * d.per < d.tiles ? (split + 1) * d.per : d.tiles;
    int tile = split * d.per + __builtin_amdgcn_readfirstlane(wave);
    if (tile < end) {
        Ids ids;
        T t0, t1;
        find(tile, ids);
        load(ids, t0);
        if (tile + WAVES < end) find(tile + WAVES, ids);
        for (;;) {
            if (tile + WAVES < end) {
                load(ids, t1);
                if (tile + 2 * WAVES < end) find(tile + 2 * WAVES, ids);
            }
            compute(t0);
            tile += WAVES;
            if (tile >= end) break;
            if (tile + WAVES < end) {
                load(ids, t0);
                if (tile + 2 * WAVES < end) find(tile + 2 * WAVES, ids);
            }
            compute(t1);
            tile += WAVES;
            if (tile >= end) break;
        }
    }
    asm volatile("s_nop 15");      // the last matrix results are read in other blocks of code

    // ---- the waves' parts joined
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 16, 64);
        l[rt] += __shfl_xor(l[rt], 32, 64);
        if (g == 0) {
            red_m[wave][rt * 16 + n] = m[rt];
            red_l[wave][rt * 16 + n] = l[rt];
        }
    }
    __syncthreads();
    const bool whole = d.used <= 1;
    float *part = a.part;
    const int all_rows = row_tiles * 16 * RT;
    const int64_t part_at = (((int64_t)b * kv.heads + h) * splits + split) * all_rows + row0;     // row of the partial results
    float *part_ml = part + (int64_t)a.nseq * kv.heads * splits * all_rows * DP;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float top = NEG;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, red_m[w][rt * 16 + n]);
        const float f = top == NEG ? 1.0f : __builtin_amdgcn_exp2f(m[rt] - top);
        if (rt) __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int t = 0; t < NT; ++t) sums[wave][n][(4 * g + j) * NT + t] = acc[rt][t][j] * f;
        __syncthreads();
        const int r16 = threadIdx.x >> 4, r = row0 + rt * 16 + r16;
        if (r < rows) {
            float mm = NEG, ll = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) mm = fmaxf(mm, red_m[w][rt * 16 + r16]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
                ll += red_l[w][rt * 16 + r16] * (mm == NEG ? 1.0f : __builtin_amdgcn_exp2f(red_m[w][rt * 16 + r16] - mm));
            const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
            const int64_t out_row = (int64_t)b * a.ldo_seq + (int64_t)(r / q.group) * a.ldo_token + (int64_t)(h * q.group + r % q.group) * a.ldo_head;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const int c0 = 4 * ((threadIdx.x & 15) + 16 * i);
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float4 y = *reinterpret_cast<const float4 *>(&sums[w][r16][c0]);
                    x[0] += y.x; x[1] += y.y; x[2] += y.z; x[3] += y.w;
                }
                if (whole) {
                    const float *vs = kv.value.s + h * DP + c0, *vk = kv.value.k + h * DP + c0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = ll == 0.0f ? 0.0f : (x[e] * inv + 0.5f) * vs[e] + vk[e];
                    kv_store<4>(a.out, q.type, out_row + c0, kv.dim - c0, a.vec_out, x);
                } else {
                    *reinterpret_cast<float4 *>(part + (part_at + rt * 16 + r16) * DP + c0) = make_float4(x[0], x[1], x[2], x[3]);
                }
            }
            if ((threadIdx.x & 15) == 0 && !whole) {
                float *ml = part_ml + (part_at + rt * 16 + r16) * 2;
                ml[0] = mm;
                ml[1] = ll;
            }
        }
        if (whole && a.lse && wave == 0 && g == 0) {
            const int rr = row0 + rt * 16 + n;
            if (rr < rows) {
                float ll = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w)
                    ll += red_l[w][rt * 16 + n] * (top == NEG ? 1.0f : __builtin_amdgcn_exp2f(red_m[w][rt * 16 + n] - top));
                const int64_t at = ((int64_t)b * q.new_tokens + rr / q.group) * ((int64_t)kv.heads * q.group) + h * q.group + rr % q.group;
                a.lse[at] = ll == 0.0f ? NEG : (top - LIFT + __log2f(ll)) * 0.69314718055994531f + shift[rt];
            }
        }
        if (!whole && a.lse && split == 0 && wave == 0 && g == 0) {      // the joining kernel adds what every token has
            const int rr = row0 + rt * 16 + n;
            if (rr < rows) {
                const int64_t at = ((int64_t)b * q.new_tokens + rr / q.group) * ((int64_t)kv.heads * q.group) + h * q.group + rr % q.group;
                a.lse[at] = shift[rt];
            }
        }
    }
}

// Parts of a row joined: a workgroup per row, dpad / 4 threads side by side per part.
__global__ __launch_bounds__(THREADS) void kv_join_kernel(KvView kv, KvQueries q, KvAttend a, int all_rows, int splits, int tile)
{
    __shared__ float4 sums[THREADS];
    __shared__ float lsum[THREADS];
    const int rows = q.new_tokens * q.group;
    const int r = blockIdx.x % rows, pair = blockIdx.x / rows, h = pair % kv.heads, b = pair / kv.heads;
    const Deal d = deal(call_tokens(kv, a, b), tile, splits);
    if (d.used <= 1) return;
    const int64_t at = (int64_t)pair * splits * all_rows + r;
    const float *part = a.part, *ml = a.part + (int64_t)a.nseq * kv.heads * splits * all_rows * kv.dpad;
    const int cols = kv.dpad >> 2, groups = THREADS / cols, col = threadIdx.x % cols, grp = threadIdx.x / cols;
    float top = NEG;
    for (int u = 0; u < d.used; ++u) top = fmaxf(top, ml[(at + (int64_t)u * all_rows) * 2]);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.0f;
    if (grp < groups) {
        for (int u = grp; u < d.used; u += groups) {
            const int64_t row = at + (int64_t)u * all_rows;
            const float f = top == NEG ? 1.0f : __builtin_amdgcn_exp2f(ml[row * 2] - top);
            const float4 y = *reinterpret_cast<const float4 *>(part + row * kv.dpad + 4 * col);
            x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
            l += ml[row * 2 + 1] * f;
        }
        sums[threadIdx.x] = x;
        lsum[threadIdx.x] = l;
    }
    __syncthreads();
    if (grp) return;
    for (int o = 1; o < groups; ++o) {
        const float4 y = sums[o * cols + col];
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
        l += lsum[o * cols + col];
    }
    const int c0 = 4 * col;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const float *vs = kv.value.s + h * kv.dpad + c0, *vk = kv.value.k + h * kv.dpad + c0;
    float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = l == 0.0f ? 0.0f : (v[e] * inv + 0.5f) * vs[e] + vk[e];
    const int64_t out_row = (int64_t)b * a.ldo_seq + (int64_t)(r / q.group) * a.ldo_token + (int64_t)(h * q.group + r % q.group) * a.ldo_head;
    kv_store<4>(a.out, q.type, out_row + c0, kv.dim - c0, a.vec_out, v);
    if (a.lse && col == 0) {
        const int64_t lat = ((int64_t)b * q.new_tokens + r / q.group) * ((int64_t)kv.heads * q.group) + h * q.group + r % q.group;
        a.lse[lat] = l == 0.0f ? NEG : (top - LIFT + __log2f(l)) * 0.69314718055994531f + a.lse[lat];
    }
}

template <int DP, bool PACKED>
void launch_rows(const KvView &kv, const KvQueries &q, const KvAttend &a, const KvAttendPlan &p, unsigned blocks, hipStream_t st)
{
    const bool wide = q.type == LPQ_TYPE_F32;
    if (p.rows == 16) {
        if (wide) kv_attend_kernel<DP, PACKED, 1, true><<<blocks, THREADS, 0, st>>>(kv, q, a, p.row_tiles, p.splits);
        else kv_attend_kernel<DP, PACKED, 1, false><<<blocks, THREADS, 0, st>>>(kv, q, a, p.row_tiles, p.splits);
    } else {
        if (wide) kv_attend_kernel<DP, PACKED, 2, true><<<blocks, THREADS, 0, st>>>(kv, q, a, p.row_tiles, p.splits);
        else kv_attend_kernel<DP, PACKED, 2, false><<<blocks, THREADS, 0, st>>>(kv, q, a, p.row_tiles, p.splits);
    }
}

template <int DP>
void launch_dim(const KvView &kv, const KvQueries &q, const KvAttend &a, const KvAttendPlan &p, unsigned blocks, hipStream_t st)
{
    if (kv.packed) launch_rows<DP, true>(kv, q, a, p, blocks, st);
    else launch_rows<DP, false>(kv, q, a, p, blocks, st);
}

int plan_tile(int dpad) { return dpad <= 128 ? 64 : 32; }

}  // namespace

// Parts of a sequence: enough workgroups for two per CU, of no fewer than a tile per wave, and none longer than 4096 tokens,
// so that sequences of very different lengths end at about the same time.
KvAttendPlan kv_attend_plan(const KvView &kv, int64_t nseq, int new_tokens, int group, int64_t tokens)
{
    KvAttendPlan p;
    const int64_t rows = (int64_t)new_tokens * group;
    p.rows = rows <= 16 ? 16 : 32;
    p.row_tiles = (int)ceil_div(rows, (int64_t)p.rows);
    const int64_t base = nseq * kv.heads * p.row_tiles, tile = plan_tile(kv.dpad);
    const int64_t most = ceil_div(tokens, tile * WAVES);
    int64_t s = ceil_div(int64_t(512), base > 0 ? base : 1);
    const int64_t longest = ceil_div(tokens, int64_t(4096));
    if (s < longest) s = longest;
    if (s > most) s = most;
    if (base > 0 && s > KV_MAX_BLOCKS / base) s = KV_MAX_BLOCKS / base;
    if (s > 1024) s = 1024;
    p.splits = (int)(s < 1 ? 1 : s);
    const int64_t all = nseq * kv.heads * p.splits * p.row_tiles * p.rows;
    p.bytes = p.splits > 1 ? (size_t)all * (kv.dpad + 2) * sizeof(float) : 0;
    return p;
}

hipError_t launch_kv_attend(const KvView &kv, const KvQueries &q, const KvAttend &a, const KvAttendPlan &p, hipStream_t st)
{
    if (a.nseq <= 0) return hipSuccess;
    const unsigned blocks = (unsigned)((int64_t)a.nseq * kv.heads * p.row_tiles * p.splits);
    switch (kv.dpad) {
    case 64: launch_dim<64>(kv, q, a, p, blocks, st); break;
    case 128: launch_dim<128>(kv, q, a, p, blocks, st); break;
    case 192: launch_dim<192>(kv, q, a, p, blocks, st); break;
    default: launch_dim<256>(kv, q, a, p, blocks, st); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits <= 1) return e;
    const unsigned rows = (unsigned)((int64_t)a.nseq * kv.heads * q.new_tokens * q.group);
    kv_join_kernel<<<rows, THREADS, 0, st>>>(kv, q, a, p.row_tiles * p.rows, p.splits, plan_tile(kv.dpad));
    return hipGetLastError();
}

}  // namespace lpq
