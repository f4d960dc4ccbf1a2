// Key-value cache: codes of new keys and values into pages, with the pages' bounds, and back.
//
// A workgroup takes the rows of one page at a time for a group of key-value heads: a thread owns 8 features of one head
// (one 16-byte load of a 16-bit type, one 8-byte store of codes) of every so-many-th row of the page, so that the constants
// of its features stay in registers and the smallest and largest code of a feature need one exchange through LDS at the
// end.  The bounds of a page are those of its tokens 0 .. last written: codes that were there before are read again (at
// most page - 1 rows), so that a sequence that was cut back and goes on again has the bounds of what it holds, and the
// result does not depend on how its tokens were grouped into calls.  Bound by memory in large calls, by the round trips to
// it in small ones: a thread asks for its rows of keys, of values and for old codes before it uses any.
//
// Measured (write, read): one row of 8 heads of 128, bfloat16: 5.1, 3.6 us; 64 rows of 64 sequences 6.7, 4.2; 26 244 rows of 6 x 100
// float16 features of 12 prompts to packed codes 31.8 (vector instructions for 20 of them, 133 to a thread's 8 values, memory for 11;
// float32 rows 42) and back 22.6; 151 419 rows of 8 x 128 back to bfloat16: 188 us, 4.9 TB/s of codes and rows (a copy of memory: 4.7).
#include <type_traits>

#include "kv_internal.h"

namespace lpq {

namespace {

constexpr int KV_THREADS = 256;
constexpr int KV_ROWS = 4;      // rows a thread has in flight
// Workgroups that a large call is shared out to.  One generation of them where each writes whole pages (25 000 rows of 6 x 100
// features: 33 us; 2048 workgroups 34, 4096 35.5), more where rows are cut anywhere (155 000 rows of 8 x 128 back: 194, 193, 189).
constexpr int KV_WRITERS = 1024, KV_READERS = 4096;

// How a call is shared out: `groups` groups of `heads` heads each, `rows` rows of the call to a workgroup of each group; a
// workgroup's threads are `lanes` rows of `heads` heads of dpad / 8 threads.
struct Share {
    int heads, groups, lanes, rows;
    unsigned per_word;      // x * per_word >> 20 = x / (dpad / 4) for the words of a workgroup's heads (fewer than 2048)
};

typedef short Pair __attribute__((ext_vector_type(2)));

// What a thread needs of the constants of its 8 features.
struct Features8 {
    float k[8], m[8];
    const float *sb, *se;
    int bottom, top;
};

// For all of a wave's loads to be there, before the first of their values is used.  Left to itself the compiler waits at each use
// behind a branch, for everything that is under way by then: the stores of the row before included.
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0F70); }

__device__ __forceinline__ void load_features(const KvConstants &c, bool packed, int at, Features8 &f)
{
    kv_load_floats8(c.k + at, f.k);
    kv_load_floats8(c.m + at, f.m);
    f.sb = c.sb + at;
    f.se = c.se + at;
    const int half = 1 << (c.bits - 1), most = packed ? 7 : 127;
    f.bottom = -half;
    f.top = half < most ? half : most;
}

// floor(t) as an integer, saturated; 0 for a NaN (as the instruction has it, C++ does not say).
__device__ __forceinline__ int floor_int(float t)
{
    int q;
    asm("v_cvt_i32_f32 %0, %1" : "=v"(q) : "v"(floorf(t)));
    return q;
}

// Equation 1 for 8 values: two separately rounded operations, floor, clamp (KvConstants::clamps).  Pairs of 16 bits: features
// 2 e and 2 e + 1.
template <bool clamps>
__device__ __forceinline__ void encode8(const Raw8 &raw, int type, int left, const Features8 &f, Pair *q)
{
    float x[8];
    int c[8];
    kv_floats8(raw, type, left, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = floor_int(__fmul_rn(__fsub_rn(x[e], f.k[e]), f.m[e]));
    if (!clamps) {
        float sb[8], se[8];
        kv_load_floats8(f.sb, sb);
        kv_load_floats8(f.se, se);
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = x[e] > se[e] ? f.top : x[e] < sb[e] ? f.bottom : c[e];
    }
    const Pair lo = {(short)f.bottom, (short)f.bottom}, hi = {(short)f.top, (short)f.top};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        q[e] = __builtin_elementwise_min(__builtin_elementwise_max(__builtin_bit_cast(Pair, __builtin_amdgcn_cvt_pk_i16(c[2 * e], c[2 * e + 1])), lo), hi);
}

__device__ __forceinline__ void store_codes8(uint8_t *row, int c0, bool packed, const Pair *q)
{
    if (packed) {       // feature 2 j in the low, 2 j + 1 in the high half of byte j
        const Pair eight = {8, 8};
        uint32_t b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t u = __builtin_bit_cast(uint32_t, (Pair)(q[e] + eight));
            b[e] = u | u >> 12;
        }
        const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
        *reinterpret_cast<uint32_t *>(row + (c0 >> 1)) = lo | hi;
    } else {
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = __builtin_bit_cast(uint32_t, q[e]);
        *reinterpret_cast<uint2 *>(row + c0) = make_uint2(__builtin_amdgcn_perm(u[1], u[0], 0x06040200u), __builtin_amdgcn_perm(u[3], u[2], 0x06040200u));
    }
}

__device__ __forceinline__ uint2 load_codes8(const uint8_t *row, int c0, bool packed)
{
    if (packed) return make_uint2(*reinterpret_cast<const uint32_t *>(row + (c0 >> 1)), 0);
    return *reinterpret_cast<const uint2 *>(row + c0);
}
__device__ __forceinline__ void codes8(uint2 w, bool packed, Pair *q)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (packed) {
            q[e] = Pair{(short)((int)((w.x >> (8 * e)) & 15) - 8), (short)((int)((w.x >> (8 * e + 4)) & 15) - 8)};
        } else {
            const uint32_t x = (e < 2 ? w.x : w.y) >> (16 * (e & 1));
            q[e] = Pair{(int8_t)x, (int8_t)(x >> 8)};
        }
    }
}
// c + 1/2 of 8 codes, exactly.
__device__ __forceinline__ void middles8(uint2 w, bool packed, float *v)
{
    const uint32_t a = packed ? w.x & 0x0f0f0f0fu : w.x ^ 0x80808080u, b = packed ? (w.x >> 4) & 0x0f0f0f0fu : w.y ^ 0x80808080u;
    const float off = packed ? 7.5f : 127.5f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t from = packed ? (e & 1 ? b : a) : (e < 4 ? a : b);
        const int byte = packed ? e >> 1 : e & 3;
        v[e] = (float)((from >> (8 * byte)) & 255u) - off;
    }
}

// Rows [begin, end) of a call that belong to sequence b, the first of them at position `first`; of b = -1: to none.
struct Sequence {
    int64_t begin, end, first;
    int b;
};
// The sequence of a row, by all 64 lanes: each looks at one of 64 starts, then between two of them.  Rows ahead of the first start,
// from the last one on, or at starts that do not ascend belong to none.
__device__ __forceinline__ Sequence sequence_of(const KvPlaces &pl, int64_t row)
{
    Sequence s;
    if (!pl.starts) {
        s.b = (int)row;
        s.begin = row;
        s.end = row + 1;
    } else {
        const int lane = threadIdx.x & 63;
        int lo = 0, count = pl.nseq + 1;                 // starts lo .. lo + count - 1: the last one <= row
        while (count > 1) {
            const int step = (count + 63) / 64, at = lane * step;
            const bool below = at < count && pl.starts[lo + at] <= row;
            const int hits = __popcll(__ballot(below));
            lo += hits ? (hits - 1) * step : 0;
            if (!hits) break;                            // before the first start
            count = count - (hits - 1) * step < step ? count - (hits - 1) * step : step;
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        s.b = lo < pl.nseq ? lo : pl.nseq - 1;
        s.begin = kv_uniform(pl.starts)[s.b];
        s.end = kv_uniform(pl.starts)[s.b + 1];
        if (s.begin < 0 || s.begin > row || s.end <= row) {
            // to the first start or to the end, else one at a time
            s.end = s.begin > row ? s.begin : s.begin >= 0 && lo == pl.nseq ? pl.n : row + 1;
            s.begin = row;
            s.b = -1;
        }
        if (s.end > pl.n) s.end = pl.n;
    }
    s.first = s.b < 0 ? 0 : kv_uniform(pl.first)[s.b];
    return s;
}
// Page of the pool that holds positions column * page on of sequence b; -1: there is none.
__device__ __forceinline__ int64_t page_of(const KvView &kv, const KvPlaces &pl, int b, int64_t column)
{
    if (column < 0 || column >= pl.table_pages) return -1;
    const int32_t t = kv_uniform(pl.table + (int64_t)b * pl.ld_table)[column];
    return t >= 0 && t < kv.pages ? t : -1;
}

// What a thread has of a workgroup's rows: features c0 .. c0 + 7 of head h, rows lane, lane + lanes, ... of a page, of the keys
// (which = 0) or of the values.  [begin, end): the workgroup's rows of the call.
struct Seat {
    int64_t begin, end;
    int which, h0, h, c0, lane;
    bool on;
};
__device__ __forceinline__ Seat seat(const KvView &kv, const KvPlaces &pl, const Share &sh)
{
    Seat s;
    const int chunks = kv.dpad >> 3, slot = threadIdx.x / chunks;
    s.which = blockIdx.x & 1;
    const int work = blockIdx.x >> 1, part = __builtin_amdgcn_readfirstlane(work / sh.groups);
    s.begin = (int64_t)part * sh.rows;
    s.end = s.begin + sh.rows < pl.n ? s.begin + sh.rows : pl.n;
    s.h0 = (work - part * sh.groups) * sh.heads;
    s.c0 = 8 * (threadIdx.x - slot * chunks);
    s.lane = slot / sh.heads;
    s.h = s.h0 + slot - s.lane * sh.heads;
    s.on = s.lane < sh.lanes && s.h < kv.heads;
    return s;
}

template <int type, bool packed, bool clamps>
__global__ __launch_bounds__(KV_THREADS, 4) void kv_write_kernel(KvView kv, KvRows kr, KvRows vr, KvPlaces pl, Share sh)
{
    __shared__ uint2 part_lo[KV_THREADS], part_hi[KV_THREADS];
    const Seat s = seat(kv, pl, sh);
    const KvRows in = s.which ? vr : kr;
    const int row_bytes = (packed ? kv.dpad >> 1 : kv.dpad), left = kv.dim - s.c0;
    Features8 f;
    if (s.on) load_features(s.which ? kv.value : kv.key, packed, s.h * kv.dpad + s.c0, f);
    Sequence q;
    q.end = -1;
    // A workgroup takes the pages whose first row of the call is among its rows.
    for (int64_t row = s.begin, end; row < s.end; row = end) {
        if (row >= q.end) q = sequence_of(pl, row);
        const int64_t at = q.first + (row - q.begin), column = at >> kv.page_shift;
        const int inside = (int)(at & (kv.page - 1));
        end = row + kv.page - inside < q.end ? row + kv.page - inside : q.end;
        if (inside > 0 && row > q.begin) continue;                         // begun by the workgroup before
        const int64_t page = q.b < 0 ? -1 : page_of(kv, pl, q.b, column);   // none at positions below 0
        if (page < 0) continue;                                            // (all of this uniform over the workgroup)
        const int lo_row = inside, hi_row = inside + (int)(end - row);     // rows of the page
        Pair mn[4], mx[4];           // of features 2 e and 2 e + 1
#pragma unroll
        for (int e = 0; e < 4; ++e) { mn[e] = Pair{127, 127}; mx[e] = Pair{-128, -128}; }
        auto widen = [&](const Pair *c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mn[e] = __builtin_elementwise_min(mn[e], c[e]);
                mx[e] = __builtin_elementwise_max(mx[e], c[e]);
            }
        };
        if (s.on) {
            uint8_t *rows = (s.which ? kv.v : kv.k) + (page * kv.heads + s.h) * kv.page * row_bytes;
            const int64_t from = (row - lo_row) * in.ld_token + s.h * in.ld_head + s.c0;
            auto encode = [&](const Raw8 &x, int t) {
                Pair c[4];
                encode8<clamps>(x, type, left, f, c);
                store_codes8(rows + t * row_bytes, s.c0, packed, c);
                if (s.which == 0) widen(c);
            };
            for (int t0 = lo_row + s.lane; t0 < hi_row; t0 += KV_ROWS * sh.lanes) {
                Raw8 x[KV_ROWS];
#pragma unroll
                for (int u = 0; u < KV_ROWS; ++u)
                    if (t0 + u * sh.lanes < hi_row) x[u] = kv_load8(in.p, type, from + (t0 + u * sh.lanes) * in.ld_token, left);
                loads_done();
#pragma unroll
                for (int u = 0; u < KV_ROWS; ++u) {
                    if (t0 + u * sh.lanes < hi_row) encode(x[u], t0 + u * sh.lanes);
                    __builtin_amdgcn_sched_barrier(0);       // one row after the other: four at once do not fit the registers
                }
            }
            if (s.which == 0) {
                for (int t1 = s.lane; t1 < lo_row; t1 += 2 * KV_ROWS * sh.lanes) {
                    uint2 w[2 * KV_ROWS];
#pragma unroll
                    for (int u = 0; u < 2 * KV_ROWS; ++u) {
                        const int t = t1 + u * sh.lanes < lo_row ? t1 + u * sh.lanes : t1;    // a row twice does not move the bounds
                        w[u] = load_codes8(rows + t * row_bytes, s.c0, packed);
                    }
#pragma unroll
                    for (int u = 0; u < 2 * KV_ROWS; ++u) {
                        Pair c[4];
                        codes8(w[u], packed, c);
                        widen(c);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
        if (s.which) continue;
        uint2 lo = {0, 0}, hi = {0, 0};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            lo.x |= (uint32_t)(mn[e].x & 255) << (16 * e) | (uint32_t)(mn[e].y & 255) << (16 * e + 8);
            lo.y |= (uint32_t)(mn[e + 2].x & 255) << (16 * e) | (uint32_t)(mn[e + 2].y & 255) << (16 * e + 8);
            hi.x |= (uint32_t)(mx[e].x & 255) << (16 * e) | (uint32_t)(mx[e].y & 255) << (16 * e + 8);
            hi.y |= (uint32_t)(mx[e + 2].x & 255) << (16 * e) | (uint32_t)(mx[e + 2].y & 255) << (16 * e + 8);
        }
        part_lo[threadIdx.x] = lo;
        part_hi[threadIdx.x] = hi;
        __syncthreads();
        {   // word t of the group's heads' lower bounds, then of the upper ones: [lane][head][feature] -> [head][2][feature]
            const int some = sh.heads < kv.heads - s.h0 ? sh.heads : kv.heads - s.h0, words = kv.dpad >> 2, stride = sh.heads * words;
            uint32_t *out = reinterpret_cast<uint32_t *>(kv.bounds + (page * kv.heads + s.h0) * 2 * kv.dpad);
            for (int t = threadIdx.x; t < 2 * some * words; t += KV_THREADS) {
                const bool upper = t >= some * words;
                const int at = upper ? t - some * words : t, head = (int)((unsigned)at * sh.per_word >> 20);
                const uint32_t *src = reinterpret_cast<const uint32_t *>(upper ? part_hi : part_lo) + at;
                Pair even, odd;          // features 0 and 2, 1 and 3 of the word, sign in the high bytes
                for (int u = 0; u < sh.lanes; ++u) {
                    const uint32_t w = src[u * stride];
                    const Pair a = __builtin_bit_cast(Pair, w << 8 & 0xff00ff00u), b = __builtin_bit_cast(Pair, w & 0xff00ff00u);
                    even = u == 0 ? a : upper ? __builtin_elementwise_max(even, a) : __builtin_elementwise_min(even, a);
                    odd = u == 0 ? b : upper ? __builtin_elementwise_max(odd, b) : __builtin_elementwise_min(odd, b);
                }
                out[(2 * head + (upper ? 1 : 0)) * words + at - head * words] = __builtin_bit_cast(uint32_t, even) >> 8 | __builtin_bit_cast(uint32_t, odd);
            }
        }
        __syncthreads();                                    // the partial bounds are used again by the next page
    }
}

// x^ = k + (c + 1/2) s, each operation rounded to binary32; rows without a page or a sequence are zeros.
template <int type, bool packed>
__global__ __launch_bounds__(KV_THREADS, 4) void kv_read_kernel(KvView kv, KvRows kr, KvRows vr, KvPlaces pl, Share sh)
{
    const Seat s = seat(kv, pl, sh);
    const KvRows out = s.which ? vr : kr;
    const int row_bytes = (packed ? kv.dpad >> 1 : kv.dpad), left = s.on ? kv.dim - s.c0 : 0;
    float k[8], step[8];
    if (left > 0) {
        const int at = s.h * kv.dpad + s.c0;
        kv_load_floats8((s.which ? kv.value.k : kv.key.k) + at, k);
        kv_load_floats8((s.which ? kv.value.s : kv.key.s) + at, step);
    }
    Sequence q;
    q.end = -1;
    for (int64_t row = s.begin, end; row < s.end; row = end) {
        if (row >= q.end) q = sequence_of(pl, row);
        const int64_t at = q.first + (row - q.begin), column = at >> kv.page_shift;
        const int inside = (int)(at & (kv.page - 1));
        end = row + kv.page - inside < q.end ? row + kv.page - inside : q.end;
        if (end > s.end) end = s.end;
        if (left <= 0) continue;
        const int64_t page = q.b < 0 ? -1 : page_of(kv, pl, q.b, column);
        const uint8_t *rows = (s.which ? kv.v : kv.k) + (page * kv.heads + s.h) * kv.page * row_bytes;
        const int hi_row = inside + (int)(end - row);
        for (int t0 = inside + s.lane; t0 < hi_row; t0 += 2 * KV_ROWS * sh.lanes) {
            uint2 w[2 * KV_ROWS];
#pragma unroll
            for (int u = 0; u < 2 * KV_ROWS; ++u) {
                const int t = t0 + u * sh.lanes;
                if (t < hi_row && page >= 0) w[u] = load_codes8(rows + t * row_bytes, s.c0, packed);
            }
            loads_done();
#pragma unroll
            for (int u = 0; u < 2 * KV_ROWS; ++u) {
                const int t = t0 + u * sh.lanes;
                if (t >= hi_row) continue;
                float x[8];
                middles8(w[u], packed, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __fadd_rn(__fmul_rn(x[e], step[e]), k[e]);
                if (page < 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = 0.0f;
                }
                kv_store<8>(out.p, type, (row - inside + t) * out.ld_token + s.h * out.ld_head + s.c0, left, x);
            }
        }
    }
}

__global__ void kv_constants_kernel(QuantParams q, int heads, int dim, int dpad, bool packed, float *out, int *not_all)
{
    const int t = blockIdx.x * blockDim.x + threadIdx.x, total = heads * dpad;
    if (t >= total) return;
    const int h = t / dpad, i = t % dpad, f = h * dim + i;
    float k = 0.f, sb = -INFINITY, se = INFINITY, m = 0.f;
    if (i < dim) {
        k = q.k[f];
        if (q.se[f] > q.sb[f]) {
            sb = q.sb[f];
            se = q.se[f];
            m = q.m[f];
        }
    }
    out[t] = k;
    out[total + t] = sb;
    out[2 * total + t] = se;
    out[3 * total + t] = m;
    out[4 * total + t] = m > 0.f ? 1.0f / m : 0.f;
    // Rounding is monotone, so every x > S_e has a product no smaller than that of S_e: where that already rounds down to the
    // top code or above, the clamp gives what the comparison with S_e would; likewise below S_b.
    const int half = 1 << (q.bits - 1), most = packed ? 7 : 127;
    const bool clamps = !(se < INFINITY) || (floorf(__fmul_rn(__fsub_rn(se, k), m)) >= (float)(half < most ? half : most) &&
                                             floorf(__fmul_rn(__fsub_rn(sb, k), m)) <= (float)-half);
    if (!clamps) *not_all = 1;
}

// Rows in equal numbers to about as many workgroups as the chip holds at once, whole pages of them to one (a write); neighbouring
// heads share a workgroup where that leaves enough of them, since their rows lie side by side outside the cache.
Share share_of(const KvView &kv, const KvPlaces &pl, bool write)
{
    Share s;
    const int slots = KV_THREADS / (kv.dpad / 8), workgroups = write ? KV_WRITERS : KV_READERS;
    const int64_t units = pl.starts ? ceil_div(pl.n, (int64_t)kv.page) + pl.nseq : pl.n;      // pages, about: sequences begin and end inside them
    s.heads = 1;
    for (int h = 2; h <= kv.heads && h <= slots; ++h)
        if (slots / h * h * 8 >= slots * 7 && kv.heads % h == 0 && 2 * units * (kv.heads / h) >= workgroups) s.heads = h;
    s.lanes = slots / s.heads;
    s.groups = (int)ceil_div(kv.heads, s.heads);
    int64_t rows = pl.starts ? ceil_div(pl.n * 2 * s.groups, (int64_t)workgroups) : 1;
    // No fewer than a thread has in flight (a write: than a page has) where that makes workgroups enough to fill the chip, else down to what an
    // average page has in this call: the pages of one workgroup follow each other.  9 sequences of 6 rows of 3 x 64: write 33.7 us in 6
    // workgroups, 6.3 in 54; back 12.3, 3.9.
    const int64_t most = write ? kv.page : s.lanes * 2 * KV_ROWS, grid = KV_MAX_BLOCKS / s.groups;
    int64_t few = pl.starts ? ceil_div(pl.n * 2 * s.groups, (int64_t)KV_WRITERS) : 1;
    if (pl.starts && few < ceil_div(pl.n, units)) few = ceil_div(pl.n, units);
    if (few > most) few = most;
    if (rows < few) rows = few;
    if (rows < ceil_div(pl.n, grid)) rows = ceil_div(pl.n, grid);
    s.rows = (int)rows;
    s.per_word = ((1u << 20) + kv.dpad / 4 - 1) / (kv.dpad / 4);
    return s;
}

}  // namespace

hipError_t launch_kv_constants(const QuantParams &q, int heads, int dim, int dpad, bool packed, float *out, int *not_all, hipStream_t st)
{
    kv_constants_kernel<<<(unsigned)ceil_div(heads * dpad, 256), 256, 0, st>>>(q, heads, dim, dpad, packed, out, not_all);
    return hipGetLastError();
}

hipError_t launch_kv_write(const KvView &kv, const KvRows &k, const KvRows &v, const KvPlaces &pl, hipStream_t st)
{
    if (pl.n <= 0 || pl.nseq <= 0) return hipSuccess;
    const Share s = share_of(kv, pl, true);
    const unsigned blocks = (unsigned)(2 * ceil_div(pl.n, (int64_t)s.rows) * s.groups);
    auto launch_as = [&](auto type, auto packed, auto clamps) {
        kv_write_kernel<decltype(type)::value, decltype(packed)::value, decltype(clamps)::value><<<blocks, KV_THREADS, 0, st>>>(kv, k, v, pl, s);
    };
    auto launch = [&](auto type) {
        const bool clamps = kv.key.clamps && kv.value.clamps;
        if (kv.packed && clamps) launch_as(type, std::true_type(), std::true_type());
        else if (kv.packed) launch_as(type, std::true_type(), std::false_type());
        else if (clamps) launch_as(type, std::false_type(), std::true_type());
        else launch_as(type, std::false_type(), std::false_type());
    };
    if (k.type == LPQ_TYPE_F32) launch(std::integral_constant<int, LPQ_TYPE_F32>());
    else if (k.type == LPQ_TYPE_F16) launch(std::integral_constant<int, LPQ_TYPE_F16>());
    else launch(std::integral_constant<int, LPQ_TYPE_BF16>());
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvView &kv, const KvRows &k, const KvRows &v, const KvPlaces &pl, hipStream_t st)
{
    if (pl.n <= 0 || pl.nseq <= 0) return hipSuccess;
    const Share s = share_of(kv, pl, false);
    const unsigned blocks = (unsigned)(2 * ceil_div(pl.n, (int64_t)s.rows) * s.groups);
    auto launch = [&](auto type) {
        if (kv.packed) kv_read_kernel<decltype(type)::value, true><<<blocks, KV_THREADS, 0, st>>>(kv, k, v, pl, s);
        else kv_read_kernel<decltype(type)::value, false><<<blocks, KV_THREADS, 0, st>>>(kv, k, v, pl, s);
    };
    if (k.type == LPQ_TYPE_F32) launch(std::integral_constant<int, LPQ_TYPE_F32>());
    else if (k.type == LPQ_TYPE_F16) launch(std::integral_constant<int, LPQ_TYPE_F16>());
    else launch(std::integral_constant<int, LPQ_TYPE_BF16>());
    return hipGetLastError();
}

}  // namespace lpq
