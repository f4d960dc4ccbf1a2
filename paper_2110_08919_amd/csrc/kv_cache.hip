// Key-value cache: codes of new keys and values into pages, with the pages' bounds, and back.
//
// A workgroup takes the rows of one page at a time for a group of key-value heads: a thread owns 8 features of one head
// (one 16-byte load of a 16-bit type, one 8-byte store of codes) of every so-many-th row of the page, so that the constants
// of its features stay in registers and the smallest and largest code of a feature need one exchange through LDS at the
// end.  The bounds of a page are those of its tokens 0 .. last written: codes that were there before are read again (at
// most page - 1 rows), so that a sequence that was cut back and goes on again has the bounds of what it holds, and the
// result does not depend on how its tokens were grouped into calls.  Bound by memory in large calls, by the round trips to
// it in small ones: a thread asks for its rows of keys, of values and for old codes before it uses any.
#include <type_traits>

#include "kv_internal.h"

namespace lpq {

namespace {

constexpr int KV_THREADS = 256;
constexpr int KV_ROWS = 4;      // rows a thread has in flight
constexpr int KV_WORKGROUPS = 2048;

// How a call is shared out: `groups` groups of `heads` heads each, `pieces` workgroups per sequence and group that take its
// pages in turn; a workgroup's threads are `lanes` rows of `heads` heads of dpad / 8 threads.
struct Share {
    int heads, groups, lanes, pieces;
};

// Equation 1 for one value: two separately rounded operations, floor, clamp (NaN -> 0).
__device__ __forceinline__ int kv_quantize(float x, float k, float sb, float se, float m, float lo, float top)
{
    const float t = __fmul_rn(__fsub_rn(x, k), m);
    float f = __builtin_amdgcn_fmed3f(floorf(t), lo, top);
    f = (x > se) ? top : f;
    f = (x < sb) ? lo : f;
    f = (t != t) ? 0.0f : f;
    return (int)f;
}

typedef short Pair __attribute__((ext_vector_type(2)));

struct Features8 {
    float k[8], sb[8], se[8], m[8], bottom, top;
};

__device__ __forceinline__ void load_features(const KvConstants &c, bool packed, int at, Features8 &f)
{
    kv_load_floats8(c.k + at, f.k);
    kv_load_floats8(c.sb + at, f.sb);
    kv_load_floats8(c.se + at, f.se);
    kv_load_floats8(c.m + at, f.m);
    const int half = 1 << (c.bits - 1), most = packed ? 7 : 127;
    f.bottom = (float)-half;
    f.top = (float)(half < most ? half : most);
}

__device__ __forceinline__ void encode8(const Raw8 &raw, int type, const Features8 &f, int *q)
{
    float x[8];
    kv_floats8(raw, type, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = kv_quantize(x[e], f.k[e], f.sb[e], f.se[e], f.m[e], f.bottom, f.top);
}

__device__ __forceinline__ void store_codes8(uint8_t *row, int c0, bool packed, const int *q)
{
    if (packed) {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w |= (uint32_t)(q[e] + 8) << (4 * e);   // feature 2j low, 2j + 1 high half of byte j
        *reinterpret_cast<uint32_t *>(row + (c0 >> 1)) = w;
    } else {
        uint2 w = {0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w.x |= (uint32_t)(q[e] & 255) << (8 * e);
            w.y |= (uint32_t)(q[e + 4] & 255) << (8 * e);
        }
        *reinterpret_cast<uint2 *>(row + c0) = w;
    }
}

__device__ __forceinline__ uint2 load_codes8(const uint8_t *row, int c0, bool packed)
{
    if (packed) return make_uint2(*reinterpret_cast<const uint32_t *>(row + (c0 >> 1)), 0);
    return *reinterpret_cast<const uint2 *>(row + c0);
}
__device__ __forceinline__ void codes8(uint2 w, bool packed, int *q)
{
    if (packed) {
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = (int)((w.x >> (4 * e)) & 15) - 8;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            q[e] = (int8_t)(w.x >> (8 * e));
            q[e + 4] = (int8_t)(w.y >> (8 * e));
        }
    }
}

// Rows [row0, row0 + count) of a call that belong to sequence b.
__device__ __forceinline__ void rows_of(const KvPlaces &pl, int b, int64_t &row0, int64_t &count)
{
    if (!pl.starts) {
        row0 = b;
        count = 1;
        return;
    }
    int64_t r0 = kv_uniform(pl.starts)[b], r1 = kv_uniform(pl.starts)[b + 1];
    r0 = r0 < 0 ? 0 : (r0 > pl.n ? pl.n : r0);
    r1 = r1 < r0 ? r0 : (r1 > pl.n ? pl.n : r1);
    row0 = r0;
    count = r1 - r0;
}

// One step of a workgroup: the part of a page that a call covers.
struct PagePart {
    int lo, hi;        // rows of the page [lo, hi)
    int64_t source;    // row of the call that is row `lo`
    int64_t page;      // of the pool; -1: there is none
};

__device__ __forceinline__ PagePart page_part(const KvView &kv, const KvPlaces &pl, int b, int64_t first, int64_t row0, int64_t count,
                                              int64_t column)
{
    PagePart p;
    const int64_t at = column << kv.page_shift;
    const int64_t from = first < at ? at : first, to = first + count < at + kv.page ? first + count : at + kv.page;
    p.lo = (int)(from - at);
    p.hi = (int)(to - at);
    p.source = row0 + (from - first);
    p.page = -1;
    if (column >= 0 && column < pl.table_pages) {
        const int32_t t = kv_uniform(pl.table + (int64_t)b * pl.ld_table)[column];
        if (t >= 0 && t < kv.pages) p.page = t;
    }
    return p;
}

// What a thread has of a workgroup's page: features c0 .. c0 + 7 of head h, rows lane, lane + lanes, ... of its keys (which = 0)
// or values.
struct Seat {
    int which, b, piece, h0, h, c0, lane;
    bool on;
};
__device__ __forceinline__ Seat seat(const KvView &kv, const Share &sh)
{
    Seat s;
    const int chunks = kv.dpad >> 3, slot = threadIdx.x / chunks;
    s.which = blockIdx.x & 1;
    const int work = blockIdx.x >> 1, per = __builtin_amdgcn_readfirstlane(work / sh.groups);
    s.b = __builtin_amdgcn_readfirstlane(per / sh.pieces);
    s.piece = per - s.b * sh.pieces;
    s.h0 = (work - per * sh.groups) * sh.heads;
    s.c0 = 8 * (threadIdx.x - slot * chunks);
    s.lane = slot / sh.heads;
    s.h = s.h0 + slot - s.lane * sh.heads;
    s.on = s.lane < sh.lanes && s.h < kv.heads;
    return s;
}

template <int type, bool packed>
__global__ __launch_bounds__(KV_THREADS, 4) void kv_write_kernel(KvView kv, KvRows kr, KvRows vr, KvPlaces pl, Share sh)
{
    __shared__ uint2 part_lo[KV_THREADS], part_hi[KV_THREADS];
    const Seat s = seat(kv, sh);
    const KvRows in = s.which ? vr : kr;
    const int row_bytes = (packed ? kv.dpad >> 1 : kv.dpad);
    int64_t row0, count, first = kv_uniform(pl.first)[s.b];
    rows_of(pl, s.b, row0, count);
    if (first < 0) {               // rows at negative positions have no place
        const int64_t skip = count < -first ? count : -first;
        row0 += skip;
        count -= skip;
        first = 0;
    }
    if (count <= 0) return;
    const int64_t column0 = first >> kv.page_shift, columns = ((first + count - 1) >> kv.page_shift) - column0 + 1;
    if (s.piece >= columns) return;
    Features8 f;
    if (s.on) load_features(s.which ? kv.value : kv.key, packed, s.h * kv.dpad + s.c0, f);
    for (int64_t i = s.piece; i < columns; i += sh.pieces) {
        const PagePart p = page_part(kv, pl, s.b, first, row0, count, column0 + i);
        if (p.page < 0) continue;      // uniform over the workgroup
        Pair mn[4], mx[4];           // of features 2 e and 2 e + 1
#pragma unroll
        for (int e = 0; e < 4; ++e) { mn[e] = Pair{127, 127}; mx[e] = Pair{-128, -128}; }
        auto widen = [&](const int *q) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const Pair x = {(short)q[2 * e], (short)q[2 * e + 1]};
                mn[e] = __builtin_elementwise_min(mn[e], x);
                mx[e] = __builtin_elementwise_max(mx[e], x);
            }
        };
        if (s.on) {
            uint8_t *rows = (s.which ? kv.v : kv.k) + (p.page * kv.heads + s.h) * kv.page * row_bytes;
            const int64_t from = (p.source - p.lo) * in.ld_token + s.h * in.ld_head;
            auto encode = [&](const Raw8 &x, int t) {
                int q[8];
                encode8(x, type, f, q);
                store_codes8(rows + t * row_bytes, s.c0, packed, q);
                widen(q);
            };
            int t0 = p.lo + s.lane;
            for (; t0 + (KV_ROWS - 1) * sh.lanes < p.hi; t0 += KV_ROWS * sh.lanes) {
                Raw8 x[KV_ROWS];
#pragma unroll
                for (int u = 0; u < KV_ROWS; ++u) x[u] = kv_load8_raw(in.p, type, from + (t0 + u * sh.lanes) * in.ld_token, s.c0, kv.dim);
#pragma unroll
                for (int u = 0; u < KV_ROWS; ++u) {
                    encode(x[u], t0 + u * sh.lanes);
                    __builtin_amdgcn_sched_barrier(0);       // one row after the other: four at once do not fit the registers
                }
            }
            for (; t0 < p.hi; t0 += sh.lanes) encode(kv_load8_raw(in.p, type, from + t0 * in.ld_token, s.c0, kv.dim), t0);
            if (s.which == 0) {
                for (int t1 = s.lane; t1 < p.lo; t1 += 2 * KV_ROWS * sh.lanes) {
                    uint2 w[2 * KV_ROWS];
#pragma unroll
                    for (int u = 0; u < 2 * KV_ROWS; ++u) {
                        const int t = t1 + u * sh.lanes < p.lo ? t1 + u * sh.lanes : t1;    // a row twice does not move the bounds
                        w[u] = load_codes8(rows + t * row_bytes, s.c0, packed);
                    }
#pragma unroll
                    for (int u = 0; u < 2 * KV_ROWS; ++u) {
                        int q[8];
                        codes8(w[u], packed, q);
                        widen(q);
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
        {   // byte t of the group's heads' lower bounds, then of the upper ones: [lane][head][feature] -> [head][2][feature]
            const int8_t *low = reinterpret_cast<const int8_t *>(part_lo), *high = reinterpret_cast<const int8_t *>(part_hi);
            const int some = sh.heads < kv.heads - s.h0 ? sh.heads : kv.heads - s.h0, stride = sh.heads * kv.dpad;
            int8_t *out = kv.bounds + (p.page * kv.heads + s.h0) * 2 * kv.dpad;
            for (int t = threadIdx.x; t < 2 * some * kv.dpad; t += KV_THREADS) {
                const bool upper = t >= some * kv.dpad;
                const int at = upper ? t - some * kv.dpad : t;
                const int8_t *src = (upper ? high : low) + at;
                int best = src[0];
                for (int u = 1; u < sh.lanes; ++u) {
                    const int q = src[u * stride];
                    best = upper ? (q > best ? q : best) : (q < best ? q : best);
                }
                const int head = at / kv.dpad;
                out[(2 * head + (upper ? 1 : 0)) * kv.dpad + at - head * kv.dpad] = (int8_t)best;
            }
        }
        if (i + sh.pieces < columns) __syncthreads();       // the partial bounds are used again by the next page
    }
}

// x^ = k + (c + 1/2) s, each operation rounded to binary32; rows without a page are zeros.
template <int type, bool packed>
__global__ __launch_bounds__(KV_THREADS, 4) void kv_read_kernel(KvView kv, KvRows kr, KvRows vr, KvPlaces pl, Share sh)
{
    const Seat s = seat(kv, sh);
    const KvRows out = s.which ? vr : kr;
    const int row_bytes = (packed ? kv.dpad >> 1 : kv.dpad), left = kv.dim - s.c0;
    if (!s.on || left <= 0) return;
    int64_t row0, count;
    const int64_t first = kv_uniform(pl.first)[s.b];
    rows_of(pl, s.b, row0, count);
    if (count <= 0) return;
    const int64_t column0 = first >> kv.page_shift, columns = ((first + count - 1) >> kv.page_shift) - column0 + 1;
    if (s.piece >= columns) return;
    float k[8], step[8];
    const int at = s.h * kv.dpad + s.c0;
    kv_load_floats8((s.which ? kv.value.k : kv.key.k) + at, k);
    kv_load_floats8((s.which ? kv.value.s : kv.key.s) + at, step);
    for (int64_t i = s.piece; i < columns; i += sh.pieces) {
        const PagePart p = page_part(kv, pl, s.b, first, row0, count, column0 + i);
        const uint8_t *rows = (s.which ? kv.v : kv.k) + (p.page * kv.heads + s.h) * kv.page * row_bytes;
        for (int t0 = p.lo + s.lane; t0 < p.hi; t0 += 2 * KV_ROWS * sh.lanes) {
            uint2 w[2 * KV_ROWS];
#pragma unroll
            for (int u = 0; u < 2 * KV_ROWS; ++u) {
                const int t = t0 + u * sh.lanes;
                if (t < p.hi && p.page >= 0) w[u] = load_codes8(rows + t * row_bytes, s.c0, packed);
            }
#pragma unroll
            for (int u = 0; u < 2 * KV_ROWS; ++u) {
                const int t = t0 + u * sh.lanes;
                if (t >= p.hi) continue;
                int q[8];
                float x[8];
                codes8(w[u], packed, q);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = p.page >= 0 ? __fadd_rn(__fmul_rn((float)q[e] + 0.5f, step[e]), k[e]) : 0.0f;
                kv_store<8>(out.p, type, (p.source + t - p.lo) * out.ld_token + s.h * out.ld_head + s.c0, left, x);
            }
        }
    }
}

__global__ void kv_constants_kernel(QuantParams q, int heads, int dim, int dpad, float *out)
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
}

// A decoding step has one page per sequence; a prompt has as many as its share of the rows fills, and a longer one than the
// others takes more turns of the same workgroups.  Neighbouring heads share a workgroup where that leaves enough of them
// (rows of neighbouring heads lie side by side outside the cache).
Share share_of(const KvView &kv, const KvPlaces &pl)
{
    Share s;
    const int slots = KV_THREADS / (kv.dpad / 8);
    const int64_t mean = ceil_div(pl.n, (int64_t)pl.nseq), most = ceil_div(pl.n, (int64_t)kv.page) + 1;
    const int64_t pages = pl.n == pl.nseq ? pl.nseq : ceil_div(mean, (int64_t)kv.page) * pl.nseq;
    s.heads = 1;
    for (int h = 2; h <= kv.heads && h <= slots; ++h)
        if (slots / h * h * 8 >= slots * 7 && kv.heads % h == 0 && pages * (kv.heads / h) >= KV_WORKGROUPS) s.heads = h;
    s.lanes = slots / s.heads;
    s.groups = (int)ceil_div(kv.heads, s.heads);
    int64_t pieces = pl.n == pl.nseq ? 1 : 2 * ceil_div(mean, (int64_t)kv.page) + 1;
    const int64_t room = ceil_div(int64_t(4096), (int64_t)pl.nseq * s.groups);     // up to 16 workgroups per CU in any case
    if (pl.n != pl.nseq && pieces < room) pieces = room;
    const int64_t grid = KV_MAX_BLOCKS / ((int64_t)pl.nseq * s.groups);            // >= 1 (the entry points); keys and values twice as many
    if (pieces > grid) pieces = grid;
    s.pieces = (int)(pieces < most ? pieces : most);
    return s;
}

}  // namespace

hipError_t launch_kv_constants(const QuantParams &q, int heads, int dim, int dpad, float *out, hipStream_t st)
{
    kv_constants_kernel<<<(unsigned)ceil_div(heads * dpad, 256), 256, 0, st>>>(q, heads, dim, dpad, out);
    return hipGetLastError();
}

hipError_t launch_kv_write(const KvView &kv, const KvRows &k, const KvRows &v, const KvPlaces &pl, hipStream_t st)
{
    if (pl.n <= 0 || pl.nseq <= 0) return hipSuccess;
    const Share s = share_of(kv, pl);
    const unsigned blocks = (unsigned)(2 * (int64_t)s.pieces * pl.nseq * s.groups);
    auto launch = [&](auto type) {
        if (kv.packed) kv_write_kernel<decltype(type)::value, true><<<blocks, KV_THREADS, 0, st>>>(kv, k, v, pl, s);
        else kv_write_kernel<decltype(type)::value, false><<<blocks, KV_THREADS, 0, st>>>(kv, k, v, pl, s);
    };
    if (k.type == LPQ_TYPE_F32) launch(std::integral_constant<int, LPQ_TYPE_F32>());
    else if (k.type == LPQ_TYPE_F16) launch(std::integral_constant<int, LPQ_TYPE_F16>());
    else launch(std::integral_constant<int, LPQ_TYPE_BF16>());
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvView &kv, const KvRows &k, const KvRows &v, const KvPlaces &pl, hipStream_t st)
{
    if (pl.n <= 0 || pl.nseq <= 0) return hipSuccess;
    const Share s = share_of(kv, pl);
    const unsigned blocks = (unsigned)(2 * (int64_t)s.pieces * pl.nseq * s.groups);
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
