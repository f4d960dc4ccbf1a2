// Key-value cache: codes of new keys and values into pages, with the pages' bounds, and back.
//
// A workgroup takes the rows of one page of one key-value head: a thread owns 8 features (one 16-byte load of a 16-bit
// type, one 8-byte store of codes) of every so-many-th row of the page, so that the constants of its features stay in
// registers and the smallest and largest code of a feature need one exchange through LDS at the end.  The bounds of a
// page are those of its tokens 0 .. last written: codes that were there before are read again (at most page - 1 rows),
// so that a sequence that was cut back and goes on again has the bounds of what it holds, and the result does not
// depend on how its tokens were grouped into calls.  Bound by memory in large calls, by latency in small ones.
#include "kv_internal.h"

namespace lpq {

namespace {

constexpr int KV_THREADS = 256;
constexpr int KV_ROWS = 4;      // rows a thread has in flight

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

struct Features8 {
    float k[8], sb[8], se[8], m[8];
};

__device__ __forceinline__ void load_floats8(const float *p, float *v)
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
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

__device__ __forceinline__ void load_codes8(const uint8_t *row, int c0, bool packed, int *q)
{
    if (packed) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(row + (c0 >> 1));
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = (int)((w >> (4 * e)) & 15) - 8;
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(row + c0);
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
    int64_t r0 = pl.starts[b], r1 = pl.starts[b + 1];
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
        const int32_t t = pl.table[(int64_t)b * pl.ld_table + column];
        if (t >= 0 && t < kv.pages) p.page = t;
    }
    return p;
}

__global__ __launch_bounds__(KV_THREADS) void kv_write_kernel(KvView kv, KvRows kr, KvRows vr, KvPlaces pl, int pieces)
{
    __shared__ uint2 part_lo[KV_THREADS], part_hi[KV_THREADS];
    const int h = blockIdx.x % kv.heads, b = (blockIdx.x / kv.heads) % pl.nseq, piece = blockIdx.x / kv.heads / pl.nseq;
    const int chunks = kv.dpad >> 3, lanes = KV_THREADS / chunks, c = threadIdx.x % chunks, r = threadIdx.x / chunks, c0 = 8 * c;
    const int row_bytes = kv.row_bytes(), left = kv.dim - c0;
    const bool on = r < lanes;
    int64_t row0, count, first = pl.first[b];
    rows_of(pl, b, row0, count);
    if (first < 0) {               // rows at negative positions have no place
        const int64_t skip = count < -first ? count : -first;
        row0 += skip;
        count -= skip;
        first = 0;
    }
    if (count <= 0) return;
    const int64_t column0 = first >> kv.page_shift, columns = ((first + count - 1) >> kv.page_shift) - column0 + 1;
    if (piece >= columns) return;
    for (int64_t i = piece; i < columns; i += pieces) {
        const PagePart p = page_part(kv, pl, b, first, row0, count, column0 + i);
        if (p.page < 0) continue;      // uniform over the workgroup
        const int64_t block = (p.page * kv.heads + h) * kv.page * row_bytes;
        Features8 f;
        if (on) {
            const int at = h * kv.dpad + c0;
            load_floats8(kv.key.k + at, f.k);
            load_floats8(kv.key.sb + at, f.sb);
            load_floats8(kv.key.se + at, f.se);
            load_floats8(kv.key.m + at, f.m);
            const int half = 1 << (kv.key.bits - 1), most = kv.packed ? 7 : 127;
            const float bottom = (float)-half, top = (float)(half < most ? half : most);
            int mn[8], mx[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) { mn[e] = 127; mx[e] = -128; }
            auto widen = [&](const int *q) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    mn[e] = q[e] < mn[e] ? q[e] : mn[e];
                    mx[e] = q[e] > mx[e] ? q[e] : mx[e];
                }
            };
            for (int t0 = r; t0 < p.lo; t0 += KV_ROWS * lanes) {
#pragma unroll
                for (int u = 0; u < KV_ROWS; ++u) {
                    const int t = t0 + u * lanes < p.lo ? t0 + u * lanes : t0;    // a row twice does not move the bounds
                    int q[8];
                    load_codes8(kv.k + block + (int64_t)t * row_bytes, c0, kv.packed, q);
                    widen(q);
                }
            }
            for (int t0 = p.lo + r; t0 < p.hi; t0 += KV_ROWS * lanes) {
                float x[KV_ROWS][8];
#pragma unroll
                for (int u = 0; u < KV_ROWS; ++u) {
                    const int t = t0 + u * lanes;
                    if (t < p.hi) kv_load8(kr.p, kr.type, (p.source + t - p.lo) * kr.ld_token + h * kr.ld_head + c0, left, x[u]);
                }
#pragma unroll
                for (int u = 0; u < KV_ROWS; ++u) {
                    const int t = t0 + u * lanes;
                    if (t >= p.hi) continue;
                    int q[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) q[e] = kv_quantize(x[u][e], f.k[e], f.sb[e], f.se[e], f.m[e], bottom, top);
                    store_codes8(kv.k + block + (int64_t)t * row_bytes, c0, kv.packed, q);
                    widen(q);
                }
            }
            uint2 lo = {0, 0}, hi = {0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo.x |= (uint32_t)(mn[e] & 255) << (8 * e);
                lo.y |= (uint32_t)(mn[e + 4] & 255) << (8 * e);
                hi.x |= (uint32_t)(mx[e] & 255) << (8 * e);
                hi.y |= (uint32_t)(mx[e + 4] & 255) << (8 * e);
            }
            part_lo[threadIdx.x] = lo;
            part_hi[threadIdx.x] = hi;
        }
        __syncthreads();
        {   // thread t: byte t of the lower bounds, then of the upper ones
            const int8_t *lo = reinterpret_cast<const int8_t *>(part_lo), *hi = reinterpret_cast<const int8_t *>(part_hi);
            for (int t = threadIdx.x; t < 2 * kv.dpad; t += KV_THREADS) {
                const bool upper = t >= kv.dpad;
                const int8_t *src = upper ? hi + t - kv.dpad : lo + t;
                int best = src[0];
                for (int u = 1; u < lanes; ++u) {
                    const int q = src[u * kv.dpad];
                    best = upper ? (q > best ? q : best) : (q < best ? q : best);
                }
                kv.bounds[(p.page * kv.heads + h) * 2 * kv.dpad + t] = (int8_t)best;
            }
        }
        if (on) {
            const int at = h * kv.dpad + c0;
            load_floats8(kv.value.k + at, f.k);
            load_floats8(kv.value.sb + at, f.sb);
            load_floats8(kv.value.se + at, f.se);
            load_floats8(kv.value.m + at, f.m);
            const int half = 1 << (kv.value.bits - 1), most = kv.packed ? 7 : 127;
            const float bottom = (float)-half, top = (float)(half < most ? half : most);
            for (int t0 = p.lo + r; t0 < p.hi; t0 += KV_ROWS * lanes) {
                float x[KV_ROWS][8];
#pragma unroll
                for (int u = 0; u < KV_ROWS; ++u) {
                    const int t = t0 + u * lanes;
                    if (t < p.hi) kv_load8(vr.p, vr.type, (p.source + t - p.lo) * vr.ld_token + h * vr.ld_head + c0, left, x[u]);
                }
#pragma unroll
                for (int u = 0; u < KV_ROWS; ++u) {
                    const int t = t0 + u * lanes;
                    if (t >= p.hi) continue;
                    int q[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) q[e] = kv_quantize(x[u][e], f.k[e], f.sb[e], f.se[e], f.m[e], bottom, top);
                    store_codes8(kv.v + block + (int64_t)t * row_bytes, c0, kv.packed, q);
                }
            }
        }
        __syncthreads();       // the partial bounds are used again by the next page
    }
}

// x^ = k + (c + 1/2) s, each operation rounded to binary32; rows without a page are zeros.
__global__ __launch_bounds__(KV_THREADS) void kv_read_kernel(KvView kv, KvRows kr, KvRows vr, KvPlaces pl, int pieces)
{
    const int h = blockIdx.x % kv.heads, b = (blockIdx.x / kv.heads) % pl.nseq, piece = blockIdx.x / kv.heads / pl.nseq;
    const int chunks = kv.dpad >> 3, lanes = KV_THREADS / chunks, c = threadIdx.x % chunks, r = threadIdx.x / chunks, c0 = 8 * c;
    const int row_bytes = kv.row_bytes(), left = kv.dim - c0;
    if (r >= lanes || left <= 0) return;
    int64_t row0, count;
    const int64_t first = pl.first[b];
    rows_of(pl, b, row0, count);
    if (count <= 0) return;
    const int64_t column0 = first >> kv.page_shift, columns = ((first + count - 1) >> kv.page_shift) - column0 + 1;
    float k[2][8], s[2][8];
    const int at = h * kv.dpad + c0;
    load_floats8(kv.key.k + at, k[0]);
    load_floats8(kv.key.s + at, s[0]);
    load_floats8(kv.value.k + at, k[1]);
    load_floats8(kv.value.s + at, s[1]);
    for (int64_t i = piece; i < columns; i += pieces) {
        const PagePart p = page_part(kv, pl, b, first, row0, count, column0 + i);
        const int64_t block = (p.page * kv.heads + h) * kv.page * row_bytes;
        for (int t0 = p.lo + r; t0 < p.hi; t0 += KV_ROWS * lanes) {
            int q[2][KV_ROWS][8];
#pragma unroll
            for (int u = 0; u < KV_ROWS; ++u) {
                const int t = t0 + u * lanes;
                if (t < p.hi && p.page >= 0) {
                    load_codes8(kv.k + block + (int64_t)t * row_bytes, c0, kv.packed, q[0][u]);
                    load_codes8(kv.v + block + (int64_t)t * row_bytes, c0, kv.packed, q[1][u]);
                }
            }
#pragma unroll
            for (int u = 0; u < KV_ROWS; ++u) {
                const int t = t0 + u * lanes;
                if (t >= p.hi) continue;
                const int64_t row = p.source + t - p.lo;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = p.page >= 0 ? __fadd_rn(__fmul_rn((float)q[w][u][e] + 0.5f, s[w][e]), k[w][e]) : 0.0f;
                    const KvRows &out = w ? vr : kr;
                    kv_store<8>(out.p, out.type, row * out.ld_token + h * out.ld_head + c0, left, x);
                }
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

// Parts a sequence's pages are dealt to.  A decoding step has one page per sequence; a prompt has as many as its share
// of the rows fills, and a longer one than the others takes more turns of the same workgroups.
int pieces_of(const KvView &kv, const KvPlaces &pl)
{
    const int64_t mean = ceil_div(pl.n, (int64_t)pl.nseq), most = ceil_div(pl.n, (int64_t)kv.page) + 1;
    int64_t pieces = pl.n == pl.nseq ? 1 : 2 * ceil_div(mean, (int64_t)kv.page) + 1;
    const int64_t room = ceil_div(int64_t(4096), (int64_t)pl.nseq * kv.heads);     // up to 16 workgroups per CU in any case
    if (pl.n != pl.nseq && pieces < room) pieces = room;
    const int64_t grid = KV_MAX_BLOCKS / ((int64_t)pl.nseq * kv.heads);            // >= 1: the entry points check it
    if (pieces > grid) pieces = grid;
    return (int)(pieces < most ? pieces : most);
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
    const int pieces = pieces_of(kv, pl);
    kv_write_kernel<<<(unsigned)(pieces * pl.nseq * kv.heads), KV_THREADS, 0, st>>>(kv, k, v, pl, pieces);
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvView &kv, const KvRows &k, const KvRows &v, const KvPlaces &pl, hipStream_t st)
{
    if (pl.n <= 0 || pl.nseq <= 0) return hipSuccess;
    const int pieces = pieces_of(kv, pl);
    kv_read_kernel<<<(unsigned)(pieces * pl.nseq * kv.heads), KV_THREADS, 0, st>>>(kv, k, v, pl, pieces);
    return hipGetLastError();
}

}  // namespace lpq
