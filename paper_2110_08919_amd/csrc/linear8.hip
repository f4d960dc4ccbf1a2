// Linear layers on 8-bit codes: rows to codes with a scale each, and products of such rows with rows of weights.
//
//   code[i][k] = rint(x[i][k] (127 / A_i)),  scale[i] = A_i / 127,  A_i = max_k |x[i][k]|
//   y[i][c]    = (sum_k a[i][k] b[c][k]) sa[i] sb[c] + bias[c],      the sums exact in 32 bits
//
// Measured with the rows' codes, bfloat16 unless said otherwise, weights not in a cache: 1 row, 4096 x 4096 5.8 us (4.3 where the weights are in the
// memory-side cache), 32 768 x 16 384 91 us, 5.9 TB/s; 48 float16 rows, 11 111 x 4100 19.1; 64 rows, 16 384 x 8192 36; 128 rows, 32 768 x 16 384
// 116 to 124; 129, 256, 512, 1024, 2048 rows, 4096 x 4096 18.5, 21.3, 24.2, 30 to 34, 48; 8192 rows, 8192 x 8192 499 to 513, of these 45 for the codes
// (4.5 TB/s, as a copy of memory) and 452 for the product, 2.43 POP/s, where a register-resident loop of the instruction sustains 3.46 on random
// bytes.  What is left there: a stage takes 0.81 us, 0.68 without its copies (0.62 at that loop's rate), and 10 us go before a tile's first stage
// and behind its last.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kv_internal.h"
#include "linear8_internal.h"
#include "mfma_common.h"
#include "wave_ops.h"

namespace lpq {

namespace {

// ------------------------------------------------------------------ rows to codes ----
constexpr int ROW_THREADS = 1024;

// 16 neighbouring values of a row as they lie in memory; those behind its end are 0.  Wide loads whatever the alignment, but for the row's
// last ones, which come one at a time.
template <int type>
struct Run16 {
    static constexpr int WORDS = type == LPQ_TYPE_F32 ? 16 : 8;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const void *base, int64_t at, int left)
    {
        constexpr int SIZE = type == LPQ_TYPE_F32 ? 4 : 2;
        const char *const p = static_cast<const char *>(base) + SIZE * at;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
        if (left >= 16) {
            uint4 t[WORDS / 4];
            __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) {
                w[4 * i] = t[i].x; w[4 * i + 1] = t[i].y; w[4 * i + 2] = t[i].z; w[4 * i + 3] = t[i].w;
            }
        } else if (left > 0) {
#pragma unroll
            for (int e = 0; e < 15; ++e)
                if (e < left) {
                    if (type == LPQ_TYPE_F32) w[e] = reinterpret_cast<const uint32_t *>(p)[e];
                    else w[e >> 1] |= (uint32_t) reinterpret_cast<const uint16_t *>(p)[e] << (16 * (e & 1));
                }
        }
    }
    // Magnitudes compare as their bits do, infinity and NaN on top; of a 16-bit type two at a time, whose larger one magnitude() takes.
    __device__ __forceinline__ void most(uint32_t &m) const
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if (type == LPQ_TYPE_F32) {
                const uint32_t b = w[i] & 0x7fffffffu;
                m = b > m ? b : m;
            } else {
                typedef uint16_t Two __attribute__((ext_vector_type(2)));
                m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(Two, w[i] & 0x7fff7fffu), __builtin_bit_cast(Two, m)));
            }
        }
    }
    static __device__ __forceinline__ uint32_t magnitude(uint32_t m)
    {
        if (type == LPQ_TYPE_F32) return m;
        const uint32_t a = m & 0xffffu, b = m >> 16, c = a > b ? a : b;
        return type == LPQ_TYPE_BF16 ? c << 16 : __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)c));
    }
    __device__ __forceinline__ float value(int e) const
    {
        if (type == LPQ_TYPE_F32) return __builtin_bit_cast(float, w[e % WORDS]);
        const uint32_t u = w[e >> 1];
        if (type == LPQ_TYPE_BF16) return __builtin_bit_cast(float, e & 1 ? u & 0xffff0000u : u << 16);
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(u >> (16 * (e & 1))));
    }
};

// What a row is multiplied by to become codes.  A row below 2^-100 is taken times 2^60 first, exactly, so that 127 / A stays finite; one that
// holds an infinity or a NaN has the codes 0 and the scale NaN, so that whatever it goes into is NaN.
struct RowFactor {
    float up, by, scale;
};
__device__ __forceinline__ RowFactor row_factor(uint32_t magnitude)
{
    const float most = __builtin_bit_cast(float, magnitude);
    RowFactor f = {most < 0x1p-100f ? 0x1p60f : 1.0f, 0.0f, most / 127.0f};
    if (magnitude >= 0x7f800000u) f.scale = NAN;
    else if (magnitude) f.by = 127.0f / (most * f.up);
    return f;
}
// Codes of 16 values; all of a wave's are of one row.  Adding 1.5 x 2^23 rounds to a whole number, to nearest even, and leaves it in the low byte.
template <int type>
__device__ __forceinline__ uint4 row_codes16(const Run16<type> &r, const RowFactor &f)
{
    uint32_t c[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        uint32_t b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v = r.value(4 * g + e);
            if (type != LPQ_TYPE_F16) v *= f.up;
            b[e] = __builtin_bit_cast(uint32_t, v * f.by + 0x1.8p23f);
        }
        const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
        c[g] = f.by == 0.0f ? 0u : lo | hi;
    }
    return make_uint4(c[0], c[1], c[2], c[3]);
}

// Codes lie in blocks of 16 rows x 64 features, 1 KB each: [row / 16][feature / 64][feature % 64 / 16][row % 16][feature % 16].  A block is what a
// wave's matrix instruction takes, 16 bytes a lane, so that every load of codes is one run of memory.
__host__ __device__ __forceinline__ int64_t block_of(int64_t row16, int64_t feature64, int blocks) { return (row16 * blocks + feature64) << 10; }

// A workgroup has ROWS rows, THREADS threads each.  Rows of up to THREADS * UNITS * 16 values are read once, longer ones twice (the second
// time from a cache).  Bound by the round trips to memory.
template <int type, int ROWS, int UNITS>
__global__ __launch_bounds__(ROW_THREADS) void encode_rows_kernel(const void *__restrict__ x, int64_t ldx, int64_t n, int d, int blocks,
                                                                  int8_t *__restrict__ codes, float *__restrict__ scales)
{
    constexpr int THREADS = ROW_THREADS / ROWS;
    const int t = threadIdx.x % THREADS, mine = threadIdx.x / THREADS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + mine, from = row < n ? row : n - 1;
    const int64_t at = from * ldx;
    const int units = 4 * blocks;
    Run16<type> raw[UNITS], r;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) raw[i].load(x, at + 16 * (t + i * THREADS), d - 16 * (t + i * THREADS));
#pragma unroll
    for (int i = 0; i < UNITS; ++i) raw[i].most(most);
    for (int u = t + UNITS * THREADS; u < units; u += THREADS) {
        r.load(x, at + 16 * u, d - 16 * u);
        r.most(most);
    }
    most = Run16<type>::magnitude(most);
    most = (uint32_t)wave_max_i32((int)most);
    if (THREADS > 64) {
        __shared__ uint32_t waves[ROW_THREADS / 64];
        if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            const uint32_t o = waves[mine * (THREADS / 64) + w];
            most = o > most ? o : most;
        }
    }
    if (row >= n) return;
    const RowFactor f = row_factor(most);
    if (t == 0) scales[row] = f.scale;
    int8_t *const out = codes + block_of(row >> 4, 0, blocks) + 16 * (row & 15);
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
        if (t + i * THREADS < units) *reinterpret_cast<uint4 *>(out + 256 * (int64_t)(t + i * THREADS)) = row_codes16(raw[i], f);
    for (int u = t + UNITS * THREADS; u < units; u += THREADS) {
        r.load(x, at + 16 * u, d - 16 * u);
        *reinterpret_cast<uint4 *>(out + 256 * (int64_t)u) = row_codes16(r, f);
    }
}

// Many rows: a wave to each of a workgroup's 8, two workgroups to a CU, so that one reads while the other writes.  The codes of 1024 features at a time
// are turned over in LDS and leave as whole lines (8 rows x 16 features are 128 bytes of a block).
constexpr int MANY_ROWS = 8, MANY_THREADS = 64 * MANY_ROWS;
template <int type, int UNITS>
__global__ __launch_bounds__(MANY_THREADS, 4) void encode_many_kernel(const void *__restrict__ x, int64_t ldx, int64_t n, int d, int blocks,
                                                                      int8_t *__restrict__ codes, float *__restrict__ scales)
{
    __shared__ uint4 turn[2][64 * MANY_ROWS];
    const int lane = threadIdx.x & 63, mine = threadIdx.x >> 6, units = 4 * blocks;
    const int64_t row0 = (int64_t)blockIdx.x * MANY_ROWS, row = row0 + mine;
    const int64_t at = (row < n ? row : n - 1) * ldx;
    Run16<type> raw[UNITS], r;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) raw[i].load(x, at + 16 * (lane + 64 * i), d - 16 * (lane + 64 * i));
#pragma unroll
    for (int i = 0; i < UNITS; ++i) raw[i].most(most);
    for (int u = lane + 64 * UNITS; u < units; u += 64) {
        r.load(x, at + 16 * u, d - 16 * u);
        r.most(most);
    }
    const RowFactor f = row_factor((uint32_t)wave_max_i32((int)Run16<type>::magnitude(most)));
    if (lane == 0 && row < n) scales[row] = f.scale;
    int8_t *const out = codes + block_of(row0 >> 4, 0, blocks) + 16 * (row0 & 8);
    const int to_unit = threadIdx.x / MANY_ROWS, to_row = threadIdx.x % MANY_ROWS;
    const auto store = [&](int i, const Run16<type> &from) {
        uint4 *const t = turn[i & 1];
        t[lane * MANY_ROWS + (mine ^ (lane & 7))] = row_codes16(from, f);
        __syncthreads();
        if (64 * i + to_unit < units && row0 + to_row < n)
            *reinterpret_cast<uint4 *>(out + 256 * (int64_t)(64 * i + to_unit) + 16 * to_row) = t[to_unit * MANY_ROWS + (to_row ^ (to_unit & 7))];
    };
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
        if (64 * i < units) store(i, raw[i]);
    for (int i = UNITS; 64 * i < units; ++i) {
        r.load(x, at + 16 * (lane + 64 * i), d - 16 * (lane + 64 * i));
        store(i, r);
    }
}

// ------------------------------------------------------------------------ products ----
// A scale as mantissa and exponent: sum * ma * mb stays in binary32's middle range whatever the scales, and the exponents come on last, with one
// rounding.  Where nothing leaves that range the result is fl(fl(fl(sum) sa) sb), bit for bit: a sum beyond 2^24 is rounded before it is scaled.
struct Scale {
    float m;
    int e;
};
__device__ __forceinline__ Scale split_scale(float s) { return {__builtin_amdgcn_frexp_mantf(s), __builtin_amdgcn_frexp_expf(s)}; }
__device__ __forceinline__ float scaled(int sum, const Scale &a, const Scale &b) { return ldexpf(((float)sum * a.m) * b.m, a.e + b.e); }

// Few rows.  Bound by reading the weights, which go from memory to registers, each byte to one wave: a workgroup's eight waves share CT tiles
// of 16 channels and take every eighth run of 128 features of them (v_mfma_i32_16x16x64_i8, channels as rows of the result), and the
// eight sums come together through LDS.  The tokens' codes, MT tiles of 16, come from the cache of their chiplet with each run.  FUSED (few rows):
// the workgroup makes the codes itself, in LDS, while its first weights are under way: one launch, and no round trip through memory (4096 x 4096: 4 rows 6.4 us,
// 16 in two launches 10.1).
// A barrier for what the waves write to and read from LDS; loads from memory stay under way.
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0); known to the compiler, which then counts only what comes after
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr int STREAM_WAVES = 8, STREAM_THREADS = 64 * STREAM_WAVES, STREAM_K = 128;
constexpr int FUSED_VALUES = 16384;           // values of x that a workgroup makes codes of: 32 a thread
constexpr int FUSED_ROWS = 8, FUSED_PAD = 16;
constexpr int STREAM_ROWS = 128, CUS = 256;

struct StreamWork {
    const int8_t *x, *w;
    const float *sx, *sw;
    int m;
    int64_t n;
    int runs;                    // of STREAM_K features
    Linear8Out out;
    const void *raw;             // FUSED: rows of `out.type`
    int64_t ld_raw;
    int d, rows;                 // FUSED: m rounded up to a power of two
};

// Loads past the end of a buffer give zeros and ask for nothing, so that the loop's loads need no branches: behind a branch the compiler
// would wait for all that is under way at every use.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer codes_buffer(const int8_t *p, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p), 0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ v4i load16(Buffer b, int at) { return __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(b, at, 0, 0)); }

constexpr int stream_waves_per_simd(int mt, int ct) { return (mt + ct <= 4 && mt < 3) || (ct == 1 && mt == 4) ? 4 : 2; }
// Runs of weights and of codes in flight.
constexpr int stream_depth(int mt, int ct) { return mt + ct <= 3 || ct == 1 ? 4 : 2; }
constexpr int stream_depth_x(int mt, int ct) { return mt + ct <= 3 ? 4 : mt >= 4 ? 1 : 2; }
constexpr int stream_channels(int mt) { return mt <= 4 ? 4 : mt <= 6 ? 3 : 2; }      // most tiles of 16 channels: the sums fit LDS

template <int MT, int CT, bool FUSED, int type>
__global__ __launch_bounds__(STREAM_THREADS, stream_waves_per_simd(MT, CT)) void linear8_stream_kernel(StreamWork g)
{
    static_assert(!FUSED || MT == 1);
    constexpr int DEPTH = stream_depth(MT, CT), DEPTH_X = stream_depth_x(MT, CT), ENDS = (CT * MT + STREAM_WAVES - 1) / STREAM_WAVES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int in_tile = lane & 15, chunk = 16 * (lane >> 4);
    const int64_t ch0 = (int64_t)blockIdx.x * 16 * CT;
    __shared__ __align__(16) int4 sums[STREAM_WAVES * CT * MT * 64];
    __shared__ __align__(16) int8_t own[FUSED ? FUSED_VALUES + FUSED_ROWS * FUSED_PAD : 16];
    __shared__ uint32_t magnitude[STREAM_WAVES];
    __shared__ Scale own_scale[FUSED_ROWS];

    // FUSED: the rows' values first, so that waiting for them is not waiting for the weights
    constexpr int UNITS = FUSED ? FUSED_VALUES / (16 * STREAM_THREADS) : 1;
    Run16<type> raw[UNITS];
    const int row_threads = FUSED ? STREAM_THREADS / g.rows : 1, row = FUSED ? (int)threadIdx.x / row_threads : 0;
    const int me = threadIdx.x - row * row_threads;
    if (FUSED) {
        const int from = row < g.m ? row : g.m - 1;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = 16 * (me + i * row_threads);
            raw[i].load(g.raw, from * g.ld_raw + u, g.d - u);
        }
    }

    const int bytes = g.runs * STREAM_K, tile_bytes = 16 * bytes;
    const int64_t tiles = (g.n - ch0 + 15) >> 4;
    const Buffer wb = codes_buffer(g.w + (ch0 >> 4) * tile_bytes, (tiles < CT ? tiles : CT) * tile_bytes);
    const Buffer xb = FUSED ? wb : codes_buffer(g.x, (int64_t)((g.m + 15) >> 4) * tile_bytes);
    const int own_at = FUSED ? (in_tile < g.m ? in_tile : g.m - 1) * (bytes + FUSED_PAD) + chunk : 0;
    v4i fw[DEPTH][CT][2], fx[DEPTH_X][MT][2];
    const auto load_x = [&](int slot, int run) {
        const int at = (run < g.runs ? run * (16 * STREAM_K) : 1 << 30) + 16 * lane;
        if (!FUSED) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < MT; ++j) fx[slot][j][k] = load16(xb, at + j * tile_bytes + 1024 * k);
        }
    };
    const auto load_w = [&](int slot, int run) {
        const int at = (run < g.runs ? run * (16 * STREAM_K) : 1 << 30) + 16 * lane;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < CT; ++i) fw[slot][i][k] = load16(wb, at + i * tile_bytes + 1024 * k);
    };
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) load_w(i, wave + i * STREAM_WAVES);
#pragma unroll
    for (int i = 0; i < DEPTH_X; ++i) load_x(i, wave + i * STREAM_WAVES);

    // what the results are multiplied by, long before it is needed
    float end_w[4], end_bias[4], end_x;
    const float *const bias = g.out.bias ? g.out.bias : g.sw;
    const auto ends = [&](int u) {
        const int token = 16 * (u % MT) + in_tile;
        end_x = FUSED ? 0.0f : g.sx[token < g.m ? token : 0];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t c = ch0 + 16 * (u / MT) + 4 * (lane >> 4) + e, at = c < g.n ? c : g.n - 1;
            end_w[e] = g.sw[at];
            end_bias[e] = bias[at];
        }
    };
    ends(wave < CT * MT ? wave : 0);

    if (FUSED) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) raw[i].most(most);
        most = (uint32_t)wave_max_i32((int)Run16<type>::magnitude(most));
        if (lane == 0) magnitude[wave] = most;
        lds_barrier();
        const int waves = STREAM_WAVES / g.rows, first = wave / waves * waves;
        for (int i = 0; i < waves; ++i) most = magnitude[first + i] > most ? magnitude[first + i] : most;
        const RowFactor f = row_factor(most);
        if (me == 0) own_scale[row] = split_scale(f.scale);
        int8_t *const to = own + row * (bytes + FUSED_PAD);
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = 16 * (me + i * row_threads);
            if (u < bytes) *reinterpret_cast<uint4 *>(to + u) = row_codes16(raw[i], f);
        }
        lds_barrier();
    }

    v4i acc[CT][MT];
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = v4i{0, 0, 0, 0};
    for (int run0 = wave; run0 < g.runs; run0 += DEPTH * STREAM_WAVES) {
#pragma unroll
        for (int s = 0; s < DEPTH; ++s) {
            const int run = run0 + s * STREAM_WAVES, sx = s % DEPTH_X;
            if (FUSED) {                   // past the end: any codes, times weights of zero
                const int at = run < g.runs ? run * STREAM_K : 0;
#pragma unroll
                for (int k = 0; k < 2; ++k) fx[sx][0][k] = *reinterpret_cast<const v4i *>(own + own_at + at + 64 * k);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < CT; ++i)
#pragma unroll
                    for (int j = 0; j < MT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[s][i][k], fx[sx][j][k], acc[i][j], 0, 0, 0);
            load_x(sx, run + DEPTH_X * STREAM_WAVES);
            load_w(s, run + DEPTH * STREAM_WAVES);
        }
    }
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j)
            sums[(wave * CT * MT + i * MT + j) * 64 + lane] = make_int4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
    lds_barrier();
#pragma unroll
    for (int i = 0; i < ENDS; ++i) {
        const int u = wave + i * STREAM_WAVES, token = 16 * (u % MT) + in_tile;
        if (u >= CT * MT) break;
        int t[4] = {0, 0, 0, 0};
#pragma unroll
        for (int v = 0; v < STREAM_WAVES; ++v) {
            const int4 o = sums[(v * CT * MT + u) * 64 + lane];
            t[0] += o.x; t[1] += o.y; t[2] += o.z; t[3] += o.w;
        }
        const int64_t c = ch0 + 16 * (u / MT) + 4 * (lane >> 4);
        if (token >= g.m || c >= g.n) continue;
        if (i > 0) ends(u);
        const Scale a = FUSED ? own_scale[token] : split_scale(end_x);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = scaled(t[e], a, split_scale(end_w[e]));
            if (g.out.bias) y[e] += end_bias[e];
        }
        kv_store<4>(g.out.p, FUSED ? type : g.out.type, token * g.out.ld + c, (int)(g.n - c < 4 ? g.n - c : 4), y);
    }
}

// Tiles.  The workgroup's four waves stand 2 x 2; a wave has TC x TT tiles of 32 channels x 32 tokens (v_mfma_i32_32x32x32_i8, channels as rows of
// the result, so that a lane holds 4 neighbouring channels of a token).  Stages of 64 features of all the workgroup's channels and tokens come
// into a ring in LDS by asynchronous copies of 16 bytes a lane, a block at a time, three stages ahead; the operands of the next half of a
// stage are read from there while the matrix instructions of this half run.  Bound by issue and by LDS: its 128 KB (256 x 256) leave one wave to a SIMD, so
// that nothing runs where a wave waits for the barrier, for operands or for its copies to be taken in.  8192 x 8192 x 8192: the matrix pipe is busy 59 %
// of the time, at 2.0 GHz: 32 instructions of 32 cycles of the 1600 that a stage takes, beside 64 KB read from LDS and 32 KB copied into it a
// workgroup, of 128 bytes a cycle.
constexpr int TILE_THREADS = 256, TILE_K = 64, TILE_STAGES = 4;

struct TileWork {
    const int8_t *x, *w;
    const float *sx, *sw;
    int64_t m, n;
    int blocks;                  // of 64 features in a row: a stage each
    int stages, per_part;        // of them with features, of a part
    int tiles_m, tiles_n, parts;
    Linear8Out out;
    int *sums;                   // parts > 1: [parts][m][n rounded up to 4]
};

// Copies of one wave: every fourth block of a stage, channels first, then tokens.
template <int TT, int TC>
struct TileCopies {
    static constexpr int BM = 64 * TT, BN = 64 * TC, COUNT = (BM + BN) / 64;
    const int8_t *from[COUNT];
    unsigned to;
    __device__ __forceinline__ void setup(const TileWork &g, int64_t row0, int64_t ch0, int stage, const char *ring, int wave, int lane)
    {
        to = lds_offset(ring) + 1024 * wave;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int block = wave + 4 * i;
            const bool channel = block < BN / 16;
            const int64_t last = ((channel ? g.n : g.m) - 1) >> 4;
            int64_t row16 = channel ? (ch0 >> 4) + block : (row0 >> 4) + block - BN / 16;
            row16 = row16 < last ? row16 : last;
            from[i] = (channel ? g.w : g.x) + block_of(row16, stage, g.blocks) + 16 * lane;
        }
    }
    __device__ __forceinline__ void one(int i, int slot)
    {
        async_copy16(from[i], to + slot * (BM + BN) * TILE_K + 4096 * i);
        from[i] += 1024;
    }
};

template <int TT, int TC, int TYPE, bool PARTS>
__global__ __launch_bounds__(TILE_THREADS) void linear8_tile_kernel(TileWork g)
{
    typedef TileCopies<TT, TC> Copies;
    constexpr int BM = 64 * TT, BN = 64 * TC, STAGE = (BM + BN) * TILE_K;
    __shared__ __align__(1024) char ring[TILE_STAGES * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // An XCD (workgroups are dealt to the eight of them in turn) has neighbouring tiles, in bands of BAND row tiles: what its CUs have at a time
    // shares panels in its L2 (1100 rows, 4096 x 4096: 49.7 us by rows alone, 40.0; 129, 32 768 x 16 384 174, 163; 8192, 8192 x 8192 the same).
    constexpr int BAND = 4;
    const int tiles = g.tiles_m * g.tiles_n, work = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);      // (the grid: a multiple of 8)
    if (work >= tiles * g.parts) return;
    const int part = PARTS ? work / tiles : 0, tile = PARTS ? work - part * tiles : work;
    const int band = tile / (BAND * g.tiles_n), in_band = tile - band * BAND * g.tiles_n, height = min(BAND, g.tiles_m - band * BAND);
    const int tn = in_band / height, tm = band * BAND + in_band - tn * height;
    const int64_t row0 = (int64_t)tm * BM, ch0 = (int64_t)tn * BN;
    const int wt = (wave & 1) * 32 * TT, wc = (wave >> 1) * 32 * TC;
    const int begin = part * g.per_part, stages = min(g.per_part, g.stages - begin);

    v16i acc[TC][TT];
#pragma unroll
    for (int i = 0; i < TC; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

    // what the results are multiplied by, long before it is needed
    float end_w = 0.0f, end_x = 0.0f, end_bias = 0.0f;
    if (!PARTS) {
        const int64_t c = ch0 + threadIdx.x < g.n ? ch0 + threadIdx.x : g.n - 1, t = row0 + threadIdx.x < g.m ? row0 + threadIdx.x : g.m - 1;
        end_w = g.sw[c];
        end_x = g.sx[t];
        if (g.out.bias) end_bias = g.out.bias[c];
        asm volatile("" : "+v"(end_w), "+v"(end_x), "+v"(end_bias));      // now: the copies below are counted
    }
    Copies copies;
    copies.setup(g, row0, ch0, begin, ring, wave, lane);
    const int at = (lane >> 5) * 256 + (lane & 15) * 16 + ((lane >> 4) & 1) * 1024;
    v4i fc[2][TC], ft[2][TT];
    const auto operand = [&](int slot, int half, int k) {
        const char *const here = ring + slot * STAGE + 512 * half + at;
        if (k < TC) fc[half][k] = *reinterpret_cast<const v4i *>(here + 64 * (wc + 32 * k));
        else ft[half][k - TC] = *reinterpret_cast<const v4i *>(here + 64 * (BN + wt + 32 * (k - TC)));
    };
    // The matrix instructions of a half, and between them the reads of the next half's operands and half of a stage's copies: a wave that
    // asks for these in one go is held up by their queues for as long as the matrix pipe then has nothing to do.
    const auto multiply = [&](int half, int next_slot, bool copy, int copy_slot) {
        constexpr int STEPS = TT * TC, READS = TT + TC, COPIES = Copies::COUNT / 2;
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int i = k / TT, j = k % TT;
            __builtin_amdgcn_sched_barrier(0);
            acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fc[half][i], ft[half][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            // reads in the first half of them, so that none is waited for
#pragma unroll
            for (int r = 2 * k * READS / STEPS; r < 2 * (k + 1) * READS / STEPS && r < READS; ++r) operand(next_slot, half ^ 1, r);
            constexpr int FROM = STEPS / 2, REST = STEPS - FROM;
            if (copy && k >= FROM) {
#pragma unroll
                for (int c = (k - FROM) * COPIES / REST; c < (k - FROM + 1) * COPIES / REST; ++c) copies.one(c + (half ? 0 : COPIES), copy_slot);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // In flight: stages 0 to 2 and half of 3 ahead of the loop, whose first half completes it.
    for (int s = 0; s < TILE_STAGES - 1 && s < stages; ++s)
#pragma unroll
        for (int i = 0; i < Copies::COUNT; ++i) copies.one(i, s);
    wait_vmcnt(min(stages - 1, TILE_STAGES - 2) * Copies::COUNT);
    lds_barrier();
#pragma unroll
    for (int r = 0; r < TT + TC; ++r) operand(0, 0, r);
    if (TILE_STAGES - 1 < stages) {
#pragma unroll
        for (int i = 0; i < Copies::COUNT / 2; ++i) copies.one(i, TILE_STAGES - 1);
    }
    for (int s = 0; s < stages; ++s) {
        multiply(0, s % TILE_STAGES, s + TILE_STAGES - 1 < stages, (s + TILE_STAGES - 1) % TILE_STAGES);
        // the next stage is there for all, and nobody reads this one any more: its place is filled again
        if (s + TILE_STAGES <= stages) __builtin_amdgcn_s_waitcnt(vmcnt_imm((TILE_STAGES - 2) * Copies::COUNT));
        else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        lds_barrier();
        multiply(1, (s + 1) % TILE_STAGES, s + TILE_STAGES < stages, s % TILE_STAGES);      // (behind the last stage: reads for nothing)
    }

    if (PARTS) {
        const int64_t wide = (g.n + 3) & ~int64_t(3);
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            const int64_t token = row0 + wt + 32 * j + (lane & 31);
#pragma unroll
            for (int i = 0; i < TC; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t c = ch0 + wc + 32 * i + 8 * q + 4 * (lane >> 5);
                    if (token < g.m && c < g.n)
                        *reinterpret_cast<int4 *>(g.sums + ((int64_t)part * g.m + token) * wide + c) =
                            make_int4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                }
        }
        return;
    }
    // The ring's memory turns each wave's tiles over, 32 tokens at a time: in by channels of a token, out in whole lines of a token's row.
    constexpr int WIDTH = 32 * TC, SIZE = TYPE == LPQ_TYPE_F32 ? 4 : 2, PITCH = WIDTH * SIZE + 16, LANES = WIDTH / 8;
    static_assert(4 * 32 * PITCH + 8 * (BM + 2 * BN) <= TILE_STAGES * STAGE);
    char *const own = ring + wave * 32 * PITCH;
    Scale *const scales_w = reinterpret_cast<Scale *>(ring + 4 * 32 * PITCH), *const scales_x = scales_w + BN;
    float *const biases = reinterpret_cast<float *>(scales_x + BM);
    lds_barrier();
    if (BN == TILE_THREADS || threadIdx.x < BN) {
        scales_w[threadIdx.x] = split_scale(end_w);
        biases[threadIdx.x] = end_bias;
    }
    if (BM == TILE_THREADS || threadIdx.x < BM) scales_x[threadIdx.x] = split_scale(end_x);
    lds_barrier();
    Scale by[TC][16];            // of a lane's channels, for all its tokens
#pragma unroll
    for (int i = 0; i < TC; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) by[i][e] = scales_w[wc + 32 * i + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const Scale a = scales_x[wt + 32 * j + (lane & 31)];
#pragma unroll
        for (int i = 0; i < TC; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = 32 * i + 8 * q + 4 * (lane >> 5);
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = scaled(acc[i][j][4 * q + e], a, by[i][4 * q + e]);
                    if (g.out.bias) y[e] += biases[wc + c + e];
                }
                kv_store<4>(own, TYPE, (lane & 31) * (PITCH / SIZE) + c, 4, y);
            }
        wave_lds_sync();
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += 64 / LANES) {
            const int r = r0 + lane / LANES, c = 8 * (lane % LANES);
            const int64_t token = row0 + wt + 32 * j + r, channel = ch0 + wc + c;
            const int left = (int)(g.n - channel < 8 ? g.n - channel : 8);
            if (token >= g.m || left <= 0) continue;
            if (TYPE == LPQ_TYPE_F32) {
                float y[8];
                __builtin_memcpy(y, own + r * PITCH + c * SIZE, 32);
                kv_store_pieces<8>(static_cast<float *>(g.out.p) + token * g.out.ld + channel, left, y);
            } else {
                uint16_t y[8];
                __builtin_memcpy(y, own + r * PITCH + c * SIZE, 16);
                kv_store_pieces<8>(static_cast<uint16_t *>(g.out.p) + token * g.out.ld + channel, left, y);
            }
        }
        wave_lds_sync();
    }
}

// Sums of parts, in order, to results: 4 channels of a token a thread.
template <int TYPE>
__global__ __launch_bounds__(TILE_THREADS) void linear8_join_kernel(TileWork g, unsigned groups)
{
    const int64_t u = (int64_t)blockIdx.x * TILE_THREADS + threadIdx.x, token = u / groups;
    if (token >= g.m) return;
    const int64_t c = 4 * (u - token * groups), each = g.m * (4 * (int64_t)groups);
    const int *const from = g.sums + token * (4 * (int64_t)groups) + c;
    int t[4] = {0, 0, 0, 0};
#pragma unroll 4
    for (int p = 0; p < g.parts; ++p) {
        const int4 v = *reinterpret_cast<const int4 *>(from + p * each);
        t[0] += v.x; t[1] += v.y; t[2] += v.z; t[3] += v.w;
    }
    const Scale a = split_scale(g.sx[token]);
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t ce = c + e < g.n ? c + e : g.n - 1;
        y[e] = scaled(t[e], a, split_scale(g.sw[ce]));
        if (g.out.bias) y[e] += g.out.bias[ce];
    }
    kv_store<4>(g.out.p, TYPE, token * g.out.ld + c, (int)(g.n - c < 4 ? g.n - c : 4), y);
}

}  // namespace

hipError_t launch_encode_rows(const void *x, int64_t ldx, int type, int64_t n, int d, int8_t *codes, float *scales, hipStream_t st)
{
    if (n == 0) return hipSuccess;
    const int blocks = row_blocks(d);
    const auto go = [&](auto t) {
        constexpr int T = decltype(t)::value, WIDE = T == LPQ_TYPE_F32 ? 2 : 1;
        if (n >= 2048) encode_many_kernel<T, 8 / WIDE><<<dim3((unsigned)ceil_div(n, (int64_t)MANY_ROWS)), MANY_THREADS, 0, st>>>(x, ldx, n, d, blocks, codes, scales);
        else if (n >= 1024 || d <= 4096) encode_rows_kernel<T, 4, 4 / WIDE><<<dim3((unsigned)ceil_div(n, (int64_t)4)), ROW_THREADS, 0, st>>>(x, ldx, n, d, blocks, codes, scales);
        else encode_rows_kernel<T, 1, 2><<<dim3((unsigned)n), ROW_THREADS, 0, st>>>(x, ldx, n, d, blocks, codes, scales);
    };
    if (type == LPQ_TYPE_F32) go(std::integral_constant<int, LPQ_TYPE_F32>());
    else if (type == LPQ_TYPE_F16) go(std::integral_constant<int, LPQ_TYPE_F16>());
    else go(std::integral_constant<int, LPQ_TYPE_BF16>());
    return hipGetLastError();
}

// What takes the shortest time by these estimates, in microseconds beside what all have in common (measured over 33 to 8192 rows, 1024 to 32 768
// channels and 1024 to 16 384 features, within a fifth; k: workgroups to a CU).  None is below the weights at 4.5 TB/s, about the best that more than 32
// rows had them at (128 rows, 32 768 x 16 384: 4.3 to 4.6; up to 32 rows, which need no estimate, 5.9); of estimates that stand there the first looked at
// stays: few rows' way, then small tiles, then few parts.  Few rows: what a workgroup reads at 60 GB/s; of tiles of 16 channels as many as leave one
// generation of workgroups (48 rows, 11 111 x 4100: 1, 2, 3, 4 tiles 23.7, 22.8, 19.1, 20.4 us; 64 rows, 16 384 x 8192: 48, 42.8, 46.6, 36.1).  Tiles:
// a stage takes 0.21 us (64 x 64), 0.33 us (128 x 128) and 0.83 us (256 x 256) alone on its CU, and more together with others.  Parts cost a launch
// and 0.42 us for a MB of sums (128 rows, 1024 x 16 384: tiles of 64 in 1, 2, 4, 8 parts 59.6, 37.5, 25.4, 21.1 us, few rows' way 40.5).
Linear8Plan linear8_plan(int64_t m, int64_t n, int d)
{
    const double stages = (double)ceil_div(d, TILE_K);
    Linear8Plan best = {0, 0, 0, 0};
    const double weights = n * 64 * stages / 4.5e6;
    double least = INFINITY;
    if (m <= STREAM_ROWS) {
        const int tiles = (int)ceil_div(m, (int64_t)16), mt = tiles == 5 ? 6 : tiles == 7 ? 8 : tiles;
        const int ct = (int)std::min<int64_t>(stream_channels(mt), std::max<int64_t>(1, ceil_div(n, 16 * CUS)));
        const double k = std::max(1.0, (double)n / (16 * ct) / CUS);
        best = {16 * mt, 16 * ct, 0, 0};
        if (mt <= 2) return best;
        least = std::max(k * 1024 * (mt + ct) * stages / 60e3, weights);
    }
    for (const int size : {64, 128, 256}) {
        const double tiles = (double)ceil_div(m, (int64_t)size) * ceil_div(n, (int64_t)size);
        for (int parts = 1; parts <= (size == 256 ? 1 : 16) && 4 * parts <= std::max(stages, 4.0); parts *= 2) {
            const double k = tiles * parts / CUS, per_part = ceil(stages / parts);
            double t = size == 64 ? per_part * std::max(0.21, 0.125 * k) : size == 128 ? per_part * std::max(0.33, 0.1 + 0.28 * k)
                                                                                       : ceil(k) * (12 + per_part * 0.83);
            t = std::max(t, weights);
            const double sums = (double)parts * m * round_up(n, 4) * 4;
            if (parts > 1) t += 3 + 0.42e-6 * sums;
            if (t >= least) continue;
            least = t;
            best = {size, size, parts, parts > 1 ? (size_t)sums : 0};
        }
    }
    if (best.parts > 1) {        // none of them empty
        best.parts = (int)ceil_div((int)stages, (int)ceil_div((int)stages, best.parts));
        best.bytes = (size_t)best.parts * m * round_up(n, 4) * 4;
    }
    return best;
}

bool linear8_fused(int64_t m, int d) { return m <= FUSED_ROWS && next_pow2((int)m) * 64 * row_blocks(d) <= FUSED_VALUES; }

template <int MT>
static void stream(const StreamWork &g, int channels, dim3 grid, hipStream_t st)
{
    constexpr int MOST = stream_channels(MT);
    if (channels == 16) linear8_stream_kernel<MT, 1, false, 0><<<grid, STREAM_THREADS, 0, st>>>(g);
    else if (channels == 32) linear8_stream_kernel<MT, 2, false, 0><<<grid, STREAM_THREADS, 0, st>>>(g);
    else if (channels == 48) linear8_stream_kernel<MT, MOST < 3 ? MOST : 3, false, 0><<<grid, STREAM_THREADS, 0, st>>>(g);
    else linear8_stream_kernel<MT, MOST, false, 0><<<grid, STREAM_THREADS, 0, st>>>(g);
}

static hipError_t launch_stream(const StreamWork &g, const Linear8Plan &plan, hipStream_t st)
{
    const dim3 grid((unsigned)ceil_div(g.n, (int64_t)plan.channels));
    switch (plan.rows) {
    case 16: stream<1>(g, plan.channels, grid, st); break;
    case 32: stream<2>(g, plan.channels, grid, st); break;
    case 48: stream<3>(g, plan.channels, grid, st); break;
    case 64: stream<4>(g, plan.channels, grid, st); break;
    case 96: stream<6>(g, plan.channels, grid, st); break;
    default: stream<8>(g, plan.channels, grid, st); break;
    }
    return hipGetLastError();
}

hipError_t launch_linear8_fused(const void *x, int64_t ldx, int64_t m, const RowCodes &w, int d, const Linear8Out &out, hipStream_t st)
{
    const StreamWork g = {nullptr, w.codes, nullptr, w.scales, (int)m, w.n, row_blocks(d) / 2, out, x, ldx, d, next_pow2((int)m)};
    const dim3 grid((unsigned)ceil_div(w.n, (int64_t)16));
    if (out.type == LPQ_TYPE_F32) linear8_stream_kernel<1, 1, true, LPQ_TYPE_F32><<<grid, STREAM_THREADS, 0, st>>>(g);
    else if (out.type == LPQ_TYPE_F16) linear8_stream_kernel<1, 1, true, LPQ_TYPE_F16><<<grid, STREAM_THREADS, 0, st>>>(g);
    else linear8_stream_kernel<1, 1, true, LPQ_TYPE_BF16><<<grid, STREAM_THREADS, 0, st>>>(g);
    return hipGetLastError();
}

hipError_t launch_linear8(const RowCodes &x, const RowCodes &w, int d, const Linear8Out &out, const Linear8Plan &plan, void *workspace, hipStream_t st)
{
    if (plan.parts == 0)
        return launch_stream({x.codes, w.codes, x.scales, w.scales, (int)x.n, w.n, row_blocks(d) / 2, out, nullptr, 0, d, 0}, plan, st);
    const int stages = (int)ceil_div(d, TILE_K);
    const TileWork g = {x.codes, w.codes, x.scales, w.scales, x.n, w.n, row_blocks(d), stages, (int)ceil_div(stages, plan.parts),
                        (int)ceil_div(x.n, (int64_t)plan.rows), (int)ceil_div(w.n, (int64_t)plan.channels), plan.parts, out,
                        static_cast<int *>(workspace)};
    const dim3 grid((unsigned)round_up((int64_t)g.tiles_m * g.tiles_n * plan.parts, 8));
    if (plan.parts > 1) {
        if (plan.rows == 128) linear8_tile_kernel<2, 2, 0, true><<<grid, TILE_THREADS, 0, st>>>(g);
        else linear8_tile_kernel<1, 1, 0, true><<<grid, TILE_THREADS, 0, st>>>(g);
    }
    const auto go = [&](auto t) {
        constexpr int T = decltype(t)::value;
        if (plan.parts > 1) {
            const int64_t groups = ceil_div(w.n, (int64_t)4);
            linear8_join_kernel<T><<<dim3((unsigned)ceil_div(x.n * groups, (int64_t)TILE_THREADS)), TILE_THREADS, 0, st>>>(g, (unsigned)groups);
        } else if (plan.rows == 256) {
            linear8_tile_kernel<4, 4, T, false><<<grid, TILE_THREADS, 0, st>>>(g);
        } else if (plan.rows == 128) {
            linear8_tile_kernel<2, 2, T, false><<<grid, TILE_THREADS, 0, st>>>(g);
        } else {
            linear8_tile_kernel<1, 1, T, false><<<grid, TILE_THREADS, 0, st>>>(g);
        }
    };
    if (out.type == LPQ_TYPE_F32) go(std::integral_constant<int, LPQ_TYPE_F32>());
    else if (out.type == LPQ_TYPE_F16) go(std::integral_constant<int, LPQ_TYPE_F16>());
    else go(std::integral_constant<int, LPQ_TYPE_BF16>());
    return hipGetLastError();
}

}  // namespace lpq
