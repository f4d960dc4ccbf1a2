// Linear layers on 8-bit codes: rows to codes with a scale each, and products of such rows with rows of weights.
//
//   code[i][k] = rint(x[i][k] (127 / A_i)),  scale[i] = A_i / 127,  A_i = max_k |x[i][k]|
//   y[i][c]    = (sum_k a[i][k] b[c][k]) sa[i] sb[c] + bias[c],      the sums exact in 32 bits
#include <algorithm>
#include <type_traits>

#include "kv_internal.h"
#include "linear8_internal.h"
#include "mfma_common.h"
#include "wave_ops.h"

namespace lpq {

namespace {

// ------------------------------------------------------------------ rows to codes ----
constexpr int ROW_THREADS = 256;
constexpr int ROW_UNITS = 8;        // units of 8 values that a thread keeps in registers

__device__ __forceinline__ uint32_t magnitude8(const float *v)
{
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;      // ordered as the magnitudes, infinity and NaN on top
        most = b > most ? b : most;
    }
    return most;
}

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
__device__ __forceinline__ uint2 row_codes8(const float *v, const RowFactor &f)
{
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = rintf((v[e] * f.up) * f.by);
        c[e] = f.by == 0.0f ? 0u : (uint32_t)(int)t;
    }
    const uint32_t lo = __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u) | __builtin_amdgcn_perm(c[3], c[2], 0x04000c0cu);
    const uint32_t hi = __builtin_amdgcn_perm(c[5], c[4], 0x0c0c0400u) | __builtin_amdgcn_perm(c[7], c[6], 0x04000c0cu);
    return make_uint2(lo, hi);
}

// Rows of up to THREADS * UNITS * 8 values are read once, by THREADS threads each, longer ones twice (the second time from a cache).
template <int type, int THREADS, int UNITS>
__global__ __launch_bounds__(ROW_THREADS) void encode_rows_kernel(const void *__restrict__ x, int64_t ldx, int64_t n, int d, int units,
                                                                  int8_t *__restrict__ codes, int64_t ld, float *__restrict__ scales)
{
    constexpr int ROWS = ROW_THREADS / THREADS;
    const int t = threadIdx.x % THREADS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
    if (ROWS > 1 && row >= n) return;
    const int64_t at = row * ldx;
    Raw8 raw[UNITS];
    float v[8];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) raw[i] = kv_load8(x, type, at + 8 * (t + i * THREADS), d - 8 * (t + i * THREADS));
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        kv_floats8(raw[i], type, d - 8 * (t + i * THREADS), v);
        const uint32_t b = magnitude8(v);
        most = b > most ? b : most;
    }
    for (int u = t + UNITS * THREADS; u < units; u += THREADS) {
        kv_floats8(kv_load8(x, type, at + 8 * u, d - 8 * u), type, d - 8 * u, v);
        const uint32_t b = magnitude8(v);
        most = b > most ? b : most;
    }
    most = (uint32_t)wave_max_i32((int)most);
    if (THREADS > 64) {
        __shared__ uint32_t waves[ROW_THREADS / 64];
        if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) most = waves[w] > most ? waves[w] : most;
    }
    const RowFactor f = row_factor(most);
    if (t == 0) scales[row] = f.scale;
    int8_t *const out = codes + row * ld;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int u = t + i * THREADS;
        if (u >= units) break;
        kv_floats8(raw[i], type, d - 8 * u, v);
        *reinterpret_cast<uint2 *>(out + 8 * u) = row_codes8(v, f);
    }
    for (int u = t + UNITS * THREADS; u < units; u += THREADS) {
        kv_floats8(kv_load8(x, type, at + 8 * u, d - 8 * u), type, d - 8 * u, v);
        *reinterpret_cast<uint2 *>(out + 8 * u) = row_codes8(v, f);
    }
}

// ------------------------------------------------------------------------ products ----
// A scale as mantissa and exponent: sum * ma * mb stays in binary32's middle range whatever the scales, and the exponents come on last, with one
// rounding.  Where nothing leaves that range the result is fl(fl(sum sa) sb), bit for bit.
struct Scale {
    float m;
    int e;
};
__device__ __forceinline__ Scale split_scale(float s) { return {__builtin_amdgcn_frexp_mantf(s), __builtin_amdgcn_frexp_expf(s)}; }
__device__ __forceinline__ float scaled(int sum, const Scale &a, const Scale &b) { return ldexpf(((float)sum * a.m) * b.m, a.e + b.e); }

// Tiles.  The workgroup's four waves stand 2 x 2; a wave has TC x TT tiles of 32 channels x 32 tokens (v_mfma_i32_32x32x32_i8, channels as rows of
// the result, so that a lane holds 4 neighbouring channels of a token).  Stages of 64 features of all the workgroup's channels and tokens come
// into a ring in LDS by asynchronous copies of 16 bytes a lane.
constexpr int TILE_THREADS = 256, TILE_K = 64, TILE_STAGES = 4;

struct TileWork {
    const int8_t *x, *w;
    const float *sx, *sw;
    int64_t ldx, ldw, m, n;
    int stages;                  // of TILE_K features
    int per_part;                // stages of a part
    int tiles_m, tiles_n, parts;
    Linear8Out out;
    int *sums;                   // parts > 1: [parts][m][n rounded up to 4]
};

template <int TT, int TC>
__device__ __forceinline__ void tile_copy(const TileWork &g, int64_t row0, int64_t ch0, int stage, char *ring, int wave, int lane)
{
    constexpr int BM = 64 * TT, BN = 64 * TC, RUNS = (BM + BN) / 16;      // runs of 16 rows, 1 KB
    const unsigned base = lds_offset(ring) + (stage % TILE_STAGES) * (BM + BN) * TILE_K;
#pragma unroll
    for (int i = 0; i < RUNS / 4; ++i) {
        const int run = wave + 4 * i, r = 16 * run + (lane >> 2), slot = lane & 3;      // channels first, then tokens
        const bool channel = r < BN;
        const int in = channel ? r : r - BN;
        const int chunk = slot ^ swz<4>(in);
        int64_t row = (channel ? ch0 : row0) + in;
        const int64_t last = (channel ? g.n : g.m) - 1;
        row = row < last ? row : last;
        async_copy16((channel ? g.w + row * g.ldw : g.x + row * g.ldx) + (int64_t)stage * TILE_K + 16 * chunk, base + 1024 * run);
    }
}

template <int TT, int TC, int TYPE, bool PARTS>
__global__ __launch_bounds__(TILE_THREADS) void linear8_tile_kernel(TileWork g)
{
    constexpr int BM = 64 * TT, BN = 64 * TC, STAGE = (BM + BN) * TILE_K, COPIES = (BM + BN) / 64;
    __shared__ __align__(1024) char ring[TILE_STAGES * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = PARTS ? blockIdx.x / (g.tiles_m * g.tiles_n) : 0, tile = PARTS ? blockIdx.x - part * (g.tiles_m * g.tiles_n) : blockIdx.x;
    const int tm = tile % g.tiles_m, tn = tile / g.tiles_m;
    const int64_t row0 = (int64_t)tm * BM, ch0 = (int64_t)tn * BN;
    const int wt = (wave & 1) * 32 * TT, wc = (wave >> 1) * 32 * TC;
    const int begin = part * g.per_part, end = PARTS ? min(begin + g.per_part, g.stages) : g.stages;

    v16i acc[TC][TT];
#pragma unroll
    for (int i = 0; i < TC; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

    for (int s = begin; s < begin + TILE_STAGES - 1 && s < end; ++s) tile_copy<TT, TC>(g, row0, ch0, s, ring, wave, lane);
    for (int s = begin; s < end; ++s) {
        const int ahead = min(end - 1 - s, TILE_STAGES - 2);
        wait_vmcnt(ahead * COPIES);
        __syncthreads();                         // the stage is there for all, and nobody reads the one before it any more
        if (s + TILE_STAGES - 1 < end) tile_copy<TT, TC>(g, row0, ch0, s + TILE_STAGES - 1, ring, wave, lane);
        const char *const here = ring + (s % TILE_STAGES) * STAGE;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            v4i fc[TC], ft[TT];
            const int chunk = 2 * k + (lane >> 5);
#pragma unroll
            for (int i = 0; i < TC; ++i) {
                const int r = wc + 32 * i + (lane & 31);
                fc[i] = *reinterpret_cast<const v4i *>(here + r * TILE_K + 16 * (chunk ^ swz<4>(r)));
            }
#pragma unroll
            for (int j = 0; j < TT; ++j) {
                const int r = wt + 32 * j + (lane & 31);
                ft[j] = *reinterpret_cast<const v4i *>(here + BN * TILE_K + r * TILE_K + 16 * (chunk ^ swz<4>(r)));
            }
#pragma unroll
            for (int i = 0; i < TC; ++i)
#pragma unroll
                for (int j = 0; j < TT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fc[i], ft[j], acc[i][j], 0, 0, 0);
        }
    }

#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const int64_t token = row0 + wt + 32 * j + (lane & 31);
        if (token >= g.m) continue;
        Scale a = {0.0f, 0};
        if (!PARTS) a = split_scale(g.sx[token]);
#pragma unroll
        for (int i = 0; i < TC; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t c = ch0 + wc + 32 * i + 8 * q + 4 * (lane >> 5);
                const int left = (int)(g.n - c < 4 ? g.n - c : 4);
                if (left <= 0) continue;
                if (PARTS) {
                    const int64_t wide = (g.n + 3) & ~int64_t(3);
                    *reinterpret_cast<int4 *>(g.sums + ((int64_t)part * g.m + token) * wide + c) =
                        make_int4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
                } else {
                    float y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t ce = c + (e < left ? e : 0);
                        y[e] = scaled(acc[i][j][4 * q + e], a, split_scale(g.sw[ce]));
                        if (g.out.bias) y[e] += g.out.bias[ce];
                    }
                    kv_store<4>(g.out.p, TYPE, token * g.out.ld + c, left, y);
                }
            }
    }
}

}  // namespace

hipError_t launch_encode_rows(const void *x, int64_t ldx, int type, int64_t n, int d, int8_t *codes, int64_t ld, float *scales, hipStream_t st)
{
    if (n == 0) return hipSuccess;
    const int units = (int)round_up(d, ROW_CODES_ALIGN) / 8;
    const auto go = [&](auto t) {
        constexpr int T = decltype(t)::value;
        if (units <= 64) encode_rows_kernel<T, 64, 1><<<dim3((unsigned)ceil_div(n, (int64_t)4)), ROW_THREADS, 0, st>>>(x, ldx, n, d, units, codes, ld, scales);
        else if (units <= 256) encode_rows_kernel<T, 256, 1><<<dim3((unsigned)n), ROW_THREADS, 0, st>>>(x, ldx, n, d, units, codes, ld, scales);
        else if (units <= 1024) encode_rows_kernel<T, 256, 4><<<dim3((unsigned)n), ROW_THREADS, 0, st>>>(x, ldx, n, d, units, codes, ld, scales);
        else encode_rows_kernel<T, 256, ROW_UNITS><<<dim3((unsigned)n), ROW_THREADS, 0, st>>>(x, ldx, n, d, units, codes, ld, scales);
    };
    if (type == LPQ_TYPE_F32) go(std::integral_constant<int, LPQ_TYPE_F32>());
    else if (type == LPQ_TYPE_F16) go(std::integral_constant<int, LPQ_TYPE_F16>());
    else go(std::integral_constant<int, LPQ_TYPE_BF16>());
    return hipGetLastError();
}

Linear8Plan linear8_plan(int64_t m, int64_t n, int d) { return {128, 128, 1, 0}; }

hipError_t launch_linear8(const RowCodes &x, const RowCodes &w, int d, const Linear8Out &out, const Linear8Plan &plan, void *workspace, hipStream_t st)
{
    const int stages = (int)ceil_div(d, TILE_K);
    const TileWork g = {x.codes, w.codes, x.scales, w.scales, x.ld, w.ld, x.n, w.n, stages, stages, (int)ceil_div(x.n, (int64_t)plan.rows),
                        (int)ceil_div(w.n, (int64_t)plan.channels), plan.parts, out, static_cast<int *>(workspace)};
    const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * plan.parts));
    if (out.type == LPQ_TYPE_F32) linear8_tile_kernel<2, 2, LPQ_TYPE_F32, false><<<grid, TILE_THREADS, 0, st>>>(g);
    else if (out.type == LPQ_TYPE_F16) linear8_tile_kernel<2, 2, LPQ_TYPE_F16, false><<<grid, TILE_THREADS, 0, st>>>(g);
    else linear8_tile_kernel<2, 2, LPQ_TYPE_BF16, false><<<grid, TILE_THREADS, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace lpq
