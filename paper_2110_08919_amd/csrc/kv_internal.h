// Declarations shared by the key-value cache kernels (kv_cache.hip, kv_select.hip, kv_attend.hip) and their C entry
// points (kv_api.hip).  gfx950 only.
#pragma once

#include "lpq_internal.h"

namespace lpq {

enum { KV_MAX_DIM = 256, KV_MIN_PAGE = 16, KV_MAX_PAGE = 256,
       KV_MAX_SELECT_ROWS = 128,      // query rows per key-value head whose summed codes fit two 7-bit digits
       KV_ATTEND_SHARES = 1024,       // most shares of an attention call, so most parts of a sequence: four workgroups per CU
       KV_MAX_BLOCKS = 1 << 22 };     // workgroups of a launch (twice that stays below 2^32 threads of 256 each)

// Constants of Equation 1 and the step s = 1 / m, five arrays of [heads][dpad] floats on the device.  Features without
// a range (S_e <= S_b) and padding hold S_b = -inf, S_e = inf, m = s = 0: they encode to 0 and read back as k (padding: 0).
struct KvConstants {
    const float *k, *sb, *se, *m, *s;
    int bits;
    bool clamps;       // clamping floor((x - k) m) to the codes' range makes the comparisons with S_b and S_e needless
};

// One layer's cache.  Codes [pages][heads][page][row_bytes], bounds [pages][heads][2][dpad] (smallest, largest key code).
struct KvView {
    uint8_t *k, *v;
    int8_t *bounds;
    KvConstants key, value;
    int64_t pages;
    int heads, dim, dpad, page, page_shift;
    bool packed;
};

// Rows [n][heads][dim] of a model's type, strides in elements.
struct KvRows {
    void *p;
    int64_t ld_token, ld_head;
    int type;
};

// Which rows belong to which sequence and where their pages are.
struct KvPlaces {
    const int32_t *first, *starts;   // starts null: one row per sequence
    const int32_t *table;
    int64_t ld_table, n;
    int nseq, table_pages;
};

struct KvQueries {
    const void *p;
    int64_t ld_seq, ld_token, ld_head;
    int type, new_tokens, group;     // group: query heads per key-value head
};

// *not_all becomes 1 unless KvConstants::clamps holds for all features.
hipError_t launch_kv_constants(const QuantParams &q, int heads, int dim, int dpad, bool packed, float *out, int *not_all, hipStream_t st);
hipError_t launch_kv_write(const KvView &kv, const KvRows &k, const KvRows &v, const KvPlaces &pl, hipStream_t st);
hipError_t launch_kv_read(const KvView &kv, const KvRows &k, const KvRows &v, const KvPlaces &pl, hipStream_t st);

struct KvSelect {
    const int32_t *lengths, *table;
    int64_t ld_table;
    int nseq, table_pages, n_select, keep_first, keep_last;
    int32_t *pages;                  // [nseq][heads][n_select]
    int32_t *scores;                 // workspace [nseq][heads][table_pages]
};
bool kv_select_needs_scores(int64_t table_pages);     // KvSelect::scores is used
hipError_t launch_kv_select(const KvView &kv, const KvQueries &q, const KvSelect &s, hipStream_t st);

struct KvAttend {
    const int32_t *lengths, *table;
    int64_t ld_table;
    int nseq, table_pages;
    const int32_t *chosen;           // null: all pages; else [nseq][heads][n_select]
    int n_select;
    float scale;
    void *out;
    int64_t ldo_seq, ldo_token, ldo_head;
    float *lse;                      // null or [nseq][new_tokens][heads * group]
    float *part;                     // workspace of kv_attend_plan
};
// How a call is shared out: `row_tiles` tiles of `rows` query rows cover a key-value head's; `grid` workgroups, as many
// of them per row tile as there are shares, take equal runs of all tiles of tokens, at least `least` each, or (least = 0) one (sequence,
// head, row tile) each.
struct KvAttendPlan {
    int row_tiles, rows, least;
    unsigned grid;
    size_t bytes;                    // of workspace
};
KvAttendPlan kv_attend_plan(const KvView &kv, int64_t nseq, int new_tokens, int group, int64_t tokens, int type);
hipError_t launch_kv_attend(const KvView &kv, const KvQueries &q, const KvAttend &a, const KvAttendPlan &plan, hipStream_t st);

#if defined(__HIPCC__)
// Memory that no kernel of the call writes, read at addresses all lanes share: scalar loads.
typedef const __attribute__((address_space(4))) int32_t *KvUniform;
__device__ __forceinline__ KvUniform kv_uniform(const int32_t *p) { return (KvUniform)(uintptr_t)p; }

// 8 consecutive features as they lie in memory: asked for by kv_load8, made floats by kv_floats8 once they are there.  Wide
// loads whatever the alignment (the hardware takes them at any address of its elements); the end of a row that is no multiple
// of 8, `left` < 8 features, comes in pieces of 4, 2 and 1 that kv_floats8 puts together.
struct Raw8 {
    uint32_t w[8];      // a 16-bit type: the first four
};
template <int BYTES>
__device__ __forceinline__ void kv_pieces(const char *p, int left, uint32_t *w)
{
    constexpr int W = BYTES;        // words of 4 features, for 2 or 4 bytes each
    if (left & 4) {
        uint32_t t[W];
        __builtin_memcpy(t, p, 4 * BYTES);
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = t[i];
    }
    if (left & 2) {
        uint32_t t[W / 2];
        __builtin_memcpy(t, p + (left & 4) * BYTES, 2 * BYTES);
#pragma unroll
        for (int i = 0; i < W / 2; ++i) w[W + i] = t[i];
    }
    if (left & 1) {
        if (BYTES == 2) w[3] = *reinterpret_cast<const uint16_t *>(p + (left & 6) * BYTES);
        else w[6] = *reinterpret_cast<const uint32_t *>(p + (left & 6) * BYTES);
    }
}
__device__ __forceinline__ Raw8 kv_load8(const void *base, int type, int64_t at, int left)
{
    Raw8 r = {{0, 0, 0, 0, 0, 0, 0, 0}};
    if (type == LPQ_TYPE_F32) {
        const char *p = static_cast<const char *>(base) + 4 * at;
        if (left >= 8) {
            uint4 a, b;
            __builtin_memcpy(&a, p, 16);
            __builtin_memcpy(&b, p + 16, 16);
            r = {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
        } else if (left > 0) {
            kv_pieces<4>(p, left, r.w);
        }
    } else {
        const char *p = static_cast<const char *>(base) + 2 * at;
        if (left >= 8) {
            uint4 a;
            __builtin_memcpy(&a, p, 16);
            r = {{a.x, a.y, a.z, a.w, 0, 0, 0, 0}};
        } else if (left > 0) {
            kv_pieces<2>(p, left, r.w);
        }
    }
    return r;
}
__device__ __forceinline__ void kv_floats8(const Raw8 &r, int type, int left, float *v)
{
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = r.w[e];
    if (left < 8) {      // what is not there was set to 0
        if (type == LPQ_TYPE_F32) {
            if (!(left & 2)) { w[4] = w[6]; w[6] = 0; }
            if (!(left & 4)) {
                w[0] = w[4]; w[1] = w[5]; w[2] = w[6];
                w[4] = w[5] = w[6] = 0;
            }
        } else {
            if (!(left & 2)) { w[2] = w[3]; w[3] = 0; }
            if (!(left & 4)) {
                w[0] = w[2]; w[1] = w[3];
                w[2] = w[3] = 0;
            }
        }
    }
    if (type == LPQ_TYPE_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __builtin_bit_cast(float, w[e]);
    } else if (type == LPQ_TYPE_BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __builtin_bit_cast(float, w[e] << 16);
            v[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = (float)__builtin_bit_cast(_Float16, (uint16_t)w[e]);
            v[2 * e + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[e] >> 16));
        }
    }
}
__device__ __forceinline__ void kv_load_floats8(const float *p, float *v)
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// 16-bit image of v in a 16-bit type, rounded to nearest even.
__device__ __forceinline__ uint16_t kv_to16(float v, int type)
{
    return type == LPQ_TYPE_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)v) : __builtin_bit_cast(uint16_t, (_Float16)v);
}

// N (4 or 8) consecutive features out; those at or past `left` are not written: what there is goes in pieces of 4, 2 and 1.
template <int N, typename T>
__device__ __forceinline__ void kv_store_pieces(T *p, int left, const T *v)
{
    if (left >= N) {
        __builtin_memcpy(p, v, sizeof(T) * N);
        return;
    }
    T w[4] = {v[0], v[1], v[2], v[3]};
    if (N == 8 && (left & 4)) {
        __builtin_memcpy(p, w, sizeof(T) * 4);
        p += 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = v[N - 4 + e];
    }
    if (left & 2) {
        __builtin_memcpy(p, w, sizeof(T) * 2);
        p += 2;
        w[0] = w[2];
    }
    if (left & 1) p[0] = w[0];
}
template <int N>
__device__ __forceinline__ void kv_store(void *base, int type, int64_t at, int left, const float *v)
{
    if (left <= 0) return;
    if (type == LPQ_TYPE_F32) {
        kv_store_pieces<N>(static_cast<float *>(base) + at, left, v);
        return;
    }
    uint16_t h[N];
#pragma unroll
    for (int e = 0; e < N; ++e) h[e] = kv_to16(v[e], type);
    kv_store_pieces<N>(static_cast<uint16_t *>(base) + at, left, h);
}
#endif

}  // namespace lpq
