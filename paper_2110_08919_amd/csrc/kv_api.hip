// C ABI of the key-value cache: argument checks, handle lifetime, workspace sizes.  No kernel lives here.
#include <algorithm>
#include <array>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <utility>

#include "kv_internal.h"

using namespace lpq;

struct lpq_kv {
    KvView view;
    float *constants = nullptr;    // device [2][5][heads * dpad]
};

static int kv_fail(int code, const char *fmt, ...)
{
    char message[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(message, sizeof(message), fmt, ap);
    va_end(ap);
    return set_error(code, message);
}

static int hip_fail(hipError_t e, const char *what)
{
    return kv_fail(e == hipErrorOutOfMemory ? LPQ_ENOMEM : LPQ_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

static int check_shape(int heads, int head_dim, int page, int64_t pages)
{
    if (heads < 1 || head_dim < 1) return kv_fail(LPQ_EINVAL, "heads = %d, features of a head = %d: both must be at least 1", heads, head_dim);
    if (head_dim > KV_MAX_DIM) return kv_fail(LPQ_ERANGE, "%d features of a head, at most %d", head_dim, (int)KV_MAX_DIM);
    if (page < KV_MIN_PAGE || page > KV_MAX_PAGE || (page & (page - 1)))
        return kv_fail(LPQ_EINVAL, "page = %d: 16, 32, 64, 128 or 256 tokens", page);
    if (pages < 1) return kv_fail(LPQ_EINVAL, "pages = %lld < 1", (long long)pages);
    if (pages >= (int64_t(1) << 31)) return kv_fail(LPQ_ERANGE, "pages = %lld, must stay below 2^31", (long long)pages);
    if (heads > MAX_D) return kv_fail(LPQ_ERANGE, "heads = %d > %d", heads, (int)MAX_D);
    return LPQ_OK;
}

static int padded_features(int head_dim) { return (int)round_up(head_dim, 64); }

extern "C" int lpq_kv_storage_bytes(int heads, int head_dim, int page, int64_t pages, int packed, size_t *codes, size_t *bounds,
                                    int *row_features)
{
    const int rc = check_shape(heads, head_dim, page, pages);
    if (rc) return rc;
    const size_t dpad = (size_t)padded_features(head_dim), per = (size_t)pages * heads;
    if (codes) *codes = per * page * dpad / (packed ? 2 : 1);
    if (bounds) *bounds = per * 2 * dpad;
    if (row_features) *row_features = (int)dpad;
    return LPQ_OK;
}

extern "C" void lpq_kv_destroy(lpq_kv *kv)
{
    if (!kv) return;
    (void)hipFree(kv->constants);
    delete kv;
}

extern "C" int lpq_kv_create(lpq_kv **out, const lpq_quantizer *keys, const lpq_quantizer *values, int heads, int page,
                             int64_t pages, int packed, void *k_dev, void *v_dev, void *bounds_dev)
{
    if (!out || !keys || !values || !k_dev || !v_dev || !bounds_dev) return kv_fail(LPQ_EINVAL, "null argument");
    QuantParams qp[2];
    const bool keys_ready = quantizer_constants(keys, &qp[0]), values_ready = quantizer_constants(values, &qp[1]);
    if (heads < 1 || qp[0].d != qp[1].d || qp[0].d % heads)
        return kv_fail(LPQ_EINVAL, "quantizers of %d and %d features for %d heads", qp[0].d, qp[1].d, heads);
    const int rc = check_shape(heads, qp[0].d / heads, page, pages);
    if (rc) return rc;
    if (packed && (qp[0].bits > 4 || qp[1].bits > 4)) return kv_fail(LPQ_EINVAL, "packed storage needs quantizers of at most 4 bits");
    if (((uintptr_t)k_dev | (uintptr_t)v_dev | (uintptr_t)bounds_dev) % 256) return kv_fail(LPQ_EINVAL, "storage must be 256-byte aligned");
    if (!keys_ready || !values_ready) return kv_fail(LPQ_ESTATE, "quantizer has no constants yet");
    lpq_kv *kv = new (std::nothrow) lpq_kv;
    if (!kv) return kv_fail(LPQ_ENOMEM, "host allocation failed");
    KvView &v = kv->view;
    v.k = static_cast<uint8_t *>(k_dev);
    v.v = static_cast<uint8_t *>(v_dev);
    v.bounds = static_cast<int8_t *>(bounds_dev);
    v.pages = pages;
    v.heads = heads;
    v.dim = qp[0].d / heads;
    v.dpad = padded_features(v.dim);
    v.page = page;
    v.page_shift = __builtin_ctz(page);
    v.packed = packed != 0;
    const size_t each = (size_t)heads * v.dpad;
    hipError_t e = hipMalloc(&kv->constants, (2 * 5 * each + 2) * sizeof(float));
    int *flags_dev = reinterpret_cast<int *>(kv->constants + 2 * 5 * each), flags[2] = {0, 0};
    if (e == hipSuccess) e = hipMemset(flags_dev, 0, sizeof(flags));
    for (int i = 0; i < 2 && e == hipSuccess; ++i)
        e = launch_kv_constants(qp[i], heads, v.dim, v.dpad, v.packed, kv->constants + (size_t)i * 5 * each, flags_dev + i, nullptr);
    if (e == hipSuccess) e = hipMemcpy(flags, flags_dev, sizeof(flags), hipMemcpyDeviceToHost);
    for (int i = 0; i < 2; ++i) {
        const float *p = kv->constants + (size_t)i * 5 * each;
        (i ? v.value : v.key) = {p, p + each, p + 2 * each, p + 3 * each, p + 4 * each, qp[i].bits, flags[i] == 0};
    }
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
        lpq_kv_destroy(kv);
        return hip_fail(e, "constants of the cache");
    }
    *out = kv;
    return LPQ_OK;
}

// Sizes that every call shares.
static int check_places(const lpq_kv *kv, int64_t nseq, const int32_t *table_dev, int64_t ld_table, int64_t table_pages)
{
    if (nseq < 0 || table_pages < 1 || ld_table < table_pages)
        return kv_fail(LPQ_EINVAL, "nseq = %lld, table of %lld columns %lld apart", (long long)nseq, (long long)table_pages, (long long)ld_table);
    if (nseq > 0 && !table_dev) return kv_fail(LPQ_EINVAL, "null table");
    if (table_pages > INT32_MAX / kv->view.page) return kv_fail(LPQ_ERANGE, "table_pages * page = %lld * %d", (long long)table_pages, kv->view.page);
    if (nseq > KV_MAX_BLOCKS / kv->view.heads) return kv_fail(LPQ_ERANGE, "nseq * heads = %lld * %d", (long long)nseq, kv->view.heads);
    return LPQ_OK;
}

static int element_bytes(int type) { return type == LPQ_TYPE_F32 ? 4 : type == LPQ_TYPE_F16 || type == LPQ_TYPE_BF16 ? 2 : 0; }

constexpr int64_t MAX_STRIDE = int64_t(1) << 40;

// Whether runs of `dim` elements, three axes of them, lie apart from each other, whichever axis is the outer one.
static bool disjoint(int64_t dim, std::array<std::pair<int64_t, int64_t>, 3> axes)    // (stride, size)
{
    std::sort(axes.begin(), axes.end());
    int64_t extent = dim;
    for (const auto &a : axes) {
        if (a.second <= 1) continue;
        if (a.first < extent) return false;
        extent += (a.second - 1) * a.first;
    }
    return true;
}

static int kv_rows(const lpq_kv *kv, const void *k, int64_t ldk_token, int64_t ldk_head, const void *v, int64_t ldv_token,
                   int64_t ldv_head, int type, int64_t n, int64_t nseq, const int32_t *first, const int32_t *starts,
                   const int32_t *table, int64_t ld_table, int64_t table_pages, bool written, KvRows *kr, KvRows *vr, KvPlaces *pl)
{
    if (!kv) return kv_fail(LPQ_EINVAL, "null argument");
    if (n < 0) return kv_fail(LPQ_EINVAL, "n < 0");
    if (!element_bytes(type)) return kv_fail(LPQ_EINVAL, "unknown type %d", type);
    const int rc = check_places(kv, nseq, table, ld_table, table_pages);
    if (rc) return rc;
    if (n > 0 && nseq > 0 && (!k || !v || !first)) return kv_fail(LPQ_EINVAL, "null argument");
    if (!starts && n != nseq) return kv_fail(LPQ_EINVAL, "n = %lld rows for %lld sequences without starts", (long long)n, (long long)nseq);
    if (n > 0 && nseq == 0) return kv_fail(LPQ_EINVAL, "n = %lld rows, but no sequence", (long long)n);
    if (n >= (int64_t(1) << 31)) return kv_fail(LPQ_ERANGE, "n = %lld, must stay below 2^31", (long long)n);
    const int64_t dim = kv->view.dim, heads = kv->view.heads;
    int64_t strides[2][2] = {{ldk_token, ldk_head}, {ldv_token, ldv_head}};
    for (auto &s : strides) {
        if (s[0] < 0 || s[1] < 0 || s[0] > MAX_STRIDE || s[1] > MAX_STRIDE)
            return kv_fail(LPQ_EINVAL, "strides %lld, %lld", (long long)s[0], (long long)s[1]);
        if (n <= 1) s[0] = 0;              // the stride of one row means nothing
        if (heads == 1) s[1] = 0;
        if (!written) continue;            // rows that are only read may overlap
        if (n > 0 && !disjoint(dim, {{{s[0], n}, {s[1], heads}, {0, 1}}}))
            return kv_fail(LPQ_EINVAL, "strides %lld, %lld of rows [n][heads][%lld] overlap", (long long)s[0], (long long)s[1], (long long)dim);
    }
    *kr = {const_cast<void *>(k), strides[0][0], strides[0][1], type};
    *vr = {const_cast<void *>(v), strides[1][0], strides[1][1], type};
    *pl = {first, starts, table, ld_table, n, (int)nseq, (int)table_pages};
    return LPQ_OK;
}

extern "C" int lpq_kv_write(const lpq_kv *kv, const void *k_dev, int64_t ldk_token, int64_t ldk_head, const void *v_dev,
                            int64_t ldv_token, int64_t ldv_head, int type, int64_t n, int64_t nseq,
                            const int32_t *first_dev, const int32_t *starts_dev, const int32_t *table_dev,
                            int64_t ld_table, int64_t table_pages, void *stream)
{
    KvRows kr, vr;
    KvPlaces pl;
    const int rc = kv_rows(kv, k_dev, ldk_token, ldk_head, v_dev, ldv_token, ldv_head, type, n, nseq, first_dev, starts_dev,
                           table_dev, ld_table, table_pages, false, &kr, &vr, &pl);
    if (rc) return rc;
    const hipError_t e = launch_kv_write(kv->view, kr, vr, pl, (hipStream_t)stream);
    return e == hipSuccess ? LPQ_OK : hip_fail(e, "lpq_kv_write");
}

extern "C" int lpq_kv_write_rotated(const lpq_kv *kv, const void *k_dev, int64_t ldk_token, int64_t ldk_head, const void *v_dev,
                                    int64_t ldv_token, int64_t ldv_head, int type, int64_t n, int64_t nseq,
                                    const int32_t *first_dev, const int32_t *starts_dev, const int32_t *table_dev,
                                    int64_t ld_table, int64_t table_pages, const float *cos_dev, const float *sin_dev,
                                    int64_t ld_angles, int64_t angles, int rotated, int interleaved, const int32_t *positions_dev,
                                    const void *q_dev, int64_t ldq_token, int64_t ldq_head, int q_heads, void *out_dev,
                                    int64_t ldo_token, int64_t ldo_head, void *stream)
{
    KvRows kr, vr;
    KvPlaces pl;
    const int rc = kv_rows(kv, k_dev, ldk_token, ldk_head, v_dev, ldv_token, ldv_head, type, n, nseq, first_dev, starts_dev,
                           table_dev, ld_table, table_pages, false, &kr, &vr, &pl);
    if (rc) return rc;
    const int dim = kv->view.dim;
    if (rotated < 2 || rotated % 2 || rotated > dim) return kv_fail(LPQ_EINVAL, "rotated = %d of %d features: an even number from 2 on", rotated, dim);
    if (n > 0 && (!cos_dev || !sin_dev)) return kv_fail(LPQ_EINVAL, "null argument");
    if (angles < 1 || ld_angles < rotated / 2 || ld_angles > MAX_STRIDE)
        return kv_fail(LPQ_EINVAL, "angles of %lld positions, %lld apart", (long long)angles, (long long)ld_angles);
    if (angles > INT32_MAX) return kv_fail(LPQ_ERANGE, "angles of %lld positions", (long long)angles);
    KvAngles a = {cos_dev, sin_dev, ld_angles, angles, positions_dev, rotated / 2, interleaved != 0, {nullptr, 0, 0, type}, {nullptr, 0, 0, type}, 0};
    if (q_dev && n > 0) {
        if (q_heads < kv->view.heads || q_heads % kv->view.heads)
            return kv_fail(LPQ_EINVAL, "%d query heads on %d key-value heads", q_heads, kv->view.heads);
        if (q_heads > 65536) return kv_fail(LPQ_ERANGE, "%d query heads", q_heads);
        if (!out_dev) return kv_fail(LPQ_EINVAL, "null output");
        int64_t strides[2][2] = {{ldq_token, ldq_head}, {ldo_token, ldo_head}};
        for (auto &s : strides) {
            if (s[0] < 0 || s[1] < 0 || s[0] > MAX_STRIDE || s[1] > MAX_STRIDE)
                return kv_fail(LPQ_EINVAL, "strides %lld, %lld of queries", (long long)s[0], (long long)s[1]);
            if (n <= 1) s[0] = 0;
            if (q_heads == 1) s[1] = 0;
        }
        if (!disjoint(dim, {{{strides[1][0], n}, {strides[1][1], q_heads}, {0, 1}}}))
            return kv_fail(LPQ_EINVAL, "strides %lld, %lld of the output overlap", (long long)ldo_token, (long long)ldo_head);
        // keys and values are read beside queries that are written
        if (out_dev == k_dev || out_dev == v_dev) return kv_fail(LPQ_EINVAL, "turned queries in the place of keys or values");
        if (out_dev == q_dev && (strides[0][0] != strides[1][0] || strides[0][1] != strides[1][1]))
            return kv_fail(LPQ_EINVAL, "queries turned in place with other strides");
        a.q = {const_cast<void *>(q_dev), strides[0][0], strides[0][1], type};
        a.out = {out_dev, strides[1][0], strides[1][1], type};
        a.q_heads = q_heads;
    }
    const hipError_t e = launch_kv_write_rotated(kv->view, kr, vr, pl, a, (hipStream_t)stream);
    return e == hipSuccess ? LPQ_OK : hip_fail(e, "lpq_kv_write_rotated");
}

extern "C" int lpq_kv_read(const lpq_kv *kv, void *k_dev, int64_t ldk_token, int64_t ldk_head, void *v_dev,
                           int64_t ldv_token, int64_t ldv_head, int type, int64_t n, int64_t nseq,
                           const int32_t *first_dev, const int32_t *starts_dev, const int32_t *table_dev,
                           int64_t ld_table, int64_t table_pages, void *stream)
{
    KvRows kr, vr;
    KvPlaces pl;
    const int rc = kv_rows(kv, k_dev, ldk_token, ldk_head, v_dev, ldv_token, ldv_head, type, n, nseq, first_dev, starts_dev,
                           table_dev, ld_table, table_pages, true, &kr, &vr, &pl);
    if (rc) return rc;
    const hipError_t e = launch_kv_read(kv->view, kr, vr, pl, (hipStream_t)stream);
    return e == hipSuccess ? LPQ_OK : hip_fail(e, "lpq_kv_read");
}

// Queries and sizes of select and attend.
static int kv_queries(const lpq_kv *kv, const void *q, int64_t ld_seq, int64_t ld_token, int64_t ld_head, int type, int64_t nseq,
                      int new_tokens, int q_heads, const int32_t *lengths, const int32_t *table, int64_t ld_table,
                      int64_t table_pages, KvQueries *out)
{
    if (!kv) return kv_fail(LPQ_EINVAL, "null argument");
    if (!element_bytes(type)) return kv_fail(LPQ_EINVAL, "unknown type %d", type);
    const int heads = kv->view.heads;
    if (new_tokens < 1 || q_heads < heads || q_heads % heads)
        return kv_fail(LPQ_EINVAL, "new_tokens = %d, %d query heads on %d key-value heads", new_tokens, q_heads, heads);
    const int rc = check_places(kv, nseq, table, ld_table, table_pages);
    if (rc) return rc;
    if (nseq > 0 && (!q || !lengths)) return kv_fail(LPQ_EINVAL, "null argument");
    if ((int64_t)new_tokens * q_heads > 65536 || nseq * new_tokens * q_heads > KV_MAX_BLOCKS)
        return kv_fail(LPQ_ERANGE, "%lld sequences of %d new tokens and %d query heads", (long long)nseq, new_tokens, q_heads);
    if (ld_seq < 0 || ld_token < 0 || ld_head < 0 || ld_seq > MAX_STRIDE || ld_token > MAX_STRIDE || ld_head > MAX_STRIDE)
        return kv_fail(LPQ_EINVAL, "strides %lld, %lld, %lld of the queries", (long long)ld_seq, (long long)ld_token, (long long)ld_head);
    if (nseq <= 1) ld_seq = 0;             // a stride over one element means nothing
    if (new_tokens == 1) ld_token = 0;
    if (q_heads == 1) ld_head = 0;
    *out = {q, ld_seq, ld_token, ld_head, type, new_tokens, q_heads / heads};
    return LPQ_OK;
}

extern "C" size_t lpq_kv_select_workspace_bytes(const lpq_kv *kv, int64_t nseq, int64_t table_pages)
{
    if (!kv || nseq < 0 || table_pages < 1 || !kv_select_needs_scores(table_pages)) return 0;
    return (size_t)nseq * kv->view.heads * table_pages * sizeof(int32_t);
}

extern "C" int lpq_kv_select(const lpq_kv *kv, const void *q_dev, int64_t ldq_seq, int64_t ldq_token, int64_t ldq_head,
                             int type, int64_t nseq, int new_tokens, int q_heads, const int32_t *lengths_dev,
                             const int32_t *table_dev, int64_t ld_table, int64_t table_pages, int n_select,
                             int keep_first, int keep_last, int32_t *pages_dev, void *workspace_dev,
                             size_t workspace_bytes, void *stream)
{
    KvQueries q;
    const int rc = kv_queries(kv, q_dev, ldq_seq, ldq_token, ldq_head, type, nseq, new_tokens, q_heads, lengths_dev, table_dev,
                              ld_table, table_pages, &q);
    if (rc) return rc;
    if (n_select < 1 || keep_first < 0 || keep_last < 0 || (int64_t)keep_first + keep_last > n_select)
        return kv_fail(LPQ_EINVAL, "n_select = %d, keep_first = %d, keep_last = %d", n_select, keep_first, keep_last);
    if (nseq > 0 && !pages_dev) return kv_fail(LPQ_EINVAL, "null output");
    if (new_tokens * q.group > KV_MAX_SELECT_ROWS)
        return kv_fail(LPQ_ERANGE, "%d query rows per key-value head, at most %d", new_tokens * q.group, (int)KV_MAX_SELECT_ROWS);
    const int64_t per = ceil_div(table_pages, (int64_t)64);
    if (nseq * kv->view.heads * per > KV_MAX_BLOCKS) return kv_fail(LPQ_ERANGE, "nseq * heads * table_pages too large");
    const size_t need = lpq_kv_select_workspace_bytes(kv, nseq, table_pages);
    if (need && (!workspace_dev || (uintptr_t)workspace_dev % 256)) return kv_fail(LPQ_EINVAL, "workspace null or not 256-byte aligned");
    if (workspace_bytes < need) return kv_fail(LPQ_ERANGE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    const KvSelect s = {lengths_dev, table_dev, ld_table, (int)nseq, (int)table_pages, n_select, keep_first, keep_last, pages_dev,
                        static_cast<int32_t *>(workspace_dev)};
    const hipError_t e = launch_kv_select(kv->view, q, s, (hipStream_t)stream);
    return e == hipSuccess ? LPQ_OK : hip_fail(e, "lpq_kv_select");
}

// A window that no sequence outgrows is none.
static int window_of(const lpq_kv *kv, int64_t table_pages, int64_t window) { return window >= table_pages * kv->view.page ? 0 : (int)window; }

// The plan of a call; chosen pages are all gone through, whatever the window.
static KvAttendPlan attend_plan(const lpq_kv *kv, int64_t nseq, int new_tokens, int group, int64_t pages, bool chosen, int type, KvMask mask)
{
    const int64_t tokens = pages * kv->view.page;
    if (chosen && mask.window) mask.window = (int)std::min<int64_t>(tokens, INT32_MAX);
    return kv_attend_plan(kv->view, nseq, new_tokens, group, tokens, type, mask);
}

static size_t attend_bytes(const lpq_kv *kv, int64_t nseq, int new_tokens, int q_heads, int64_t table_pages, int n_select, const KvMask &mask)
{
    if (!kv || nseq < 1 || new_tokens < 1 || q_heads < kv->view.heads || q_heads % kv->view.heads || table_pages < 1 || n_select < 0) return 0;
    // enough for queries of any type
    size_t most = 0;
    for (const int type : {LPQ_TYPE_F32, LPQ_TYPE_F16, LPQ_TYPE_BF16})
        most = std::max(most, attend_plan(kv, nseq, new_tokens, q_heads / kv->view.heads, n_select ? n_select : table_pages, n_select > 0, type, mask).bytes);
    return most;
}

extern "C" size_t lpq_kv_attend_workspace_bytes(const lpq_kv *kv, int64_t nseq, int new_tokens, int q_heads, int64_t table_pages,
                                                int n_select)
{
    return attend_bytes(kv, nseq, new_tokens, q_heads, table_pages, n_select, {0, 0, nullptr, 0, 0});
}

extern "C" size_t lpq_kv_attend_masked_workspace_bytes(const lpq_kv *kv, int64_t nseq, int new_tokens, int q_heads, int64_t table_pages,
                                                       int n_select, int64_t window, int sinks, int tree)
{
    if (!kv || table_pages < 1 || table_pages > INT32_MAX / kv->view.page || window < 0 || sinks < 0) return 0;
    static const uint8_t some = 0;
    return attend_bytes(kv, nseq, new_tokens, q_heads, table_pages, n_select, {window_of(kv, table_pages, window), sinks, tree ? &some : nullptr, 0, 0});
}

static int attend(const lpq_kv *kv, const void *q_dev, int64_t ldq_seq, int64_t ldq_token, int64_t ldq_head, int type, int64_t nseq, int new_tokens,
                  int q_heads, float scale, const int32_t *lengths_dev, const int32_t *table_dev, int64_t ld_table, int64_t table_pages,
                  const int32_t *chosen_dev, int n_select, const KvMask &mask, void *out_dev, int64_t ldo_seq, int64_t ldo_token, int64_t ldo_head,
                  float *lse_dev, void *workspace_dev, size_t workspace_bytes, void *stream, const char *name)
{
    KvQueries q;
    const int rc = kv_queries(kv, q_dev, ldq_seq, ldq_token, ldq_head, type, nseq, new_tokens, q_heads, lengths_dev, table_dev,
                              ld_table, table_pages, &q);
    if (rc) return rc;
    if (nseq > 0 && !out_dev) return kv_fail(LPQ_EINVAL, "null output");
    if (!std::isfinite(scale)) return kv_fail(LPQ_EINVAL, "scale is not finite");
    if (chosen_dev && n_select < 1) return kv_fail(LPQ_EINVAL, "n_select = %d < 1", n_select);
    if (chosen_dev && n_select > INT32_MAX / kv->view.page) return kv_fail(LPQ_ERANGE, "n_select * page = %d * %d", n_select, kv->view.page);
    const int64_t dim = kv->view.dim;
    if (ldo_seq < 0 || ldo_token < 0 || ldo_head < 0 || ldo_seq > MAX_STRIDE || ldo_token > MAX_STRIDE || ldo_head > MAX_STRIDE) return kv_fail(LPQ_EINVAL, "strides of the output");
    if (nseq <= 1) ldo_seq = 0;
    if (new_tokens == 1) ldo_token = 0;
    if (q_heads == 1) ldo_head = 0;
    if (!disjoint(dim, {{{ldo_seq, nseq}, {ldo_token, new_tokens}, {ldo_head, q_heads}}}))
        return kv_fail(LPQ_EINVAL, "strides %lld, %lld, %lld of the output overlap", (long long)ldo_seq, (long long)ldo_token, (long long)ldo_head);
    const KvAttendPlan plan = attend_plan(kv, nseq, new_tokens, q.group, chosen_dev ? n_select : table_pages, chosen_dev != nullptr, type, mask);
    if (plan.bytes && (!workspace_dev || (uintptr_t)workspace_dev % 256)) return kv_fail(LPQ_EINVAL, "workspace null or not 256-byte aligned");
    if (workspace_bytes < plan.bytes) return kv_fail(LPQ_ERANGE, "workspace of %zu bytes, %zu needed", workspace_bytes, plan.bytes);
    const KvAttend a = {lengths_dev, table_dev, ld_table, (int)nseq, (int)table_pages, chosen_dev, n_select, scale, out_dev, ldo_seq,
                        ldo_token, ldo_head, lse_dev, static_cast<float *>(workspace_dev)};
    const hipError_t e = launch_kv_attend(kv->view, q, a, mask, plan, (hipStream_t)stream);
    return e == hipSuccess ? LPQ_OK : hip_fail(e, name);
}

extern "C" int lpq_kv_attend(const lpq_kv *kv, const void *q_dev, int64_t ldq_seq, int64_t ldq_token, int64_t ldq_head,
                             int type, int64_t nseq, int new_tokens, int q_heads, float scale,
                             const int32_t *lengths_dev, const int32_t *table_dev, int64_t ld_table, int64_t table_pages,
                             const int32_t *chosen_dev, int n_select, void *out_dev, int64_t ldo_seq, int64_t ldo_token,
                             int64_t ldo_head, float *lse_dev, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    return attend(kv, q_dev, ldq_seq, ldq_token, ldq_head, type, nseq, new_tokens, q_heads, scale, lengths_dev, table_dev, ld_table, table_pages,
                  chosen_dev, n_select, {0, 0, nullptr, 0, 0}, out_dev, ldo_seq, ldo_token, ldo_head, lse_dev, workspace_dev, workspace_bytes, stream,
                  "lpq_kv_attend");
}

extern "C" int lpq_kv_attend_masked(const lpq_kv *kv, const void *q_dev, int64_t ldq_seq, int64_t ldq_token, int64_t ldq_head,
                                    int type, int64_t nseq, int new_tokens, int q_heads, float scale,
                                    const int32_t *lengths_dev, const int32_t *table_dev, int64_t ld_table, int64_t table_pages,
                                    const int32_t *chosen_dev, int n_select, int64_t window, int sinks, const uint8_t *tree_dev,
                                    int64_t ldt_seq, int64_t ldt_token, void *out_dev, int64_t ldo_seq, int64_t ldo_token,
                                    int64_t ldo_head, float *lse_dev, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    if (!kv) return kv_fail(LPQ_EINVAL, "null argument");
    if (window < 0 || sinks < 0) return kv_fail(LPQ_EINVAL, "window = %lld, sinks = %d: neither may be below 0", (long long)window, sinks);
    if (sinks > 0 && window == 0) return kv_fail(LPQ_EINVAL, "%d sinks without a window", sinks);
    if (tree_dev && window > 0) return kv_fail(LPQ_EINVAL, "a window and a tree: the positions of drafted tokens are not known");
    if (tree_dev) {
        if (new_tokens > KV_MAX_TREE) return kv_fail(LPQ_ERANGE, "a tree of %d new tokens, at most %d", new_tokens, (int)KV_MAX_TREE);
        if (ldt_seq < 0 || ldt_token < 0 || ldt_seq > MAX_STRIDE || ldt_token > MAX_STRIDE)
            return kv_fail(LPQ_EINVAL, "strides %lld, %lld of the tree", (long long)ldt_seq, (long long)ldt_token);
        if (nseq <= 1) ldt_seq = 0;            // a stride over one element means nothing
        if (new_tokens == 1) ldt_token = 0;
    }
    const int rc = check_places(kv, nseq, table_dev, ld_table, table_pages);      // before the window is compared with the table
    if (rc) return rc;
    const int within = window_of(kv, table_pages, window);
    return attend(kv, q_dev, ldq_seq, ldq_token, ldq_head, type, nseq, new_tokens, q_heads, scale, lengths_dev, table_dev, ld_table, table_pages,
                  chosen_dev, n_select, {within, sinks, tree_dev, ldt_seq, ldt_token}, out_dev, ldo_seq, ldo_token, ldo_head, lse_dev, workspace_dev,
                  workspace_bytes, stream, "lpq_kv_attend_masked");
}
