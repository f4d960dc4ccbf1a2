// C ABI of linear layers on 8-bit codes: argument checks and workspace sizes.  No kernel lives here.
#include <cstdarg>
#include <cstdio>

#include "linear8_internal.h"

using namespace lpq;

static int fail(int code, const char *fmt, ...)
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
    return fail(e == hipErrorOutOfMemory ? LPQ_ENOMEM : LPQ_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

static int element_bytes(int type) { return type == LPQ_TYPE_F32 ? 4 : type == LPQ_TYPE_F16 || type == LPQ_TYPE_BF16 ? 2 : 0; }

constexpr int64_t MAX_STRIDE = int64_t(1) << 40;

extern "C" size_t lpq_row_codes_bytes(int64_t n, int d)
{
    return n < 0 || n > LINEAR8_MAX_ROWS || d < 1 || d > LINEAR8_MAX_D ? 0 : (size_t)ceil_div(n, (int64_t)16) * row_blocks(d) * 1024;
}

static int check_features(int d)
{
    if (d < 1) return fail(LPQ_EINVAL, "d = %d < 1", d);
    if (d > LINEAR8_MAX_D) return fail(LPQ_ERANGE, "d = %d, at most %d: a sum of products of codes must fit 32 bits", d, (int)LINEAR8_MAX_D);
    return LPQ_OK;
}

// Rows that are only read may overlap.
static int check_rows(const char *what, const void *p, int64_t ld, int type, int64_t n, int64_t d, bool written)
{
    if (n < 0) return fail(LPQ_EINVAL, "%lld %s", (long long)n, what);
    if (n > LINEAR8_MAX_ROWS) return fail(LPQ_ERANGE, "%lld %s, at most %d", (long long)n, what, (int)LINEAR8_MAX_ROWS);
    if (!element_bytes(type)) return fail(LPQ_EINVAL, "unknown type %d", type);
    if (n > 0 && !p) return fail(LPQ_EINVAL, "null %s", what);
    if (ld < (written && n > 1 ? d : 0) || ld > MAX_STRIDE) return fail(LPQ_EINVAL, "%s of %lld elements, %lld apart", what, (long long)d, (long long)ld);
    return LPQ_OK;
}

static int check_codes(const char *what, const void *codes, const float *scales, int64_t n)
{
    if (n < 0) return fail(LPQ_EINVAL, "%lld %s", (long long)n, what);
    if (n > LINEAR8_MAX_ROWS) return fail(LPQ_ERANGE, "%lld %s, at most %d", (long long)n, what, (int)LINEAR8_MAX_ROWS);
    if (n > 0 && (!codes || !scales)) return fail(LPQ_EINVAL, "null %s", what);
    if ((uintptr_t)codes % 256) return fail(LPQ_EINVAL, "%s must be 256-byte aligned", what);
    return LPQ_OK;
}

extern "C" int lpq_encode_rows(const void *x_dev, int64_t ldx, int type, int64_t n, int d, int8_t *codes_dev, float *scales_dev, void *stream)
{
    int rc = check_features(d);
    if (!rc) rc = check_rows("rows", x_dev, ldx, type, n, d, false);
    if (!rc) rc = check_codes("codes", codes_dev, scales_dev, n);
    if (rc) return rc;
    const hipError_t e = launch_encode_rows(x_dev, ldx, type, n, d, codes_dev, scales_dev, (hipStream_t)stream);
    return e == hipSuccess ? LPQ_OK : hip_fail(e, "lpq_encode_rows");
}

// Sizes whose tiles one launch can cover.
static int check_product(int64_t m, int64_t n)
{
    if (ceil_div(m, (int64_t)128) * ceil_div(n, (int64_t)128) > (1 << 22)) return fail(LPQ_ERANGE, "%lld rows times %lld channels", (long long)m, (long long)n);
    return LPQ_OK;
}

extern "C" size_t lpq_matmul_i8_workspace_bytes(int64_t m, int64_t n, int d)
{
    if (m < 1 || n < 1 || m > LINEAR8_MAX_ROWS || n > LINEAR8_MAX_ROWS || d < 1 || d > LINEAR8_MAX_D) return 0;
    return linear8_plan(m, n, d).bytes;
}

static int check_workspace(const void *workspace_dev, size_t bytes, size_t need)
{
    if (need && (!workspace_dev || (uintptr_t)workspace_dev % 256)) return fail(LPQ_EINVAL, "workspace null or not 256-byte aligned");
    if (bytes < need) return fail(LPQ_ERANGE, "workspace of %zu bytes, %zu needed", bytes, need);
    return LPQ_OK;
}

extern "C" int lpq_matmul_i8(const int8_t *a_dev, const float *a_scales_dev, int64_t m, const int8_t *b_dev, const float *b_scales_dev, int64_t n, int d,
                             const float *bias_dev, void *out_dev, int64_t ldo, int type, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    int rc = check_features(d);
    if (!rc) rc = check_codes("rows", a_dev, a_scales_dev, m);
    if (!rc) rc = check_codes("channels", b_dev, b_scales_dev, n);
    if (!rc) rc = check_rows("outputs", out_dev, ldo, type, n > 0 ? m : 0, n, true);
    if (!rc) rc = check_product(m, n);
    if (!rc && m > 0 && n > 0) rc = check_workspace(workspace_dev, workspace_bytes, lpq_matmul_i8_workspace_bytes(m, n, d));
    if (rc || m == 0 || n == 0) return rc;
    const hipError_t e = launch_linear8({a_dev, a_scales_dev, m}, {b_dev, b_scales_dev, n}, d, {out_dev, ldo, type, bias_dev},
                                        linear8_plan(m, n, d), workspace_dev, (hipStream_t)stream);
    return e == hipSuccess ? LPQ_OK : hip_fail(e, "lpq_matmul_i8");
}

// Workspace of lpq_linear8: the rows' codes, their scales, then what the product needs.
struct Linear8Space {
    size_t scales, parts, bytes;
};
static Linear8Space linear8_space(int64_t m, int64_t n, int d)
{
    if (linear8_fused(m, d)) return {0, 0, 0};
    Linear8Space s;
    s.scales = lpq_row_codes_bytes(m, d);
    s.parts = (size_t)round_up(s.scales + 4 * m, 256);
    s.bytes = s.parts + lpq_matmul_i8_workspace_bytes(m, n, d);
    return s;
}

extern "C" size_t lpq_linear8_workspace_bytes(int64_t m, int64_t n, int d)
{
    if (m < 1 || n < 1 || m > LINEAR8_MAX_ROWS || n > LINEAR8_MAX_ROWS || d < 1 || d > LINEAR8_MAX_D) return 0;
    return linear8_space(m, n, d).bytes;
}

extern "C" int lpq_linear8(const void *x_dev, int64_t ldx, int type, int64_t m, const int8_t *codes_dev, const float *scales_dev, int64_t n,
                           int d, const float *bias_dev, void *out_dev, int64_t ldo, void *workspace_dev, size_t workspace_bytes,
                           void *stream)
{
    int rc = check_features(d);
    if (!rc) rc = check_rows("rows", x_dev, ldx, type, m, d, false);
    if (!rc) rc = check_codes("channels", codes_dev, scales_dev, n);
    if (!rc) rc = check_rows("outputs", out_dev, ldo, type, n > 0 ? m : 0, n, true);
    if (!rc) rc = check_product(m, n);
    if (rc || m == 0 || n == 0) return rc;
    const Linear8Space s = linear8_space(m, n, d);
    rc = check_workspace(workspace_dev, workspace_bytes, s.bytes);
    if (rc) return rc;
    const Linear8Out out = {out_dev, ldo, type, bias_dev};
    const RowCodes weights = {codes_dev, scales_dev, n};
    if (linear8_fused(m, d)) {
        const hipError_t e = launch_linear8_fused(x_dev, ldx, m, weights, d, out, (hipStream_t)stream);
        return e == hipSuccess ? LPQ_OK : hip_fail(e, "lpq_linear8");
    }
    char *const space = static_cast<char *>(workspace_dev);
    int8_t *const rows = reinterpret_cast<int8_t *>(space);
    float *const row_scales = reinterpret_cast<float *>(space + s.scales);
    hipError_t e = launch_encode_rows(x_dev, ldx, type, m, d, rows, row_scales, (hipStream_t)stream);
    if (e == hipSuccess)
        e = launch_linear8({rows, row_scales, m}, weights, d, out, linear8_plan(m, n, d), space + s.parts, (hipStream_t)stream);
    return e == hipSuccess ? LPQ_OK : hip_fail(e, "lpq_linear8");
}

extern "C" int lpq_linear8_plan_info(int64_t m, int64_t n, int d, int64_t *out, int out_count)
{
    if (!out || out_count < LPQ_LINEAR8_INFO_COUNT) return fail(LPQ_EINVAL, "out must hold LPQ_LINEAR8_INFO_COUNT values");
    int rc = check_features(d);
    if (!rc && (m < 1 || n < 1)) rc = fail(LPQ_EINVAL, "%lld rows, %lld channels", (long long)m, (long long)n);
    if (!rc && (m > LINEAR8_MAX_ROWS || n > LINEAR8_MAX_ROWS)) rc = fail(LPQ_ERANGE, "%lld rows, %lld channels", (long long)m, (long long)n);
    if (!rc) rc = check_product(m, n);
    if (rc) return rc;
    const Linear8Plan p = linear8_plan(m, n, d);
    out[0] = p.rows;
    out[1] = p.channels;
    out[2] = p.parts;
    out[3] = linear8_fused(m, d);
    return LPQ_OK;
}
