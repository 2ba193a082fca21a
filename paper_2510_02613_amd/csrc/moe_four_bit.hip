// Host side of the 4-bit operators: argument checking and launches.
#include <cstdarg>

#include "four_bit.h"

using namespace emoe;

namespace emoe {
moe_status_t set_error(moe_status_t st, const char *fmt, va_list ap);
}

namespace {

moe_status_t fail(moe_status_t st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    set_error(st, fmt, ap);
    va_end(ap);
    return st;
}

#define EMOE_TRY(call) { const moe_status_t st_ = (call); if (st_ != MOE_OK) return st_; }

constexpr int32_t kMost = 1 << 21;
constexpr int32_t kMaxGroups = 2047;            // as many as a layer has slots
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int64_t kMaxRowStride = 1 << 24;      // of the rows of a: a tile of them is addressed with 32 bits

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

moe_status_t check_dtype(int32_t dtype, const char *what)
{
    if (dtype != MOE_F32 && dtype != MOE_BF16) return fail(MOE_ERR_ARG, "%s %d is not a moe_dtype_t", what, dtype);
    return MOE_OK;
}
moe_status_t check_rows(const void *p, int64_t ld, int32_t cols, int32_t dtype, const char *what)
{
    const int64_t step = dtype == MOE_BF16 ? 8 : 4;
    if (!p) return fail(MOE_ERR_ARG, "%s is NULL", what);
    if (!aligned(p, 16)) return fail(MOE_ERR_ARG, "%s must be 16-byte aligned", what);
    if (ld < cols || ld % step) return fail(MOE_ERR_ARG, "ld of %s, %lld, must be %d at least and a multiple of %d (16-byte rows)", what, (long long)ld, cols, (int)step);
    if (ld > kMaxStride) return fail(MOE_ERR_UNSUPPORTED, "ld of %s > 2^40", what);
    return MOE_OK;
}

// what the two products share; cols: of the result, w_rows: of a group's weights
moe_status_t check_product(int32_t m, int32_t cols, int32_t w_rows, int32_t k, int32_t groups, int32_t out_dtype, const void *a, int64_t ld_a, const int32_t *offsets,
                           const void *w, const void *w_scale, const void *out, int64_t ld_out)
{
    EMOE_TRY(check_dtype(out_dtype, "out_dtype"));
    if (m < 0 || cols <= 0 || k <= 0 || groups <= 0) return fail(MOE_ERR_SHAPE, "m %d must not be negative, columns %d, k %d and groups %d positive", m, cols, k, groups);
    if (k % kFourGroup) return fail(MOE_ERR_UNSUPPORTED, "k must be a multiple of %d (the columns that share a power of two)", kFourGroup);
    if (m > kMost || w_rows > kMost || k > kMost) return fail(MOE_ERR_UNSUPPORTED, "m, k or the rows of w > %d", kMost);
    if (groups > kMaxGroups) return fail(MOE_ERR_UNSUPPORTED, "groups > %d", kMaxGroups);
    if (!offsets && groups != 1) return fail(MOE_ERR_ARG, "%d groups without offsets", groups);
    if (!w || !w_scale) return fail(MOE_ERR_ARG, "w and w_scale must be non-NULL");
    if (!aligned(w, 16)) return fail(MOE_ERR_ARG, "w must be 16-byte aligned");
    if (!aligned(offsets, 4)) return fail(MOE_ERR_ARG, "offsets must be 4-byte aligned");
    if (m == 0) return MOE_OK;
    EMOE_TRY(check_rows(a, ld_a, k, MOE_BF16, "a"));
    if (ld_a >= kMaxRowStride) return fail(MOE_ERR_UNSUPPORTED, "ld of a is %d or larger", (int)kMaxRowStride);
    return check_rows(out, ld_out, cols, out_dtype, "out");
}

}  // namespace

extern "C" {

moe_status_t moe_four_bit_quantize(const moe_four_bit_quantize_t *n, void *hip_stream)
{
    if (!n) return fail(MOE_ERR_ARG, "arguments are NULL");
    EMOE_TRY(check_dtype(n->dtype, "dtype"));
    if (n->rows < 0 || n->cols <= 0) return fail(MOE_ERR_SHAPE, "rows %d must not be negative and cols %d positive", n->rows, n->cols);
    if (n->cols % kFourGroup) return fail(MOE_ERR_UNSUPPORTED, "cols must be a multiple of %d (the columns that share a power of two)", kFourGroup);
    if (n->rows > kMost || n->cols > kMost) return fail(MOE_ERR_UNSUPPORTED, "rows or cols > %d", kMost);
    if (n->rows == 0) return MOE_OK;
    EMOE_TRY(check_rows(n->x, n->ld_x, n->cols, n->dtype, "x"));
    if (!n->q || !n->scale) return fail(MOE_ERR_ARG, "q and scale must be non-NULL");
    if (!aligned(n->q, 4) || n->ld_q < n->cols / 2 || n->ld_q % 4) return fail(MOE_ERR_ARG, "q must be 4-byte aligned, its ld (%lld) %d at least and a multiple of 4", (long long)n->ld_q, n->cols / 2);
    if (n->ld_scale < n->cols / kFourGroup) return fail(MOE_ERR_ARG, "ld of scale, %lld, must be %d at least", (long long)n->ld_scale, n->cols / kFourGroup);
    if (n->ld_q > kMaxStride || n->ld_scale > kMaxStride) return fail(MOE_ERR_UNSUPPORTED, "ld of q or scale > 2^40");
    if (n->values) EMOE_TRY(check_rows(n->values, n->ld_values, n->cols, n->dtype, "values"));
    const int64_t es = n->dtype == MOE_BF16 ? 2 : 4;
    FourRows j = {};
    j.rows = n->rows; j.cols = n->cols;
    j.x = (const char *)n->x; j.ld_x = n->ld_x * es;
    j.q = (uint8_t *)n->q; j.ld_q = n->ld_q; j.scale = (uint8_t *)n->scale; j.ld_scale = n->ld_scale;
    j.values = (char *)n->values; j.ld_values = n->ld_values * es;
    const hipError_t e = launch_four_quantize(j, n->dtype == MOE_BF16, (hipStream_t)hip_stream);
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "quantise launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

moe_status_t moe_four_bit_matmul(const moe_four_bit_matmul_t *p, void *hip_stream)
{
    if (!p) return fail(MOE_ERR_ARG, "arguments are NULL");
    EMOE_TRY(check_product(p->m, p->n, p->n, p->k, p->groups, p->out_dtype, p->a, p->ld_a, p->offsets, p->w, p->w_scale, p->out, p->ld_out));
    if (p->m == 0) return MOE_OK;
    if (p->add) EMOE_TRY(check_rows(p->add, p->ld_add, p->n, p->out_dtype, "add"));
    FourGemm g = {};
    g.a = (const uint16_t *)p->a; g.ld_a = p->ld_a; g.w = (const uint8_t *)p->w; g.ws = (const uint8_t *)p->w_scale;
    g.m = p->m; g.n = p->n; g.k = p->k; g.groups = p->groups; g.offsets = p->offsets; g.sparse = p->groups > 2 * p->m;
    g.add = p->add; g.ld_add = p->ld_add; g.out = p->out; g.ld_out = p->ld_out;
    if (!four_product_fits(g)) return fail(MOE_ERR_UNSUPPORTED, "n * groups: more tiles than a launch can have workgroups");
    const hipError_t e = launch_four_matmul(g, p->out_dtype == MOE_BF16, (hipStream_t)hip_stream);
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "product launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

moe_status_t moe_four_bit_swiglu(const moe_four_bit_swiglu_t *p, void *hip_stream)
{
    if (!p) return fail(MOE_ERR_ARG, "arguments are NULL");
    if (p->inter > kMost / 2) return fail(MOE_ERR_UNSUPPORTED, "inter > %d", kMost / 2);
    EMOE_TRY(check_product(p->m, p->inter, 2 * p->inter, p->k, p->groups, p->out_dtype, p->a, p->ld_a, p->offsets, p->w, p->w_scale, p->out, p->ld_out));
    if (p->m == 0) return MOE_OK;
    FourGemm g = {};
    g.a = (const uint16_t *)p->a; g.ld_a = p->ld_a; g.w = (const uint8_t *)p->w; g.ws = (const uint8_t *)p->w_scale;
    g.m = p->m; g.n = p->inter; g.k = p->k; g.groups = p->groups; g.offsets = p->offsets; g.sparse = p->groups > 2 * p->m;
    g.out = p->out; g.ld_out = p->ld_out;
    if (!four_product_fits(g)) return fail(MOE_ERR_UNSUPPORTED, "inter * groups: more tiles than a launch can have workgroups");
    const hipError_t e = launch_four_swiglu(g, p->out_dtype == MOE_BF16, (hipStream_t)hip_stream);
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "product launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

}  // extern "C"
