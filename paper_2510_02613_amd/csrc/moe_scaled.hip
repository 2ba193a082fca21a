// Host side of the operators of the 8-bit path: argument checking and launches.  The layer with 8-bit experts is in moe_api.hip.
#include <cstdarg>

#include "scaled.h"

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

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

constexpr int32_t kMaxRows = 1 << 21;     // rows of a call: grids stay inside the launch limits
constexpr int64_t kMaxStride = 1 << 23;   // bytes from one 8-bit row to the next, and scales: a tile's rows are addressed with 32 bits

moe_status_t check_dtype(int32_t dtype, const char *what)
{
    if (dtype != MOE_F32 && dtype != MOE_BF16) return fail(MOE_ERR_ARG, "%s %d is not a moe_dtype_t", what, dtype);
    return MOE_OK;
}
// a matrix of bf16 or fp32 rows: 16-byte rows, or with odd widths allowed 16-byte row starts
moe_status_t check_rows(const void *p, int64_t ld, int32_t cols, int32_t dtype, const char *what)
{
    const int64_t step = dtype == MOE_BF16 ? 8 : 4;
    if (!aligned(p, 16)) return fail(MOE_ERR_ARG, "%s must be 16-byte aligned", what);
    if (ld < cols || ld % step) return fail(MOE_ERR_ARG, "ld of %s, %lld, must be %d at least and a multiple of %d (16-byte rows)", what, (long long)ld, cols, (int)step);
    return MOE_OK;
}
moe_status_t check_scales(const float *p, int64_t ld, int32_t blocks, const char *what)
{
    if (!aligned(p, 4)) return fail(MOE_ERR_ARG, "%s must be 4-byte aligned", what);
    if (ld < blocks) return fail(MOE_ERR_ARG, "ld of %s, %lld, must be %d at least", what, (long long)ld, blocks);
    return MOE_OK;
}
moe_status_t check_8bit_out(const void *q, int64_t ld_q, const float *scale, int64_t ld_scale, int32_t cols)
{
    if (!aligned(q, 8) || ld_q < cols || ld_q % 8) return fail(MOE_ERR_ARG, "q must be 8-byte aligned, its ld (%lld) %d at least and a multiple of 8", (long long)ld_q, cols);
    return check_scales(scale, ld_scale, scale_blocks(cols), "the scales");
}
moe_status_t check_row_shape(int32_t rows, int32_t cols)
{
    if (rows < 0 || cols <= 0) return fail(MOE_ERR_SHAPE, "rows %d must not be negative and cols %d positive", rows, cols);
    if (cols % 8) return fail(MOE_ERR_UNSUPPORTED, "cols must be a multiple of 8 (16-byte rows)");
    if (rows > kMaxRows) return fail(MOE_ERR_UNSUPPORTED, "rows > %d", kMaxRows);
    return MOE_OK;
}

// what the two products share: [m,k] 8-bit rows times [n,k] 8-bit weights
moe_status_t check_product(int32_t m, int32_t n, int32_t k, const void *a, int64_t ld_a, const float *a_scale, int64_t ld_a_scale, const void *w, const float *w_scale)
{
    if (m < 0 || n <= 0 || k <= 0) return fail(MOE_ERR_SHAPE, "m %d must not be negative, n %d and k %d positive", m, n, k);
    if (k % 16) return fail(MOE_ERR_UNSUPPORTED, "k must be a multiple of 16 (16-byte rows)");
    if (m > kMaxRows || n > kMaxRows) return fail(MOE_ERR_UNSUPPORTED, "m or n > %d", kMaxRows);
    if (ld_a >= kMaxStride || k >= kMaxStride) return fail(MOE_ERR_UNSUPPORTED, "rows of a or w are %d bytes long or longer", (int)kMaxStride);
    if (!w || !w_scale) return fail(MOE_ERR_ARG, "w and w_scale must be non-NULL");
    if (!aligned(w, 16) || !aligned(w_scale, 4)) return fail(MOE_ERR_ARG, "w must be 16-byte and w_scale 4-byte aligned");
    if (m == 0) return MOE_OK;
    if (!a || !a_scale) return fail(MOE_ERR_ARG, "a and a_scale must be non-NULL");
    if (!aligned(a, 16) || ld_a < k || ld_a % 16) return fail(MOE_ERR_ARG, "a must be 16-byte aligned, its ld (%lld) %d at least and a multiple of 16", (long long)ld_a, k);
    if (ld_a_scale >= kMaxStride / 4) return fail(MOE_ERR_UNSUPPORTED, "ld of a_scale is %d or larger", (int)(kMaxStride / 4));
    return check_scales(a_scale, ld_a_scale, scale_blocks(k), "a_scale");
}

// How a product of m rows is run: the streaming kernels, or tiles of tile_rows rows; its workgroups.
struct Plan { bool stream; int tile_rows; long long groups; };
constexpr long long kMaxGroups = (1ll << 32) / 512 - 512;   // workgroups of 512 threads that a launch can have, less those that a last round is shared out to

// The faster by what both were measured to take (us).  Streaming: 3 + 0.28 per 32 rows and million weights, with swiglu 7 (a second launch quantises) and
// 0.24: 4096 x 7168 64 rows 19.3 (fast tiles 34.9), 128 rows 38 (fast 34.9), 333 rows 89 (exact 55, fast 36); 7168 x 2048 64 rows 12.8 (fast 13.5), 128 rows
// 20 (fast 13.7), 333 rows 46 (exact 23, fast 16); 1544 x 1424 in fp32 333 rows 8.9 (19.1), 1000 rows 20 (20.1); swiglu 2048 x 7168 128 rows 39 (60), 333 rows 75 (60.7), 1408 x 2048 128 rows 15 (21.2), 333 rows 21.9 (21.3).
Plan plan_product(int32_t m, int32_t n, int32_t k, bool swiglu, bool exact)
{
    const double weights = (swiglu ? 2e-6 : 1e-6) * n * k;
    double best = (swiglu ? 7.0 + 0.24 * weights * ((m + 31) / 32) : 3.0 + 0.28 * weights * ((m + 31) / 32));
    Plan p = {true, stream_tile_rows(m, n, swiglu), 0};
    p.groups = (m + p.tile_rows - 1ll) / p.tile_rows * ((n + 15) / 16);      // at most
    const int most = exact ? 128 : 256;
    for (int rows : {32, 64, 128, 192, 256}) {
        if (rows > most) break;
        const long long tiles = (m + rows - 1) / rows;
        const double us = tiles_us(tiles, rows, n, k, swiglu, exact);
        if (us < best) { best = us; p = {false, rows, tiles * tiles_slices(n, swiglu)}; }
    }
    return p;
}

SGemm product(int32_t m, int32_t n, int32_t k, const void *a, int64_t ld_a, const float *a_scale, int64_t ld_a_scale, const void *w, const float *w_scale)
{
    SGemm g = {};
    g.a = (const uint8_t *)a; g.as = a_scale; g.ld_a = ld_a; g.ld_as = ld_a_scale;
    g.w = (const uint8_t *)w; g.ws = w_scale;
    g.m = m; g.n = n; g.k = k; g.kb = scale_blocks(k);
    g.together = 4;
    return g;
}

#define EMOE_TRY(call) { const moe_status_t st_ = (call); if (st_ != MOE_OK) return st_; }

}  // namespace

extern "C" {

moe_status_t moe_rms_norm(const moe_rms_norm_t *n, void *hip_stream)
{
    if (!n) return fail(MOE_ERR_ARG, "arguments are NULL");
    EMOE_TRY(check_dtype(n->dtype, "dtype"));
    EMOE_TRY(check_row_shape(n->rows, n->cols));
    if (n->cols > kMaxRowCols) return fail(MOE_ERR_UNSUPPORTED, "cols > %d", kMaxRowCols);
    if (!(n->eps >= 0.f) || n->eps > 3.4028235e38f) return fail(MOE_ERR_ARG, "eps must be finite and not negative");
    if (n->rows == 0) return MOE_OK;
    if (!n->sum && !n->out && !n->q) return fail(MOE_ERR_ARG, "no output: sum, out and q are NULL");
    if ((n->q != nullptr) != (n->q_scale != nullptr)) return fail(MOE_ERR_ARG, "q and q_scale must be given together");
    if (n->sum && !n->residual) return fail(MOE_ERR_ARG, "sum without a residual");
    if (!n->x) return fail(MOE_ERR_ARG, "x is NULL");
    EMOE_TRY(check_rows(n->x, n->ld_x, n->cols, n->dtype, "x"));
    if (n->residual) EMOE_TRY(check_rows(n->residual, n->ld_residual, n->cols, n->dtype, "residual"));
    if (n->weight && !aligned(n->weight, 16)) return fail(MOE_ERR_ARG, "weight must be 16-byte aligned");
    if (n->sum) EMOE_TRY(check_rows(n->sum, n->ld_sum, n->cols, n->dtype, "sum"));
    if (n->out) EMOE_TRY(check_rows(n->out, n->ld_out, n->cols, n->dtype, "out"));
    if (n->q) EMOE_TRY(check_8bit_out(n->q, n->ld_q, n->q_scale, n->ld_scale, n->cols));
    RowsJob j = {};
    j.rows = n->rows; j.cols = n->cols; j.norm = 1; j.eps = n->eps;
    j.x = n->x; j.residual = n->residual; j.weight = n->weight; j.sum = n->sum; j.out = n->out;
    j.q = (uint8_t *)n->q; j.scale = n->q_scale;
    j.ld_x = n->ld_x; j.ld_residual = n->ld_residual; j.ld_sum = n->ld_sum; j.ld_out = n->ld_out; j.ld_q = n->ld_q; j.ld_scale = n->ld_scale;
    const hipError_t e = launch_rows(j, n->dtype == MOE_BF16, (hipStream_t)hip_stream);
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "norm launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

moe_status_t moe_quantize(const moe_quantize_t *n, void *hip_stream)
{
    if (!n) return fail(MOE_ERR_ARG, "arguments are NULL");
    EMOE_TRY(check_dtype(n->dtype, "dtype"));
    EMOE_TRY(check_row_shape(n->rows, n->cols));
    if (n->block_rows != 1 && n->block_rows != kScaleBlock) return fail(MOE_ERR_ARG, "block_rows %d is neither 1 nor %d", n->block_rows, kScaleBlock);
    if (n->block_rows == 1 && n->cols > kMaxRowCols) return fail(MOE_ERR_UNSUPPORTED, "cols > %d", kMaxRowCols);
    if (n->cols > kMaxRows) return fail(MOE_ERR_UNSUPPORTED, "cols > %d", kMaxRows);
    if (n->rows == 0) return MOE_OK;
    if (!n->x || !n->q || !n->scale) return fail(MOE_ERR_ARG, "x, q and scale must be non-NULL");
    EMOE_TRY(check_rows(n->x, n->ld_x, n->cols, n->dtype, "x"));
    EMOE_TRY(check_8bit_out(n->q, n->ld_q, n->scale, n->ld_scale, n->cols));
    RowsJob j = {};
    j.rows = n->rows; j.cols = n->cols;
    j.x = n->x; j.ld_x = n->ld_x;
    j.q = (uint8_t *)n->q; j.scale = n->scale; j.ld_q = n->ld_q; j.ld_scale = n->ld_scale;
    const bool bf16 = n->dtype == MOE_BF16;
    const hipError_t e = n->block_rows == 1 ? launch_rows(j, bf16, (hipStream_t)hip_stream) : launch_quantize_blocks(j, bf16, (hipStream_t)hip_stream);
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "quantise launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

moe_status_t moe_scaled_matmul(const moe_scaled_matmul_t *p, void *hip_stream)
{
    if (!p) return fail(MOE_ERR_ARG, "arguments are NULL");
    const bool fast = (p->out_dtype & MOE_FAST_PRODUCTS) != 0;
    const int32_t dtype = p->out_dtype & ~MOE_FAST_PRODUCTS;
    EMOE_TRY(check_dtype(dtype, "out_dtype"));
    if (fast && dtype != MOE_BF16) return fail(MOE_ERR_UNSUPPORTED, "MOE_FAST_PRODUCTS is for bf16 results");
    EMOE_TRY(check_product(p->m, p->n, p->k, p->a, p->ld_a, p->a_scale, p->ld_a_scale, p->w, p->w_scale));
    if (p->m == 0) return MOE_OK;
    if (!p->out) return fail(MOE_ERR_ARG, "out is NULL");
    EMOE_TRY(check_rows(p->out, p->ld_out, p->n, dtype, "out"));
    if (p->add) EMOE_TRY(check_rows(p->add, p->ld_add, p->n, dtype, "add"));
    SGemm g = product(p->m, p->n, p->k, p->a, p->ld_a, p->a_scale, p->ld_a_scale, p->w, p->w_scale);
    g.out = p->out; g.ld_out = p->ld_out; g.add = p->add; g.ld_add = p->ld_add;
    const bool bf16 = dtype == MOE_BF16;
    const Plan plan = plan_product(g.m, g.n, g.k, false, !fast);
    if (plan.groups > kMaxGroups) return fail(MOE_ERR_UNSUPPORTED, "a result of %d x %d needs more workgroups than a launch can have", g.m, g.n);
    g.split_tail = plan.tile_rows > 64;
    const hipError_t e = plan.stream ? launch_scaled_stream(g, false, bf16, plan.tile_rows, (hipStream_t)hip_stream)
                                     : launch_scaled_tiles(g, fast ? TilesOut::fast_bf16 : bf16 ? TilesOut::bf16 : TilesOut::f32, plan.tile_rows, (hipStream_t)hip_stream);
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "product launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

size_t moe_scaled_swiglu_workspace_bytes(int32_t m, int32_t inter, int32_t k)
{
    if (m <= 0 || inter <= 0 || k <= 0 || m > kMaxRows || inter > kMaxRows || !plan_product(m, inter, k, true, true).stream) return 0;
    return ((size_t)m * inter * 4 + 255) / 256 * 256;
}

size_t moe_scaled_swiglu_max_workspace_bytes(int32_t max_m, int32_t inter, int32_t k)
{
    if (max_m <= 0 || inter <= 0 || k <= 0 || max_m > kMaxRows || inter > kMaxRows) return 0;
    // the most rows that are streamed: which form runs is the same for all m with as many parts of 32 rows
    for (int32_t parts = (max_m + 31) / 32; parts > 0; --parts) {
        const size_t bytes = moe_scaled_swiglu_workspace_bytes(parts * 32 < max_m ? parts * 32 : max_m, inter, k);
        if (bytes) return bytes;
    }
    return 0;
}

moe_status_t moe_scaled_swiglu(const moe_scaled_swiglu_t *p, void *hip_stream)
{
    if (!p) return fail(MOE_ERR_ARG, "arguments are NULL");
    EMOE_TRY(check_product(p->m, p->inter, p->k, p->a, p->ld_a, p->a_scale, p->ld_a_scale, p->w, p->w_scale));
    if (p->inter % 16) return fail(MOE_ERR_UNSUPPORTED, "inter must be a multiple of 16 (16-byte rows)");
    if (p->inter > kMaxRowCols) return fail(MOE_ERR_UNSUPPORTED, "inter > %d", kMaxRowCols);
    if (p->m == 0) return MOE_OK;
    if (!p->q || !p->q_scale) return fail(MOE_ERR_ARG, "q and q_scale must be non-NULL");
    EMOE_TRY(check_8bit_out(p->q, p->ld_q, p->q_scale, p->ld_scale, p->inter));
    const size_t need = moe_scaled_swiglu_workspace_bytes(p->m, p->inter, p->k);
    if (need && (!p->workspace || !aligned(p->workspace, 256))) return fail(MOE_ERR_ARG, "workspace must be non-NULL and 256-byte aligned");
    if (p->workspace_bytes < need) return fail(MOE_ERR_CAPACITY, "workspace has %zu bytes, the product needs %zu", p->workspace_bytes, need);
    SGemm g = product(p->m, p->inter, p->k, p->a, p->ld_a, p->a_scale, p->ld_a_scale, p->w, p->w_scale);
    const Plan plan = plan_product(g.m, g.n, g.k, true, true);
    if (plan.groups > kMaxGroups) return fail(MOE_ERR_UNSUPPORTED, "a result of %d x %d needs more workgroups than a launch can have", g.m, g.n);
    hipError_t e = hipSuccess;
    if (!plan.stream) {
        g.q = (uint8_t *)p->q; g.qs = p->q_scale; g.ld_q = p->ld_q; g.ld_qs = p->ld_scale;
        g.split_tail = plan.tile_rows > 64;
        e = launch_scaled_tiles(g, TilesOut::swiglu_exact, plan.tile_rows, (hipStream_t)hip_stream);
    } else {
        g.out = p->workspace; g.ld_out = p->inter;
        e = launch_scaled_stream(g, true, false, plan.tile_rows, (hipStream_t)hip_stream);
    }
    if (e == hipSuccess && plan.stream) {
        RowsJob j = {};
        j.rows = p->m; j.cols = p->inter;
        j.x = p->workspace; j.ld_x = p->inter;
        j.q = (uint8_t *)p->q; j.scale = p->q_scale; j.ld_q = p->ld_q; j.ld_scale = p->ld_scale;
        e = launch_rows(j, false, (hipStream_t)hip_stream);
    }
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "product launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

}  // extern "C"
