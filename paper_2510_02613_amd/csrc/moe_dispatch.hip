// Host side of the operators that sort tokens by expert and add them up again: argument checking and launches.
#include <cstdarg>

#include "dispatch.h"

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

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

moe_status_t check_shape(int32_t tokens, int32_t top_k, int32_t cols, int32_t dtype)
{
    if (dtype != MOE_F32 && dtype != MOE_BF16) return fail(MOE_ERR_ARG, "dtype %d is not a moe_dtype_t", dtype);
    if (tokens < 0 || top_k <= 0 || cols <= 0) return fail(MOE_ERR_SHAPE, "tokens %d must not be negative, top_k %d and cols %d positive", tokens, top_k, cols);
    if (cols % 8) return fail(MOE_ERR_UNSUPPORTED, "cols must be a multiple of 8 (16-byte rows)");
    if (tokens > kMost || cols > kMost) return fail(MOE_ERR_UNSUPPORTED, "tokens or cols > %d", kMost);
    if (top_k > kDispatchMaxK) return fail(MOE_ERR_UNSUPPORTED, "top_k > %d", kDispatchMaxK);
    return MOE_OK;
}
moe_status_t check_rows(const void *p, int64_t ld, int32_t cols, int32_t dtype, const char *what)
{
    const int64_t step = dtype == MOE_BF16 ? 8 : 4;
    if (!p) return fail(MOE_ERR_ARG, "%s is NULL", what);
    if (!aligned(p, 16)) return fail(MOE_ERR_ARG, "%s must be 16-byte aligned", what);
    if (ld < cols || ld % step) return fail(MOE_ERR_ARG, "ld of %s, %lld, must be %d at least and a multiple of %d (16-byte rows)", what, (long long)ld, cols, (int)step);
    if (ld > (int64_t)1 << 40) return fail(MOE_ERR_UNSUPPORTED, "ld of %s > 2^40", what);
    return MOE_OK;
}
moe_status_t check_words(const void *p, const char *what)
{
    if (!p) return fail(MOE_ERR_ARG, "%s is NULL", what);
    if (!aligned(p, 4)) return fail(MOE_ERR_ARG, "%s must be 4-byte aligned", what);
    return MOE_OK;
}

}  // namespace

extern "C" {

size_t moe_sort_tokens_workspace_bytes(int32_t tokens, int32_t top_k, int32_t n_groups)
{
    if (tokens < 0 || tokens > kMost || top_k <= 0 || top_k > kDispatchMaxK || n_groups <= 0 || n_groups > kDispatchMaxGroups) return 0;
    return (size_t)sort_blocks(tokens, top_k) * (n_groups + 1) * sizeof(int32_t);
}

moe_status_t moe_sort_tokens(const moe_sort_tokens_t *n, void *hip_stream)
{
    if (!n) return fail(MOE_ERR_ARG, "arguments are NULL");
    EMOE_TRY(check_shape(n->tokens, n->top_k, n->cols, n->dtype));
    if (n->n_groups <= 0) return fail(MOE_ERR_SHAPE, "n_groups %d must be positive", n->n_groups);
    if (n->n_groups > kDispatchMaxGroups) return fail(MOE_ERR_UNSUPPORTED, "n_groups > %d", kDispatchMaxGroups);
    EMOE_TRY(check_words(n->offsets, "offsets"));
    if (n->expert_map) {
        if (n->n_experts <= 0) return fail(MOE_ERR_SHAPE, "n_experts %d must be positive with an expert_map", n->n_experts);
        EMOE_TRY(check_words(n->expert_map, "expert_map"));
    }
    SortJob j = {};
    if (n->tokens > 0) {
        EMOE_TRY(check_words(n->ids, "ids"));
        EMOE_TRY(check_words(n->source, "source"));
        EMOE_TRY(check_words(n->row, "row"));
        EMOE_TRY(check_rows(n->x, n->ld_x, n->cols, n->dtype, "x"));
        EMOE_TRY(check_rows(n->rows, n->ld_rows, n->cols, n->dtype, "rows"));
        const size_t need = moe_sort_tokens_workspace_bytes(n->tokens, n->top_k, n->n_groups);
        if (need) {
            if (!n->workspace || !aligned(n->workspace, 16)) return fail(MOE_ERR_ARG, "a 16-byte aligned workspace is needed");
            if (n->workspace_bytes < need) return fail(MOE_ERR_CAPACITY, "the workspace has %zu bytes, %zu are needed", n->workspace_bytes, need);
        }
        const int64_t es = n->dtype == MOE_BF16 ? 2 : 4;
        j.x = (const char *)n->x; j.rows = (char *)n->rows;
        j.ld_x = n->ld_x * es; j.ld_rows = n->ld_rows * es;
        j.chunks = (int32_t)(n->cols * es / 16);
        j.counts = (int32_t *)n->workspace;
    }
    j.tokens = n->tokens; j.top_k = n->top_k; j.n_groups = n->n_groups; j.n_experts = n->n_experts; j.zero_rest = n->zero_rest != 0;
    j.ids = n->ids; j.map = n->expert_map;
    j.offsets = n->offsets; j.source = n->source; j.row = n->row;
    const hipError_t e = launch_sort_tokens(j, (hipStream_t)hip_stream);
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "sort launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

moe_status_t moe_combine_tokens(const moe_combine_tokens_t *n, void *hip_stream)
{
    if (!n) return fail(MOE_ERR_ARG, "arguments are NULL");
    EMOE_TRY(check_shape(n->tokens, n->top_k, n->cols, n->dtype));
    if (n->tokens == 0) return MOE_OK;
    EMOE_TRY(check_rows(n->y, n->ld_y, n->cols, n->dtype, "y"));
    EMOE_TRY(check_words(n->row, "row"));
    if (n->weights) EMOE_TRY(check_words(n->weights, "weights"));
    EMOE_TRY(check_rows(n->out, n->ld_out, n->cols, n->dtype, "out"));
    const int64_t es = n->dtype == MOE_BF16 ? 2 : 4;
    CombineJob j = {};
    j.tokens = n->tokens; j.top_k = n->top_k; j.chunks = (int32_t)(n->cols * es / 16);
    j.y = (const char *)n->y; j.ld_y = n->ld_y * es;
    j.row = n->row; j.weights = n->weights;
    j.out = (char *)n->out; j.ld_out = n->ld_out * es;
    const hipError_t e = launch_combine_tokens(j, n->dtype == MOE_BF16, (hipStream_t)hip_stream);
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "combine launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

moe_status_t moe_combine_tokens_backward(const moe_combine_tokens_backward_t *n, void *hip_stream)
{
    if (!n) return fail(MOE_ERR_ARG, "arguments are NULL");
    EMOE_TRY(check_shape(n->tokens, n->top_k, n->cols, n->dtype));
    if (n->tokens == 0) return MOE_OK;
    if (!n->grad_y && !n->grad_weights) return fail(MOE_ERR_ARG, "no output: grad_y and grad_weights are NULL");
    EMOE_TRY(check_rows(n->grad_out, n->ld_grad_out, n->cols, n->dtype, "grad_out"));
    EMOE_TRY(check_words(n->row, "row"));
    if (n->weights) EMOE_TRY(check_words(n->weights, "weights"));
    const int64_t es = n->dtype == MOE_BF16 ? 2 : 4;
    CombineJob j = {};
    if (n->grad_y) {
        EMOE_TRY(check_rows(n->grad_y, n->ld_grad_y, n->cols, n->dtype, "grad_y"));
        if (n->source) EMOE_TRY(check_words(n->source, "source"));
        j.grad_y = (char *)n->grad_y; j.ld_grad_y = n->ld_grad_y * es; j.source = n->source;
    }
    if (n->grad_weights) {
        EMOE_TRY(check_words(n->grad_weights, "grad_weights"));
        EMOE_TRY(check_rows(n->y, n->ld_y, n->cols, n->dtype, "y"));
        j.grad_weights = n->grad_weights; j.y = (const char *)n->y; j.ld_y = n->ld_y * es;
    }
    j.tokens = n->tokens; j.top_k = n->top_k; j.chunks = (int32_t)(n->cols * es / 16);
    j.grad_out = (const char *)n->grad_out; j.ld_grad_out = n->ld_grad_out * es;
    j.row = n->row; j.weights = n->weights;
    const hipError_t e = launch_combine_tokens_backward(j, n->dtype == MOE_BF16, (hipStream_t)hip_stream);
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "combine backward launch failed: %s", hipGetErrorString(e));
    return MOE_OK;
}

}  // extern "C"
