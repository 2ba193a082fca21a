/*
 * elasticmoe_dispatch.h -- tokens sorted by expert and back, as operators of their own, with their gradients: for callers whose expert
 * products are not the layer's (moe_four_bit_matmul of elasticmoe_four_bit.h, a library's products, adapters).  Entry points, statuses,
 * memory and error rules are those of elasticmoe.h.
 */
#ifndef ELASTICMOE_DISPATCH_H
#define ELASTICMOE_DISPATCH_H

#include "elasticmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Token t has top_k assignments, numbered a = t * top_k + j; assignment a belongs to group
 *     g = expert_map[ids[t, j]]   (expert_map NULL: g = ids[t, j]).
 * An id outside [0, n_experts) or a group outside [0, n_groups) is an assignment that is not this rank's.  The others are given rows, ordered by
 * group and inside a group by assignment (an id may occur twice in a token):
 *     offsets[g] .. offsets[g + 1] - 1  the rows of group g,  offsets[n_groups] of them in all,
 *     source[r]                         the assignment of row r, -1 behind the last row,
 *     row[t, j]                         the row of the assignment, -1 where it has none.
 * Every call writes all of offsets, source and row, whatever the routing, and the same on every pass.
 * Strides (ld) count elements from one row to the next; rows start on 16 bytes.  All pointers are device pointers, nothing is allocated or
 * synchronised.  Outputs must not overlap each other or the inputs.
 * What all three calls refuse: MOE_ERR_UNSUPPORTED: cols no multiple of 8 or > 2^21, tokens > 2^21, top_k > 32, n_groups > 2047.
 */

/*
 * rows[r] = x[source[r] / top_k]: the tokens' rows in the order of their groups.
 * Rows behind the last one are not touched, or zeroed where zero_rest is set.  No tokens: offsets are zeros.
 * Many assignments are counted first, in the caller's workspace of moe_sort_tokens_workspace_bytes (0: none needed; more assignments or groups of
 * the same kind never need less).  Calls that share a workspace must be ordered against each other (one stream).
 *   MOE_ERR_CAPACITY: workspace too small.
 */
typedef struct {
    int32_t tokens, top_k, n_groups;
    int32_t n_experts;            /* entries of expert_map; not read without one */
    int32_t cols;
    int32_t dtype;                /* moe_dtype_t of x and rows */
    int32_t zero_rest;
    const int32_t *ids;           /* [tokens, top_k] */
    const int32_t *expert_map;    /* [n_experts] or NULL */
    const void *x;                /* [tokens, cols] */
    int64_t ld_x;
    void   *rows;                 /* [tokens * top_k, cols] */
    int64_t ld_rows;
    int32_t *offsets;             /* [n_groups + 1] */
    int32_t *source;              /* [tokens * top_k] */
    int32_t *row;                 /* [tokens, top_k] */
    void   *workspace;            /* 16-byte aligned, or NULL when none is needed */
    size_t  workspace_bytes;
} moe_sort_tokens_t;
size_t moe_sort_tokens_workspace_bytes(int32_t tokens, int32_t top_k, int32_t n_groups);
moe_status_t moe_sort_tokens(const moe_sort_tokens_t *args, void *hip_stream);

/*
 * out[t] = sum over j of weights[t, j] * y[row[t, j]], in the order of j, assignments without a row left out: added up in fp32, rounded once.
 * weights NULL: ones, which is the gradient of moe_sort_tokens (y: the rows' gradient, out: the tokens').  A token without rows gets zeros.
 * An entry of row outside [0, tokens * top_k) has no row, and its weight does not count, whatever it is; rows that no entry names are not read.
 */
typedef struct {
    int32_t tokens, top_k, cols;
    int32_t dtype;                /* moe_dtype_t of y and out */
    const void *y;                /* [tokens * top_k, cols] */
    int64_t ld_y;
    const int32_t *row;           /* [tokens, top_k] */
    const float *weights;         /* [tokens, top_k] or NULL */
    void   *out;                  /* [tokens, cols] */
    int64_t ld_out;
} moe_combine_tokens_t;
moe_status_t moe_combine_tokens(const moe_combine_tokens_t *args, void *hip_stream);

/*
 * The gradient of the above, for grad_out = the gradient of out:
 *     grad_y[row[t, j]] = weights[t, j] * grad_out[t],   grad_weights[t, j] = <grad_out[t], y[row[t, j]]>, 0 where there is no row,
 * each rounded once from fp32; either may be NULL, not both.  Entries of row must differ from each other, as those of moe_sort_tokens do.
 * Rows of grad_y that no entry of row names -- those behind the last one, those of assignments whose entry a caller set to -1 -- are not touched, or
 * zeroed where source is given.
 */
typedef struct {
    int32_t tokens, top_k, cols;
    int32_t dtype;                /* moe_dtype_t of grad_out, y and grad_y */
    const void *grad_out;         /* [tokens, cols] */
    int64_t ld_grad_out;
    const void *y;                /* [tokens * top_k, cols]; not read without grad_weights */
    int64_t ld_y;
    const int32_t *row;           /* [tokens, top_k] */
    const float *weights;         /* [tokens, top_k] or NULL: ones */
    const int32_t *source;        /* [tokens * top_k] as moe_sort_tokens writes it, or NULL */
    void   *grad_y;               /* [tokens * top_k, cols] or NULL */
    int64_t ld_grad_y;
    float  *grad_weights;         /* [tokens, top_k] or NULL */
} moe_combine_tokens_backward_t;
moe_status_t moe_combine_tokens_backward(const moe_combine_tokens_backward_t *args, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ELASTICMOE_DISPATCH_H */
