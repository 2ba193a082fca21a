/*
 * elasticmoe_four_bit.h -- experts held in 4 bits: quantising, and the products of bf16 rows with 4-bit weights, dense or group by group of
 * sorted rows (elasticmoe_dispatch.h).  Entry points, statuses, memory and error rules are those of elasticmoe.h.
 */
#ifndef ELASTICMOE_FOUR_BIT_H
#define ELASTICMOE_FOUR_BIT_H

#include "elasticmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A 4-bit matrix [rows, cols], cols a multiple of 32, is two e2m1 values a byte -- 0, 0.5, 1, 1.5, 2, 3, 4, 6, the sign in bit 3; the even column in
 * bits 0..3 -- and an e8m0 byte b, the power of two 2^(b - 127), for each row and 32 consecutive columns; b = 255 makes its 32 values NaN.
 * Quantising takes the smallest power of two (2^-127 at least) that leaves no magnitude of the 32 above 6, and v / 2^p to the nearest, ties to the even
 * code; signs are kept, of zeros too.  A group that holds a NaN or an infinity gets b = 255 and zeros.  Powers of 2^126 and 2^127 reach values of 2^128 and
above, which are infinities in fp32 and bf16: as quantised values, where magnitudes from 3.5 * 2^126 (2.98e38) on get 2^128, and as the weights of a product.
 * Strides (ld) count elements from one row to the next, bytes for q and scale; rows behind the last one are not touched.  All pointers are device pointers,
 * nothing is allocated or synchronised, rows == 0 and m == 0 are no-ops.  Unless a call says otherwise its outputs must not overlap each other or its inputs.
 */

/*
 * x in 4 bits; values, where given, the numbers that the 4 bits stand for, in x's type.
 *   MOE_ERR_UNSUPPORTED: cols no multiple of 32, rows or cols > 2^21.
 */
typedef struct {
    int32_t rows, cols;
    int32_t dtype;          /* moe_dtype_t of x and values */
    const void *x;          /* [rows, cols], 16-byte aligned rows */
    int64_t ld_x;
    void   *q;              /* [rows, cols / 2], 4-byte aligned rows */
    int64_t ld_q;
    void   *scale;          /* [rows, cols / 32] */
    int64_t ld_scale;
    void   *values;         /* [rows, cols] or NULL, 16-byte aligned rows; may be x itself (same address and ld) */
    int64_t ld_values;
} moe_four_bit_quantize_t;
moe_status_t moe_four_bit_quantize(const moe_four_bit_quantize_t *args, void *hip_stream);

/*
 * out = a w^T (+ add): bf16 rows times 4-bit weights.  With offsets (device, as moe_sort_tokens writes them) row r of group g, offsets[g] <= r <
 * offsets[g + 1], takes the weights w[g]; rows in no group are not touched, and what offsets name outside [0, m) is left out.  Offsets must not decrease.
 * A weight times its power of two is a bf16 number (below 2^128), so that products are exact; their sums are fp32's, rounded once at the end.  The order of a sum
 * depends on the sizes of the call, not on what runs beside it.  out may be add itself (same address and ld).
 * Made for few rows a group, where the weights' bytes are what a product costs; many rows work too, at about half the rate of a bf16 product.
 *   MOE_ERR_UNSUPPORTED: k no multiple of 32; m, n or k > 2^21; ld_a >= 2^24; groups > 2047; more tiles than a launch can have workgroups.
 */
typedef struct {
    int32_t m, n, k;
    int32_t groups;         /* 1 without offsets */
    int32_t out_dtype;      /* moe_dtype_t of add and out */
    const void *a;          /* [m, k] bf16, 16-byte aligned rows */
    int64_t ld_a;
    const int32_t *offsets; /* [groups + 1] or NULL */
    const void *w;          /* [groups, n, k / 2], contiguous, 16-byte aligned */
    const void *w_scale;    /* [groups, n, k / 32], contiguous */
    const void *add;        /* [m, n] or NULL; 16-byte aligned rows */
    int64_t ld_add;
    void   *out;            /* [m, n]; 16-byte aligned rows (n may be any number) */
    int64_t ld_out;
} moe_four_bit_matmul_t;
moe_status_t moe_four_bit_matmul(const moe_four_bit_matmul_t *args, void *hip_stream);

/*
 * The first half of SwiGLU experts: out = silu(a Wg^T) * (a Wu^T), from the fp32 sums, rounded once.  Offsets and groups as above.
 *   MOE_ERR_UNSUPPORTED: as above, for n = 2 inter.
 */
typedef struct {
    int32_t m, inter, k;
    int32_t groups;         /* 1 without offsets */
    int32_t out_dtype;      /* moe_dtype_t of out */
    const void *a;          /* [m, k] bf16, 16-byte aligned rows */
    int64_t ld_a;
    const int32_t *offsets; /* [groups + 1] or NULL */
    const void *w;          /* [groups, 2 inter, k / 2], contiguous, 16-byte aligned: gate rows, then up rows */
    const void *w_scale;    /* [groups, 2 inter, k / 32], contiguous */
    void   *out;            /* [m, inter]; 16-byte aligned rows */
    int64_t ld_out;
} moe_four_bit_swiglu_t;
moe_status_t moe_four_bit_swiglu(const moe_four_bit_swiglu_t *args, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ELASTICMOE_FOUR_BIT_H */
