/*
 * elasticmoe_scaled.h -- the 8-bit path of the MoE expert layer: e4m3 experts with block scales, and the operators
 * around them.  Entry points, statuses, memory and error rules are those of elasticmoe.h.
 */
#ifndef ELASTICMOE_SCALED_H
#define ELASTICMOE_SCALED_H

#include "elasticmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * An 8-bit matrix is bytes in e4m3 (4 exponent bits, 3 mantissa bits, largest value 448, no infinities) and fp32 scales:
 * one for each row and 128 consecutive columns of an activation, one for each block of 128 x 128 of a weight matrix; the
 * last block of a row or column may be shorter.  An element stands for byte * scale.  Quantising a group takes
 *     a = max |v|,  scale = a / 448,  byte = 448 v / a rounded to the nearest, ties to even;
 * a group whose a is below 2^-110 gets scale 0 and zeros, a group that holds a NaN or an infinity stands for NaN throughout.
 * Strides (ld) count elements from one row to the next; rows behind the last one are not touched.  All pointers are
 * device pointers, nothing is allocated or synchronised, rows == 0 and m == 0 are no-ops.  Unless a call says otherwise
 * its outputs must not overlap each other or its inputs.
 */

/*
 * RMS norm of x, or of x + residual, with up to three results, each rounded once from fp32:
 *     r = x + residual,   y = r / sqrt(mean(r^2) + eps) * weight
 *     sum = r,   out = y,   (q, q_scale) = y quantised per row and 128 columns.
 * sum and out may each be x or residual themselves (same address and ld).  Any of the three may be left out, not all.
 * The squares are summed in fp32, of rows whose squares would leave it times a power of two: any finite r has its norm, but for a row of zeros where
 * eps is 0, which is NaN.  (r itself is fp32: where x + residual overflows, y is NaN.)
 *   MOE_ERR_UNSUPPORTED: cols no multiple of 8 or > 32768, rows > 2^21.
 */
typedef struct {
    int32_t rows, cols;
    int32_t dtype;          /* moe_dtype_t of x, residual, weight, sum and out */
    float   eps;            /* finite, not negative */
    const void *x;          /* [rows, cols], 16-byte aligned rows as all of them */
    int64_t ld_x;
    const void *residual;   /* or NULL */
    int64_t ld_residual;
    const void *weight;     /* [cols] or NULL: ones */
    void   *sum;            /* or NULL; needs a residual */
    int64_t ld_sum;
    void   *out;            /* or NULL */
    int64_t ld_out;
    void   *q;              /* or NULL; 8-byte aligned rows */
    int64_t ld_q;
    float  *q_scale;        /* [rows, ceil(cols/128)], NULL iff q is */
    int64_t ld_scale;
} moe_rms_norm_t;
moe_status_t moe_rms_norm(const moe_rms_norm_t *args, void *hip_stream);

/*
 * Quantising: block_rows == 1 rows of activations (scale [rows, ceil(cols/128)]), block_rows == 128 a weight matrix
 * (scale [ceil(rows/128), ceil(cols/128)]).
 *   MOE_ERR_UNSUPPORTED: cols no multiple of 8, > 32768 with block_rows == 1, > 2^21; rows > 2^21.
 */
typedef struct {
    int32_t rows, cols;
    int32_t dtype;          /* moe_dtype_t of x */
    int32_t block_rows;     /* 1 or 128 */
    const void *x;          /* [rows, cols], 16-byte aligned rows */
    int64_t ld_x;
    void   *q;              /* 8-byte aligned rows */
    int64_t ld_q;
    float  *scale;
    int64_t ld_scale;
} moe_quantize_t;
moe_status_t moe_quantize(const moe_quantize_t *args, void *hip_stream);

/*
 * out = a w^T (+ add): 8-bit rows times 8-bit weights.  Products are exact, the sums of a scale block's 128 and of the blocks' sums
 * times their two scales fp32; one rounding at the end.  out may be add itself (same address and ld).
 * bf16 results may come from the 8-bit matrix instructions, at up to twice the rate for many rows, where the caller asks for it: those drop of
 * eight products what lies 2^-14 below the largest (1.5e-5 to 6e-5 of the norm of usual results; where large products
 * cancel, what they leave is lost).  Few rows are streamed with exact products then too: a row may come out differently in calls of different m.
 *   MOE_ERR_UNSUPPORTED: MOE_FAST_PRODUCTS with fp32 results; k no multiple of 16, m or n > 2^21, rows of a or w of 2^23 bytes or more, ld_a_scale of 2^21 or
 *   more, more tiles than a launch can have workgroups (some 2^39 results).
 */
#define MOE_FAST_PRODUCTS 0x100
typedef struct {
    int32_t m, n, k;
    int32_t out_dtype;      /* moe_dtype_t of add and out; MOE_BF16 | MOE_FAST_PRODUCTS: bf16 from the 8-bit instructions */
    const void  *a;         /* [m, k] e4m3, 16-byte aligned rows */
    int64_t ld_a;
    const float *a_scale;   /* [m, ceil(k/128)] */
    int64_t ld_a_scale;
    const void  *w;         /* [n, k] e4m3, contiguous, 16-byte aligned */
    const float *w_scale;   /* [ceil(n/128), ceil(k/128)], contiguous */
    const void  *add;       /* [m, n] or NULL; 16-byte aligned rows */
    int64_t ld_add;
    void   *out;            /* [m, n]; 16-byte aligned rows (n may be any number) */
    int64_t ld_out;
} moe_scaled_matmul_t;
moe_status_t moe_scaled_matmul(const moe_scaled_matmul_t *args, void *hip_stream);

/*
 * The first half of a dense SwiGLU expert: h = silu(a Wg^T) * (a Wu^T), quantised per row and 128 columns from fp32.
 * Few rows, or little weights, go through fp32 rows in the caller's workspace: moe_scaled_swiglu_workspace_bytes of the same sizes (0: none needed;
 * more rows may need none where fewer need some), or once and for all moe_scaled_swiglu_max_workspace_bytes, which is enough for every m up to max_m.
 * Calls that share a workspace must be ordered against each other (one stream).
 *   MOE_ERR_UNSUPPORTED: as for the product above; inter no multiple of 16 or > 32768.   MOE_ERR_CAPACITY: workspace too small.
 */
typedef struct {
    int32_t m, inter, k;
    const void  *a;         /* [m, k] e4m3, 16-byte aligned rows */
    int64_t ld_a;
    const float *a_scale;   /* [m, ceil(k/128)] */
    int64_t ld_a_scale;
    const void  *w;         /* [2 inter, k] e4m3, contiguous, 16-byte aligned: gate rows, then up rows */
    const float *w_scale;   /* [2 ceil(inter/128), ceil(k/128)], contiguous: the gate rows' blocks, then the up rows' */
    void   *q;              /* [m, inter]; 8-byte aligned rows */
    int64_t ld_q;
    float  *q_scale;        /* [m, ceil(inter/128)] */
    int64_t ld_scale;
    void   *workspace;      /* 256-byte aligned, or NULL when none is needed */
    size_t  workspace_bytes;
} moe_scaled_swiglu_t;
size_t moe_scaled_swiglu_workspace_bytes(int32_t m, int32_t inter, int32_t k);
size_t moe_scaled_swiglu_max_workspace_bytes(int32_t max_m, int32_t inter, int32_t k);
moe_status_t moe_scaled_swiglu(const moe_scaled_swiglu_t *args, void *hip_stream);

/*
 * A layer whose experts are held in 8 bits: half the weight bytes.  It is created with
 *   buf->w13 [S,2I,H] and buf->w2 [S,H,I]   e4m3 pools in the place of act_dtype ones,
 *   w13_scale  [S, 2 ceil(I/128), ceil(H/128)]  the gate rows' blocks of a slot, then the up rows',
 *   w2_scale   [S, ceil(H/128), ceil(I/128)],
 * all of it the caller's, like the rest of buf, and a workspace of moe_scaled_workspace_bytes(cfg).  cfg->act_dtype is MOE_BF16, the
 * type of x and out.  From then on it is a layer as any other: placements (moe_set_expert_map, moe_set_expert_replicas), page pools
 * (slots of 2 I H and H I bytes; scales stay with the slot's number when pages are exchanged, the caller exchanges them too), profiling, moe_forward and moe_forward_routed, which quantise x.  Products are exact and
 * their sums fp32's, the rows of h are quantised (from fp32) between the GEMMs, the expert outputs wait for the combine in fp32, and out is rounded once.
 *   MOE_FLAG_FAST_PRODUCTS  the caller takes the 8-bit matrix instructions for the passes that do not stream their weights, at up to twice the rate
 *                           for many tokens: those drop of eight products what lies 2^-14 below the largest.  That moves one of some three thousand
 *                           bytes of h to its neighbour, 0.0012 of the norm of usual outputs beside the 0.0017 of out's rounding (where large products
 *                           cancel, what they leave is lost).  Expert outputs wait in 16 bits with a scale per 64 columns then (5e-5).  A pass of few tokens
 *                           is streamed, and exact, all the same: a token's output depends on how many there are.  Other layers refuse the flag.
 * moe_workspace_view's h names the rows of h in 8 bits, its y is not for reading.  MOE_FLAG_FORCE_GENERIC and moe_load_expert are MOE_ERR_UNSUPPORTED on such a layer;
 * moe_forward_static, which knows no layer, takes act_dtype pools only.
 *   MOE_ERR_UNSUPPORTED (beyond moe_layer_create): act_dtype not MOE_BF16, H or I no multiple of 16 or > 32768,
 *   max_tokens * hidden >= 2^32, max_tokens * (top_k + n_shared) > 2^21.
 *   moe_load_expert_scaled  moe_load_expert for such a layer: the sources of the weights (16-byte aligned) and of their scales.
 *   moe_forward_scaled      a pass for tokens that are in 8 bits already (moe_rms_norm writes them): xq [T,H] e4m3, contiguous and 16-byte
 *                           aligned, x_scale [T, ceil(H/128)] contiguous.  topk_ids and topk_w as in moe_forward_routed, or both NULL:
 *                           the gate runs on x, bf16 [T,H]; with them given x may be NULL (not with MOE_FLAG_IDENTITY_EXPERTS).
 *                           MOE_ERR_UNSUPPORTED on a layer whose experts are not in 8 bits.  All else as moe_forward.
 */
#define MOE_FLAG_FAST_PRODUCTS 16u
size_t moe_scaled_workspace_bytes(const moe_config_t *cfg);
moe_status_t moe_layer_create_scaled(const moe_config_t *cfg, const moe_buffers_t *buf, const float *w13_scale, const float *w2_scale, moe_layer_t **out);
moe_status_t moe_load_expert_scaled(moe_layer_t *layer, int32_t slot, const void *src_w13, const float *src_w13_scale,
                                    const void *src_w2, const float *src_w2_scale,
                                    void *copy_stream, void *serve_stream, int32_t copy_blocks);
moe_status_t moe_forward_scaled(moe_layer_t *layer, const void *x, const void *xq, const float *x_scale, int32_t T,
                                const int32_t *topk_ids, const float *topk_w, int32_t shared_begin, int32_t shared_end,
                                void *out, void *hip_stream, uint32_t flags);

#ifdef __cplusplus
}
#endif
#endif /* ELASTICMOE_SCALED_H */
