// Internal declarations of the 4-bit operators: e2m1 values with a power of two for each row and 32 columns.
#pragma once
#include "elasticmoe_four_bit.h"
#include "moe_internal.h"

namespace emoe {

constexpr int kFourGroup = 32;            // columns that share a power of two: 16 bytes of a row

struct FourRows {
    int32_t rows, cols;
    const char *x;                        // strides in bytes
    uint8_t *q, *scale;
    char *values;
    int64_t ld_x, ld_q, ld_scale, ld_values;
};
hipError_t launch_four_quantize(const FourRows &j, bool bf16, hipStream_t st);

// out[r, c] = sum_k a[r, k] w[g(r)][c, k] (+ add), with swiglu n gate rows, then n up rows, and silu(gate) * up
struct FourGemm {
    const uint16_t *a;
    int64_t ld_a;
    const uint8_t *w, *ws;
    int32_t m, n, k, groups;
    const int32_t *offsets;               // NULL: all rows are group 0's
    int32_t sparse;                       // more groups than twice the rows: many have none
    const void *add;
    int64_t ld_add;
    void *out;
    int64_t ld_out;
};
bool four_product_fits(const FourGemm &g);    // its workgroups are as many as a launch can have
hipError_t launch_four_matmul(const FourGemm &g, bool out_bf16, hipStream_t st);
hipError_t launch_four_swiglu(const FourGemm &g, bool out_bf16, hipStream_t st);
constexpr long long kMostThreads = (1ll << 32) - 1;        // of a launch

}  // namespace emoe
