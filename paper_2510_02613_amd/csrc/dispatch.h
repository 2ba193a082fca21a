// Internal declarations of the operators that sort tokens by expert and add them up again.
#pragma once
#include "elasticmoe_dispatch.h"
#include "moe_internal.h"

namespace emoe {

constexpr int kDispatchMaxK = 32;         // assignments of a token
constexpr int kDispatchMaxGroups = 2047;  // as many as a layer has slots
constexpr int kSortBlock = 1024;          // assignments that share a row of counts
// Up to here every workgroup counts all assignments itself.  us (counted first in brackets), 8 assignments a token, 128 groups, rows of 512 bytes: 160 tokens 5.5 (8.5),
// 384 7.3 (8.7), 512 7.7 (8.6); 640 9.5 (9.1), 1024 11.1 (9.6), 2048 17.0 (10.6).  With 2047 groups this one launch stays ahead for longer: 1024 tokens 13.8 (16.9).
constexpr int kSortOneLaunch = 4096;
// Up to here (counts in all) every workgroup adds the blocks' counts up itself.  us (one workgroup that scans them, in brackets), the same: 8192 tokens, 8256 counts,
// 21.6 (38.7), 32768 tokens 78 (116), 65536, just above, 231 (240), 131072 744 (474).  Which side is ahead hangs on more than the counts: 9000 tokens and 2047
// groups, 145408 counts, 98 (203).
constexpr long long kSortSums = 65536;

// Rows are handled as runs of 16 bytes (`chunks` of them), strides in bytes.
struct SortJob {
    int32_t tokens, top_k, n_groups, n_experts, chunks, zero_rest;
    const int32_t *ids, *map;
    const char *x;
    char *rows;
    int64_t ld_x, ld_rows;
    int32_t *offsets, *source, *row;
    int32_t *counts;                      // [blocks of kSortBlock assignments][n_groups + 1], the last for assignments without a row
};
struct CombineJob {
    int32_t tokens, top_k, chunks;
    const char *y, *grad_out;             // backward: both
    char *out, *grad_y;
    int64_t ld_y, ld_out, ld_grad_out, ld_grad_y;
    const int32_t *row, *source;
    const float *weights;
    float *grad_weights;
};
int sort_blocks(int tokens, int top_k);   // rows of counts, 0: none needed
hipError_t launch_sort_tokens(const SortJob &j, hipStream_t st);
hipError_t launch_combine_tokens(const CombineJob &j, bool bf16, hipStream_t st);
hipError_t launch_combine_tokens_backward(const CombineJob &j, bool bf16, hipStream_t st);

}  // namespace emoe
