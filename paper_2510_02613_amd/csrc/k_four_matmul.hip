// The 4-bit product: which form of the kernel runs.
#include "four_rows.h"

namespace emoe {
namespace {

// us (the next best form in brackets), n x k, bf16 results:
//   eight wavefronts along K on 32 columns: 7168 x 2048 1 row 4.1 (4.6), 16 rows 5.3 (5.4)
//   4 x 2 wavefronts on 64 columns: 7168 x 2048 32 rows 7.0 (7.3), one token of a Qwen3-30B-A3B-shaped layer 4.7 (5.4)
//   128 columns: 7168 x 2048 64 rows 8.9 (12.6), 128 rows 12.4 (15.6), 1543 x 1440 173 rows 6.6 (8.7)
//   256 columns, sorted rows: 40 tokens of the Qwen3 shape 20.5 (24), 64 tokens of a DeepSeek-V3-shaped rank 47 (55)
//   32 rows, 128 columns: 333 tokens of the Qwen3 shape 33 (42), 7168 x 2048 256 rows 18 (23)
// Sorted rows with a short k from more than 10 rows a group on, for some groups have half as many again: 10.6 rows each 28.3 (16-row tiles 29.7), 8.1 rows each 28.1 (25.5),
// where a few experts are popular 30.2 (36.4) and 27.3 (32.0).  With a longer k (1408) both are alike between 10 and 16.
//   64 rows, 256 columns: 7168 x 2048 512 rows 27 (33), 1000 rows 51 (52); not for sorted rows (4096 tokens of the Qwen3 shape 241, with 32 rows 220)
// Powers a line at a time up to k = 1024, by way of LDS above: 333 and 40 tokens of the Qwen3 shape (k = 768) 33 and 20.5 (35 and 21.7),
// 64 tokens of the rank (k = 2048) 52 (47).
template <typename TOut>
hipError_t launch(const FourGemm &g, hipStream_t st)
{
    const int each = rows_each(g);
    const bool brief = g.k <= 1024;
    const int few = g.offsets && brief ? 10 : 16;
    if (!g.offsets && each > 64 && workgroups(g, 256, 64) >= 200) return launch_as<false, 8, 1, 4, 2, 1, 256, 2, false, TOut>(g, row_tiles(g, 64), st);
    if (each > few && workgroups(g, 128, 32) >= 300) {
        if (brief) return launch_as<false, 4, 1, 2, 2, 1, 256, 3, true, TOut>(g, row_tiles(g, 32), st);
        return launch_as<false, 4, 1, 2, 2, 1, 256, 3, false, TOut>(g, row_tiles(g, 32), st);
    }
    if (each <= few && workgroups(g, 256, 16) >= 300) {
        if (brief) return launch_as<false, 8, 1, 1, 2, 1, 512, 4, true, TOut>(g, row_tiles(g, 16), st);
        return launch_as<false, 8, 1, 1, 2, 1, 512, 4, false, TOut>(g, row_tiles(g, 16), st);
    }
    if (workgroups(g, 128, 16) >= 140) return launch_as<false, 8, 1, 1, 1, 1, 1024, 4, false, TOut>(g, row_tiles(g, 16), st);
    if (workgroups(g, 64, 16) >= 200) return launch_as<false, 4, 2, 1, 1, 1, 1024, 2, true, TOut>(g, row_tiles(g, 16), st);
    // few workgroups: all of the rows' columns in LDS at once where they fit twice
    if (lds_of<false, 1, 8, 1, 2, 0, true>(g) <= kMostLds / 2) return launch_as<false, 1, 8, 1, 2, 1, 0, 2, true, TOut>(g, row_tiles(g, 16), st);
    return launch_as<false, 1, 8, 1, 2, 1, 2048, 2, true, TOut>(g, row_tiles(g, 16), st);
}

}  // namespace

bool four_product_fits(const FourGemm &g) { return (g.n + 15ll) / 16 * g.groups + 8 <= kMostThreads / 512; }

hipError_t launch_four_matmul(const FourGemm &g, bool out_bf16, hipStream_t st) { return out_bf16 ? launch<uint16_t>(g, st) : launch<float>(g, st); }

}  // namespace emoe
