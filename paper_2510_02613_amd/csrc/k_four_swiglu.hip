// The 4-bit product with SwiGLU: which form of the kernel runs.
#include "four_rows.h"

namespace emoe {
namespace {

// us (the next best form in brackets), inter x k, bf16 results:
//   eight wavefronts along K on 16 columns: 1408 x 2048 3 rows 4.7 (8.2), 2048 x 7168 16 rows 11.7 (18), one token of a DeepSeek-V3-shaped rank 10.6 (13.4)
//   2 x 4 wavefronts on 32 columns: 2048 x 7168 64 rows 17.9 (28.5), 8 tokens of that rank 42 (51)
//   64 columns: 768 x 2048 256 rows 9.2 (12.3), 2048 x 7168 200 rows 35 (42), 20 tokens of a Qwen3-30B-A3B-shaped layer 35 (38)
//   128 columns: 64 tokens of the rank (long rows) 87 (107)
//   32 rows, 64 columns: 333 tokens of the Qwen3 shape 52 (61), 1000 tokens 116 (119), 2048 x 7168 400 rows 47 (69)
//   (more than 10 sorted rows a group, as some have half as many again: Qwen3 shape 10.6 rows each 49 (16-row tiles 51), 8.1 rows each 48 (43.7), where a few experts are
//   popular 56 (62) and 51 (55))
//   32 rows, 128 columns: 333 tokens of the rank 102 (115), 4096 tokens of the Qwen3 shape 385 (409), 768 x 2048 2000 rows 26 (32)
// A tile of 64 rows is no faster anywhere (382 for 385, 27 for 26).
template <typename TOut>
hipError_t launch(const FourGemm &g, hipStream_t st)
{
    const int each = rows_each(g);
    const bool brief = g.k <= 4096;
    const int few = g.offsets && brief ? 10 : 16;
    if (g.m > 16) {
        if (each > 16 && (!brief || each > 64) && workgroups(g, 128, 32) >= 300) return launch_as<true, 4, 1, 2, 2, 1, 256, 2, false, TOut>(g, row_tiles(g, 32), st);
        if (each > few && workgroups(g, 64, 32) >= 300) return launch_as<true, 4, 1, 2, 1, 1, 256, 3, false, TOut>(g, row_tiles(g, 32), st);
        if (each <= 16 && !brief && g.m > 2 * g.groups && workgroups(g, 128, 16) >= 300) return launch_as<true, 8, 1, 1, 1, 1, 512, 4, false, TOut>(g, row_tiles(g, 16), st);
        if ((brief || !g.offsets) && workgroups(g, 64, 16) >= 150) return launch_as<true, 4, 1, 1, 1, 1, 512, 3, false, TOut>(g, row_tiles(g, 16), st);
        if (workgroups(g, 32, 16) >= 200) return launch_as<true, 2, 4, 1, 1, 1, 1024, 2, true, TOut>(g, row_tiles(g, 16), st);
    }
    // few workgroups: all of the rows' columns in LDS at once where they fit twice
    if (lds_of<true, 1, 8, 1, 1, 0, true>(g) <= kMostLds / 2) return launch_as<true, 1, 8, 1, 1, 1, 0, 2, true, TOut>(g, row_tiles(g, 16), st);
    return launch_as<true, 1, 8, 1, 1, 1, 2048, 2, true, TOut>(g, row_tiles(g, 16), st);
}

}  // namespace

hipError_t launch_four_swiglu(const FourGemm &g, bool out_bf16, hipStream_t st) { return out_bf16 ? launch<uint16_t>(g, st) : launch<float>(g, st); }

}  // namespace emoe
