// The 4-bit product: which form of the kernel runs.
#include "four_rows.h"

namespace emoe {
namespace {

template <typename TOut>
hipError_t launch(const FourGemm &g, hipStream_t st)
{
    const int each = rows_each(g), many = g.offsets ? 128 : 64;
    const bool brief = g.k <= 1024;      // powers a line at a time
    if (each > many && workgroups(g, 256, 64) >= 200) return launch_as<false, 8, 1, 4, 2, 1, 256, 2, false, TOut>(g, row_tiles(g, 64), st);
    if (each > 16 && workgroups(g, 128, 32) >= 300) {
        if (brief) return launch_as<false, 4, 1, 2, 2, 1, 256, 3, true, TOut>(g, row_tiles(g, 32), st);
        return launch_as<false, 4, 1, 2, 2, 1, 256, 3, false, TOut>(g, row_tiles(g, 32), st);
    }
    if (each <= 16 && workgroups(g, 256, 16) >= 300) {
        if (brief) return launch_as<false, 8, 1, 1, 2, 1, 512, 4, true, TOut>(g, row_tiles(g, 16), st);
        return launch_as<false, 8, 1, 1, 2, 1, 512, 4, false, TOut>(g, row_tiles(g, 16), st);
    }
    if (workgroups(g, 128, 16) >= 140) return launch_as<false, 8, 1, 1, 1, 1, 1024, 4, false, TOut>(g, row_tiles(g, 16), st);
    if (workgroups(g, 64, 16) >= 200) return launch_as<false, 4, 2, 1, 1, 1, 1024, 2, true, TOut>(g, row_tiles(g, 16), st);
    if (lds_of<false, 1, 8, 1, 2, 0, true>(g) <= kMostLds / 2) return launch_as<false, 1, 8, 1, 2, 1, 0, 2, true, TOut>(g, row_tiles(g, 16), st);
    return launch_as<false, 1, 8, 1, 2, 1, 2048, 2, true, TOut>(g, row_tiles(g, 16), st);
}

}  // namespace

bool four_product_fits(const FourGemm &g) { return (g.n + 15ll) / 16 * g.groups + 8 <= kMostThreads / 512; }

hipError_t launch_four_matmul(const FourGemm &g, bool out_bf16, hipStream_t st) { return out_bf16 ? launch<uint16_t>(g, st) : launch<float>(g, st); }

}  // namespace emoe
