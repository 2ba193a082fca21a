// The 4-bit product with SwiGLU: which form of the kernel runs.
#include "four_rows.h"

namespace emoe {
namespace {

template <typename TOut>
hipError_t launch(const FourGemm &g, hipStream_t st)
{
    const int each = rows_each(g), many = g.offsets ? 128 : 64;
    const bool brief = g.k <= 4096;
    if (g.m > 16) {
        if (each > many && workgroups(g, 128, 64) >= 300) return launch_as<true, 8, 1, 4, 1, 1, 256, 2, false, TOut>(g, row_tiles(g, 64), st);
        if (each > 16 && workgroups(g, brief ? 64 : 128, 32) >= 300) {
            if (brief) return launch_as<true, 4, 1, 2, 1, 1, 256, 3, false, TOut>(g, row_tiles(g, 32), st);
            return launch_as<true, 4, 1, 2, 2, 1, 256, 2, false, TOut>(g, row_tiles(g, 32), st);
        }
        if (!brief && each <= 16 && g.m > 2 * g.groups && workgroups(g, 128, 16) >= 300) return launch_as<true, 8, 1, 1, 1, 1, 512, 4, false, TOut>(g, row_tiles(g, 16), st);
        if ((brief || !g.offsets) && workgroups(g, 64, 16) >= 150) return launch_as<true, 4, 1, 1, 1, 1, 512, 3, false, TOut>(g, row_tiles(g, 16), st);
        if (workgroups(g, 32, 16) >= 200) return launch_as<true, 2, 4, 1, 1, 1, 1024, 2, true, TOut>(g, row_tiles(g, 16), st);
    }
    if (lds_of<true, 1, 8, 1, 1, 0, true>(g) <= kMostLds / 2) return launch_as<true, 1, 8, 1, 1, 1, 0, 2, true, TOut>(g, row_tiles(g, 16), st);
    return launch_as<true, 1, 8, 1, 1, 1, 2048, 2, true, TOut>(g, row_tiles(g, 16), st);
}

}  // namespace

hipError_t launch_four_swiglu(const FourGemm &g, bool out_bf16, hipStream_t st) { return out_bf16 ? launch<uint16_t>(g, st) : launch<float>(g, st); }

}  // namespace emoe
