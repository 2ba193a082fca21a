// The 4-bit product with SwiGLU: which form of the kernel runs.
#include "four_rows.h"

namespace emoe {
namespace {

constexpr int kEnough = 200;             // workgroups that fill the chip

template <typename TOut>
hipError_t launch(const FourGemm &g, hipStream_t st)
{
    const int each = rows_each(g);
    const bool brief = g.k <= 4096;
    if (g.m > 16) {
        if (each > 64 && workgroups(g, 128, 64) >= kEnough) return launch_as<true, 8, 1, 4, 1, 1, 256, 2, false, TOut>(g, row_tiles(g, 64), st);
        if (each > 16 && workgroups(g, brief ? 64 : 128, 32) >= kEnough) {
            if (brief) return launch_as<true, 4, 1, 2, 1, 1, 256, 3, false, TOut>(g, row_tiles(g, 32), st);
            return launch_as<true, 4, 1, 2, 2, 1, 256, 2, false, TOut>(g, row_tiles(g, 32), st);
        }
        if (each <= 16 && workgroups(g, brief ? 64 : 128, 16) >= kEnough) {
            if (brief) return launch_as<true, 4, 1, 1, 1, 1, 512, 3, false, TOut>(g, row_tiles(g, 16), st);
            return launch_as<true, 8, 1, 1, 1, 1, 512, 4, false, TOut>(g, row_tiles(g, 16), st);
        }
        if (workgroups(g, 32, 16) >= kEnough) return launch_as<true, 2, 4, 1, 1, 1, 1024, 2, true, TOut>(g, row_tiles(g, 16), st);
    }
    if (lds_of<true, 1, 8, 1, 1, 0, true>(g) <= kMostLds / 2) return launch_as<true, 1, 8, 1, 1, 1, 0, 2, true, TOut>(g, row_tiles(g, 16), st);
    return launch_as<true, 1, 8, 1, 1, 1, 2048, 2, true, TOut>(g, row_tiles(g, 16), st);
}

}  // namespace

hipError_t launch_four_swiglu(const FourGemm &g, bool out_bf16, hipStream_t st) { return out_bf16 ? launch<uint16_t>(g, st) : launch<float>(g, st); }

}  // namespace emoe
