// Block-scaled e4m3 products of few rows: the weights are streamed once, straight into the matrix cores' operands.
//
//   out[r, c] = sum_b as[r, b] ws[c / 128, b] sum_{k in block b} a[r, k] w[c, k]
//
// The sum over a scale block starts at zero and is added to the fp32 accumulators times as * ws.  Both operands are loaded the same
// way -- lane (quad, l15) has bytes [16 quad, 16 quad + 16) and the same 64 further of its row's 128 -- so which k an instruction
// pairs with which does not matter: both sides agree.  The bytes go through bf16, which holds every e4m3 value, and its matrix
// instructions (multiply_exact in scaled.h): twice as many as of the 8-bit ones, which nobody waits for here.
// Weight rows are the first operand: a lane then holds four neighbouring columns of one row of the result.
//
// A workgroup is eight wavefronts on 16 or 32 weight rows (with swiglu as many gate and up rows) times 16 or 32 rows; wavefront i takes the
// K-steps i, i + 8, ..., neighbours read neighbouring lines, and their partial sums are added in that order through LDS.
// Bound by the weight stream for up to 32 rows, above by the rows, which every workgroup reads out of L2.
#include "scaled.h"

namespace emoe {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;

// this lane's 32 bytes of a row's K-step; `left`: bytes of the row from this lane's first on (a step that ends inside the block: what is behind the end is zero)
__device__ __forceinline__ Bytes32 fetch(const uint8_t *p, int left)
{
    Bytes32 f;
    f.lo = f.hi = make_uint4(0, 0, 0, 0);
    if (left > 0) f.lo = *(const uint4 *)p;
    if (left > 64) f.hi = *(const uint4 *)(p + 64);
    return f;
}

// MT 16-row tiles of a, WG 16-row tiles of weights (with swiglu of gate and of up rows), D K-steps on their way per wavefront
template <bool kSwiglu, int MT, int WG, int D, typename TOut>
__global__ __launch_bounds__(kThreads) void k_scaled_stream(SGemm g, int n_slices)
{
    constexpr int WT = kSwiglu ? 2 * WG : WG;                  // with swiglu WG tiles of gate rows, then their up rows
    constexpr int STRIDE = WT * 16 + 4;                        // floats of a row's partial sums in LDS
    __shared__ float red[kWaves][MT * 16][STRIDE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, quad = lane >> 4;
    const int tile = blockIdx.x / n_slices, n0 = (blockIdx.x % n_slices) * 16 * WG;
    MTile mt = {0, tile * MT * 16, min(MT * 16, g.m - tile * MT * 16), 0};
    if (g.tiles) {
        if (tile >= *g.n_tiles) return;
        mt = g.tiles[tile];
    }
    const uint8_t *wp[WT], *ap[MT];
    const float *sp[MT];
#pragma unroll
    for (int t = 0; t < WT; ++t)
        wp[t] = g.w + (size_t)mt.slot * g.w_slot + ((size_t)min(n0 + t % WG * 16 + l15, g.n - 1) + (size_t)(t / WG) * g.n) * g.k + quad * 16;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int r = mt.row_begin + min(m * 16 + l15, mt.rows - 1);
        const size_t ar = g.perm ? g.perm[r] : r;
        ap[m] = g.a + ar * g.ld_a + quad * 16;
        sp[m] = g.as + ar * g.ld_as;
    }
    const float *wsp = g.ws + (size_t)mt.slot * g.ws_slot + (size_t)(n0 / kScaleBlock) * g.kb;
    const float *wsu = wsp + (size_t)scale_blocks(g.n) * g.kb;
    const int live = (mt.rows + 15) >> 4;                      // 16-row tiles that exist

    f32x4 acc[WT][MT];
#pragma unroll
    for (int t = 0; t < WT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = (f32x4){0.f, 0.f, 0.f, 0.f};
    Bytes32 wf[D][WT], af[D][MT];
    float sa[D][MT], sw[D][kSwiglu ? 2 : 1];
    auto request = [&](int d, int b) __attribute__((always_inline)) {
        const int k0 = b * kScaleBlock, left = g.k - k0 - quad * 16;
#pragma unroll
        for (int t = 0; t < WT; ++t) wf[d][t] = fetch(wp[t] + k0, left);
#pragma unroll
        for (int m = 0; m < MT; ++m)
            if (m < live) { af[d][m] = fetch(ap[m] + k0, left); sa[d][m] = sp[m][b]; }
        sw[d][0] = wsp[b];
        if (kSwiglu) sw[d][kSwiglu ? 1 : 0] = wsu[b];
    };
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (wave + d * kWaves < g.kb) request(d, wave + d * kWaves);
    for (int b0 = wave; b0 < g.kb; b0 += D * kWaves) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int b = b0 + d * kWaves;
            if (b < g.kb) {
                Bf16x32 wb[WT];
#pragma unroll
                for (int t = 0; t < WT; ++t) wb[t].from(wf[d][t]);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    if (m < live) {
                        Bf16x32 ab;
                        ab.from(af[d][m]);
#pragma unroll
                        for (int t = 0; t < WT; ++t) {
                            const f32x4 s = multiply_exact(wb[t], ab);
                            const float f = sa[d][m] * sw[d][t / WG];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[t][m][e] = fmaf(s[e], f, acc[t][m][e]);
                        }
                    }
                if (b + D * kWaves < g.kb) request(d, b + D * kWaves);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
        if (m < live)
#pragma unroll
            for (int t = 0; t < WT; ++t) *(f32x4 *)&red[wave][m * 16 + l15][t * 16 + quad * 4] = acc[t][m];
    __syncthreads();
    // four columns of a row per thread
    for (int i = threadIdx.x; i < mt.rows * 4 * WG; i += kThreads) {
        const int row = i / (4 * WG), c4 = (i % (4 * WG)) * 4, col = n0 + c4;
        if (col >= g.n) continue;
        f32x4 s[kSwiglu ? 2 : 1];
#pragma unroll
        for (int t = 0; t < (kSwiglu ? 2 : 1); ++t) {
            s[t] = *(const f32x4 *)&red[0][row][t * WG * 16 + c4];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) s[t] += *(const f32x4 *)&red[w][row][t * WG * 16 + c4];
        }
        const size_t r = mt.row_begin + row;
        TOut *o = (TOut *)g.out + r * g.ld_out + col;
        const TOut *add = g.add ? (const TOut *)g.add + r * g.ld_add + col : nullptr;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = kSwiglu ? silu_mul(s[0][e], s[kSwiglu ? 1 : 0][e]) : s[0][e];
            if (add && col + e < g.n) v[e] += load_f32<TOut>(add, e);
        }
        if (col + 4 <= g.n) {
            if constexpr (sizeof(TOut) == 4) *(float4 *)o = make_float4(v[0], v[1], v[2], v[3]);
            else *(uint2 *)o = make_uint2((uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16), (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
        } else {
            for (int e = 0; e < g.n - col; ++e) store_f32<TOut>(o, e, v[e]);
        }
    }
}

template <bool kSwiglu, int MT, int WG, int D, typename TOut>
void launch_as(const SGemm &g, hipStream_t st)
{
    const int slices = (g.n + 16 * WG - 1) / (16 * WG), tiles = g.tiles ? g.max_tiles : (g.m + MT * 16 - 1) / (MT * 16);
    hipLaunchKernelGGL((k_scaled_stream<kSwiglu, MT, WG, D, TOut>), dim3(slices * tiles), dim3(kThreads), 0, st, g, slices);
}
}  // namespace

// us, (16-row tiles of a, of weights, K-steps ahead), weights from memory, bf16 results:
//   7168 x 2048       1 row  (1,1,2) 6.4  (2,2,1) 6.1    16 rows 8.2  7.0    64 rows 19.3  12.8   (4,2,1) 11.6   333 rows 84  45.6  46.6
//   4096 x 7168       1 row          8.7          10.8   16 rows 11.3 14.4   64 rows 34.0  19.3           29.2   333 rows 162 89    81
//    768 x 2048       1 row          4.2          4.9    64 rows 5.3  7.5
// so the two-by-two form as soon as it has a workgroup for most compute units.  With swiglu (gate and up: twice the weight rows)
//   1408 x 2048       17 rows (1,1,2) 9.5  (2,1,2) 10.0 (2,2,1) 11.8   64 rows 12.8 11.3 13.0   333 rows 31 28.7 21.9
//   2048 x 7168       17 rows         17.2         19.1         25.1   64 rows 28.2 22.7 28.7   333 rows 122 98  75
int stream_tile_rows(int m, int n, bool swiglu)
{
    const long long t32 = (m + 31) / 32;
    if (swiglu) return (n + 15) / 16 * t32 >= 170 ? 32 : 16;
    return (n + 31) / 32 * t32 >= 200 ? 32 : 16;
}

hipError_t launch_scaled_stream(const SGemm &g, bool swiglu, bool out_bf16, int tile_rows, hipStream_t st)
{
    const long long tiles = g.tiles ? g.max_tiles : (g.m + tile_rows - 1) / tile_rows;
    if (swiglu) {
        if (tile_rows == 16)                          launch_as<true, 1, 1, 2, float>(g, st);
        else if ((g.n + 31) / 32 * tiles >= 400)      launch_as<true, 2, 2, 1, float>(g, st);
        else                                          launch_as<true, 2, 1, 2, float>(g, st);
    } else if (out_bf16) {
        if (tile_rows == 16) launch_as<false, 1, 1, 2, uint16_t>(g, st);
        else                 launch_as<false, 2, 2, 1, uint16_t>(g, st);
    } else {
        if (tile_rows == 16) launch_as<false, 1, 1, 2, float>(g, st);
        else                 launch_as<false, 2, 2, 1, float>(g, st);
    }
    return hipGetLastError();
}

}  // namespace emoe
