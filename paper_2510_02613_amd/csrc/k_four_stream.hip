// Products of bf16 rows with 4-bit weights, the weights streamed straight into the matrix cores' operands.
//
//   out[r, c] = sum_k a[r, k] code[c, k] 2^p[c, k / 32]
//
// A code times its power of two is a bf16 number (2^-128 .. 6 * 2^126 and its infinities): the conversion instruction makes two of them from a byte and the
// power, the products are exact and the sums fp32's.
// A K-step is 128 columns: lane (quad, l15) has the 16 bytes of row l15 that hold columns 32 quad .. 32 quad + 31 of the step, one group with one power, and of
// an activation row the 64 bytes of the same columns.  Instruction i takes the eight from 8 i of both.  Which k an instruction pairs with which does not
// matter: both sides agree.  Weight rows are the first operand: a lane then holds four neighbouring columns of one row of the result.
//
// A workgroup is eight wavefronts, KW of them along K (wavefront i takes the steps i, i + KW, ..., their sums are added in that order through LDS) on
// 8 / KW times WT tiles of 16 weight rows (with swiglu WT of gate and WT of up rows) times MT tiles of 16 rows.
// Bound by the weight stream for few rows, above by the rows, which every workgroup reads out of L2.
#include "four_bit.h"

namespace emoe {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr long long kMostGroups = (1ll << 32) / kThreads - 1;   // workgroups that a launch can have

__device__ __forceinline__ bf16x8 weights8(uint32_t codes, float power)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 3);
    return (bf16x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// four neighbouring columns of a row
template <bool kSwiglu, typename TOut>
__device__ __forceinline__ void finish(const FourGemm &g, size_t r, int col, const f32x4 &s, const f32x4 &up)
{
    TOut *o = (TOut *)g.out + r * g.ld_out + col;
    const TOut *add = g.add ? (const TOut *)g.add + r * g.ld_add + col : nullptr;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = kSwiglu ? silu_mul(s[e], up[e]) : s[e];
        if (!kSwiglu && add && col + e < g.n) v[e] += load_f32<TOut>(add, e);
    }
    if (col + 4 <= g.n) {
        if constexpr (sizeof(TOut) == 4) *(float4 *)o = make_float4(v[0], v[1], v[2], v[3]);
        else *(uint2 *)o = make_uint2((uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16), (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
    } else {
        for (int e = 0; e < g.n - col; ++e) store_f32<TOut>(o, e, v[e]);
    }
}

template <bool kSwiglu, int MT, int WT, int KW, int D, typename TOut>
__global__ __launch_bounds__(kThreads) void k_four_stream(FourGemm g, int slices)
{
    constexpr int LT = kSwiglu ? 2 * WT : WT, NW = kWaves / KW;
    constexpr int STRIDE = LT * 16 + 4;                        // floats of a row's partial sums in LDS
    __shared__ float red[KW > 1 ? kWaves : 1][16][STRIDE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, quad = lane >> 4;
    const int kw = wave % KW, nw = wave / KW;
    const int group = blockIdx.x / slices, slice = blockIdx.x - group * slices;
    const int n0 = (slice * NW + nw) * WT * 16;                // this wavefront's first column
    int lo = 0, hi = g.m;
    if (g.offsets) {
        lo = max(g.offsets[group], 0);
        hi = min(g.offsets[group + 1], g.m);
    }
    const int steps = (g.k + kFourStep - 1) / kFourStep;
    const size_t w_rows = (size_t)(kSwiglu ? 2 : 1) * g.n;
    const uint8_t *wp[LT], *sp[LT];
#pragma unroll
    for (int t = 0; t < LT; ++t) {
        const size_t row = (size_t)group * w_rows + (size_t)(t / WT) * g.n + min(n0 + t % WT * 16 + l15, g.n - 1);
        wp[t] = g.w + row * (g.k / 2) + quad * 16;
        sp[t] = g.ws + row * (g.k / kFourGroup) + quad;
    }
    for (int r0 = lo + (int)blockIdx.y * MT * 16; r0 < hi; r0 += (int)gridDim.y * MT * 16) {
        const int rows = min(MT * 16, hi - r0), live = (rows + 15) >> 4;
        const uint16_t *ap[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) ap[m] = g.a + (size_t)(r0 + min(m * 16 + l15, rows - 1)) * g.ld_a + quad * 32;
        f32x4 acc[LT][MT];
#pragma unroll
        for (int t = 0; t < LT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[t][m] = (f32x4){0.f, 0.f, 0.f, 0.f};
        u32x4 wf[D][LT], af[D][MT][4];
        uint32_t sf[D][LT];
        auto request = [&](int d, int b) __attribute__((always_inline)) {
            const bool in = b * kFourStep + quad * kFourGroup < g.k;       // a step that ends behind the row: zeros
#pragma unroll
            for (int t = 0; t < LT; ++t) {
                wf[d][t] = (u32x4){0, 0, 0, 0};
                sf[d][t] = 0;
                if (in) {
                    wf[d][t] = *(const u32x4 *)(wp[t] + (size_t)b * (kFourStep / 2));
                    sf[d][t] = sp[t][(size_t)b * (kFourStep / kFourGroup)];
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
                if (m < live)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        af[d][m][i] = (u32x4){0, 0, 0, 0};
                        if (in) af[d][m][i] = *(const u32x4 *)(ap[m] + (size_t)b * kFourStep + i * 8);
                    }
        };
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (kw + d * KW < steps) request(d, kw + d * KW);
        for (int b0 = kw; b0 < steps; b0 += D * KW) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                const int b = b0 + d * KW;
                if (b < steps) {
#pragma unroll
                    for (int t = 0; t < LT; ++t) {
                        const float power = __uint_as_float(sf[d][t] << 23);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const bf16x8 w = weights8(wf[d][t][i], power);
#pragma unroll
                            for (int m = 0; m < MT; ++m)
                                if (m < live) acc[t][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, af[d][m][i]), acc[t][m], 0, 0, 0);
                        }
                    }
                    if (b + D * KW < steps) request(d, b + D * KW);
                }
            }
        }
        if constexpr (KW == 1) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
                if (m * 16 + l15 < rows)
#pragma unroll
                    for (int t = 0; t < WT; ++t) {
                        const int col = n0 + t * 16 + quad * 4;
                        if (col < g.n) finish<kSwiglu, TOut>(g, r0 + m * 16 + l15, col, acc[t][m], acc[kSwiglu ? t + WT : t][m]);
                    }
        } else {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (m >= live) break;
                if (m > 0) __syncthreads();
#pragma unroll
                for (int t = 0; t < LT; ++t) *(f32x4 *)&red[wave][l15][t * 16 + quad * 4] = acc[t][m];
                __syncthreads();
                const int mine = min(16, rows - m * 16);
                for (int i = threadIdx.x; i < NW * 16 * WT * 4; i += kThreads) {
                    const int c4 = i % (WT * 4) * 4, row = i / (WT * 4) % 16, of = i / (WT * 64);
                    const int col = (slice * NW + of) * WT * 16 + c4;
                    if (row >= mine || col >= g.n) continue;
                    f32x4 s[kSwiglu ? 2 : 1];
#pragma unroll
                    for (int h = 0; h < (kSwiglu ? 2 : 1); ++h) {
                        s[h] = *(const f32x4 *)&red[of * KW][row][h * WT * 16 + c4];
#pragma unroll
                        for (int w = 1; w < KW; ++w) s[h] += *(const f32x4 *)&red[of * KW + w][row][h * WT * 16 + c4];
                    }
                    finish<kSwiglu, TOut>(g, r0 + m * 16 + row, col, s[0], s[kSwiglu ? 1 : 0]);
                }
            }
            __syncthreads();
        }
    }
}

template <bool kSwiglu, int MT, int WT, int KW, int D, typename TOut>
void launch_as(const FourGemm &g, int row_tiles, hipStream_t st)
{
    const int per = kWaves / KW * WT * 16, slices = (g.n + per - 1) / per;
    // workgroups go on to further row tiles of theirs where a launch could not have one for each
    const long long most = kMostGroups / ((long long)slices * g.groups);
    row_tiles = (int)(most < row_tiles ? most : row_tiles);
    row_tiles = row_tiles < 1 ? 1 : row_tiles > 65535 ? 65535 : row_tiles;
    hipLaunchKernelGGL((k_four_stream<kSwiglu, MT, WT, KW, D, TOut>), dim3(slices * g.groups, row_tiles), dim3(kThreads), 0, st, g, slices);
}

template <bool kSwiglu, typename TOut>
void launch_for(const FourGemm &g, hipStream_t st)
{
    const int each = (g.m + g.groups - 1) / g.groups;          // rows of a group, on average
    if (each <= 16) launch_as<kSwiglu, 1, 1, 8, 2, TOut>(g, g.groups > 1 ? min(2, (g.m + 15) / 16) : (g.m + 15) / 16, st);
    else            launch_as<kSwiglu, 2, 1, 8, 1, TOut>(g, g.groups > 1 ? (2 * each + 31) / 32 : (g.m + 31) / 32, st);
}

}  // namespace

bool four_product_fits(const FourGemm &g)
{
    return (g.n + 15ll) / 16 * g.groups <= kMostGroups;
}

hipError_t launch_four_product(const FourGemm &g, bool swiglu, bool out_bf16, hipStream_t st)
{
    if (swiglu && out_bf16) launch_for<true, uint16_t>(g, st);
    else if (swiglu)        launch_for<true, float>(g, st);
    else if (out_bf16)      launch_for<false, uint16_t>(g, st);
    else                    launch_for<false, float>(g, st);
    return hipGetLastError();
}

}  // namespace emoe
