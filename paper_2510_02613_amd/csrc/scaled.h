// Internal declarations of the 8-bit path: e4m3 values with fp32 scales, one for each row and 128 columns of an
// activation, one for each block of 128 x 128 of a weight matrix.
#pragma once
#include "elasticmoe_scaled.h"
#include "moe_internal.h"

namespace emoe {

constexpr int kScaleBlock = 128;             // columns (and weight rows) that share a scale: one K-step of the products
constexpr float kE4m3Top = 448.f;            // the largest e4m3 value
constexpr float kZeroGroup = 0x1p-110f;      // a group whose largest magnitude is below this counts as zero (its quotients would leave fp32)
__host__ __device__ constexpr int scale_blocks(int n) { return (n + kScaleBlock - 1) / kScaleBlock; }
__host__ __device__ constexpr int scaled_out_groups(int n) { return (n + 63) / 64; }   // of a row of expert outputs

// Rows of values -> their norm, their sum with a residual, their 8-bit form.
struct RowsJob {
    int32_t rows, cols;
    int32_t norm;                 // 0: the rows are quantised as they are
    float eps;
    const void *x, *residual, *weight;
    void *sum, *out;
    uint8_t *q;
    float *scale;
    int64_t ld_x, ld_residual, ld_sum, ld_out, ld_q, ld_scale;
};
hipError_t launch_rows(const RowsJob &j, bool bf16, hipStream_t st);                 // cols % 8 == 0, cols <= kMaxRowCols
hipError_t launch_quantize_blocks(const RowsJob &j, bool bf16, hipStream_t st);      // scale [ceil(rows/128)][ld_scale]
constexpr int kMaxRowCols = 32768;
hipError_t launch_fill_scales(float *dst13, const float *src13, size_t n13, float *dst2, const float *src2, size_t n2, hipStream_t st);

// A product of 8-bit rows with 8-bit weights: out[r, c] = sum_b as[r, b] ws[c / 128, b] sum_{k in b} a[r, k] w[c, k].
struct SGemm {
    const uint8_t *a;             // rows of ld_a bytes
    const float *as;              // rows of ld_as scales
    int64_t ld_a, ld_as;
    const uint8_t *w;             // [n][k], with swiglu [2n][k]: gate rows, then up rows
    const float *ws;              // [blocks of n (gate, then up)][kb]
    size_t w_slot, ws_slot;       // elements from one slot to the next (tile lists)
    int32_t m, n, k, kb;          // rows (no tile list), output columns, contraction, its blocks
    // a tile list: tile i is tiles[i].rows rows of slot tiles[i].slot; row r of the list is row perm[r] of a (perm NULL: row r)
    const MTile *tiles;
    const int32_t *n_tiles;
    const int32_t *perm;
    int32_t max_tiles;
    int32_t together;             // tiles that share weights and are worked on side by side
    int32_t split_tail;           // the rows of a last round that is not full may be shared out to more workgroups
    // result rows; with swiglu silu(gate) * up
    void *out;
    int64_t ld_out;
    const void *add;              // NULL, or rows of out's type that are added
    int64_t ld_add;
    float *os;                    // scales of block16 rows
    int64_t ld_os;
    uint8_t *q;                   // swiglu of the large tiles: 8-bit rows and their scales in the place of out
    float *qs;
    int64_t ld_q, ld_qs;
};
// few rows: the weights are streamed; out fp32 or bf16, swiglu: fp32 rows h.  Tiles of 16 or 32 rows.
hipError_t launch_scaled_stream(const SGemm &g, bool swiglu, bool out_bf16, int tile_rows, hipStream_t st);
int stream_tile_rows(int m, int n, bool swiglu);
// many rows: tiles of up to 128 rows with exact products; with the 8-bit matrix instructions (fast_bf16, a layer's block16 and swiglu) of up to 256.
enum class TilesOut { bf16, f32, swiglu_exact, fast_bf16, block16, swiglu };
int tiles_slices(int n, bool swiglu);       // workgroups a tile's weight rows are shared out to
double tiles_us(long long tiles, int tile_rows, int n, int k, bool swiglu, bool exact);   // what a launch takes, roughly
hipError_t launch_scaled_tiles(const SGemm &g, TilesOut out, int tile_rows, hipStream_t st);
// the weighted sum of a layer's expert outputs p.y: fp32 rows (scales NULL), or block16 rows with scales [rows][ceil(H/64)]
hipError_t launch_scaled_combine(const Pass &p, const float *scales, hipStream_t st);

#ifdef __HIPCC__
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A lane's share of 16 rows x 128 columns of e4m3: 32 bytes of one row, lane (quad, l15) those of row l15.
struct Bytes32 { uint4 lo, hi; };
__device__ __forceinline__ i32x8 operand(const Bytes32 &f)
{
    return (i32x8){(int)f.lo.x, (int)f.lo.y, (int)f.lo.z, (int)f.lo.w, (int)f.hi.x, (int)f.hi.y, (int)f.hi.z, (int)f.hi.w};
}
// the same as bf16, which holds every e4m3 value
struct Bf16x32 {
    bf16x8 v[4];
    template <int quarter>                       // 8 of the 32
    __device__ __forceinline__ void from_quarter(const Bytes32 &f)
    {
        const uint4 &h = quarter < 2 ? f.lo : f.hi;
        const uint32_t w[2] = {quarter & 1 ? h.z : h.x, quarter & 1 ? h.w : h.y};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, true);
            v[quarter][4 * i] = a[0]; v[quarter][4 * i + 1] = a[1];
            v[quarter][4 * i + 2] = b[0]; v[quarter][4 * i + 3] = b[1];
        }
    }
    __device__ __forceinline__ void from(const Bytes32 &f)
    {
        from_quarter<0>(f); from_quarter<1>(f); from_quarter<2>(f); from_quarter<3>(f);
    }
};
// 16 x 16 sums of 128 products.  The 8-bit matrix instructions add products in groups of eight and drop of each what lies
// 2^-14 and more below the largest, whatever the accumulator's type: 1.5e-5 of the result's norm on normal values, 6e-5 on values spread over
// six binades, where a rounding to bf16 is up to 2^-8 of a value; but where large products cancel, all of what is left.  So they run only where the caller
// asks for them (multiply_fast), and everything else comes from the bf16 instructions, at half the rate, whose products of e4m3
// values are exact and whose sums are fp32's (multiply_exact).
__device__ __forceinline__ f32x4 multiply_fast(const Bytes32 &a, const Bytes32 &b)
{
    const f32x4 z = {0.f, 0.f, 0.f, 0.f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), z, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply_exact(const Bf16x32 &a, const Bf16x32 &b)
{
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], s, 0, 0, 0);
    return s;
}

// 448 v / a for the group maximum a, correctly rounded where the quotient is short: numbers of few bits meet the half-way points
// between two e4m3 values often, and the rounding to 8 bits has to see them as such.  0.875 v is exact for bf16 v; one
// Newton step makes up for the reciprocal's last bit.
struct GroupScale {
    float a, r;
    __device__ __forceinline__ explicit GroupScale(float top)
    {
        const bool zero = top < kZeroGroup;
        a = zero ? 0.f : top * 0x1p-9f;
        r = zero ? 0.f : __builtin_amdgcn_rcpf(a);
    }
    __device__ __forceinline__ float quotient(float v) const
    {
        const float y = 0.875f * v, t = y * r;
        return fmaf(fmaf(-a, t, y), r, t);
    }
    static __device__ __forceinline__ float scale(float top) { return top < kZeroGroup ? 0.f : top / kE4m3Top; }
};
// four e4m3 values in a word, round to nearest even; |v| <= 448 by the choice of the scale
__device__ __forceinline__ uint32_t pack_e4m3(float v0, float v1, float v2, float v3)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v0, v1, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v2, v3, w, true);
}
// magnitudes are compared as integers: a NaN is then larger than all else and makes its whole group NaN, whatever the order
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// Expert outputs between the second GEMM and the weighted sum in a pass whose caller takes the 8-bit matrix instructions: 16-bit whole numbers with one fp32 scale, largest magnitude / 32767, for 64 columns of
// a row.  As many bytes as bf16 and 30 times less rounding (5e-5 of normal values' norm against 1.7e-3): what comes behind, the weighted sum in fp32, is then
// rounded once, at the end.  A group that holds a NaN or an infinity is NaN throughout.
struct Block16 { uint16_t v; };
struct Block16Scale {
    float scale, r;
    __device__ __forceinline__ explicit Block16Scale(float top) : scale(top * (1.f / 32767.f)), r(top < kZeroGroup ? 0.f : 32767.f / top) {}
    __device__ __forceinline__ uint32_t pack(float a, float b) const
    {
        return ((uint32_t)__float2int_rn(a * r) & 0xffffu) | ((uint32_t)__float2int_rn(b * r) << 16);
    }
};
// maximum over 8 neighbouring lanes, in all of them
__device__ __forceinline__ uint32_t lanes8_max(uint32_t v)
{
#define EMOE_DPP(ctrl) { const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false); v = o > v ? o : v; }
    EMOE_DPP(0xb1) EMOE_DPP(0x4e) EMOE_DPP(0x141)      // lanes 1 and 2 apart, then mirrored in the half row
#undef EMOE_DPP
    return v;
}
// maximum over the 16 lanes of a DPP row, in all of them
__device__ __forceinline__ uint32_t row16_max(uint32_t v)
{
#define EMOE_ROR(n) { const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + n, 0xf, 0xf, false); v = o > v ? o : v; }
    EMOE_ROR(8) EMOE_ROR(4) EMOE_ROR(2) EMOE_ROR(1)
#undef EMOE_ROR
    return v;
}
#endif

}  // namespace emoe
