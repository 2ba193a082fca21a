// What the kernels of the 4-bit products share: operands, the last step of a result.
#pragma once
#include "four_bit.h"

namespace emoe {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// eight weights: four bytes of codes times the power whose bits these are
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

// eight neighbouring columns of a row, bf16
template <bool kSwiglu>
__device__ __forceinline__ void finish8(const FourGemm &g, size_t r, int col, const f32x4 &s0, const f32x4 &s1, const f32x4 &u0, const f32x4 &u1)
{
    u32x4 o, add = {0, 0, 0, 0};
    if (!kSwiglu && g.add) add = *(const u32x4 *)((const uint16_t *)g.add + r * g.ld_add + col);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int e = (2 * i + h) % 4;
            const float s = i < 2 ? s0[e] : s1[e];
            v[h] = kSwiglu ? silu_mul(s, i < 2 ? u0[e] : u1[e]) : s;
            if (!kSwiglu && g.add) v[h] += __uint_as_float(h ? add[i] & 0xffff0000u : add[i] << 16);
        }
        o[i] = (uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16);
    }
    *(u32x4 *)((uint16_t *)g.out + r * g.ld_out + col) = o;
}

}  // namespace emoe
