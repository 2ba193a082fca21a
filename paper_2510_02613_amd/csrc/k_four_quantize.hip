// Rows of values -> e2m1 codes and a power of two per 32 columns.
//
//   p = the smallest power with max |v| <= 6 * 2^p,  code = v / 2^p to the nearest, ties to the even code
//
// With the maximum's exponent field E and mantissa field m, 6 * 2^p = 1.5 * 2^(p + 2): the power's byte is E - 2, one more where m > 0.5.  The conversion
// instructions divide by the power exactly, round to nearest even and keep signs.
// A thread has eight columns, four neighbouring lanes a group: one pass over the row, a wide load a thread, no LDS.
// Bound by the rows read and written: 4096 x 7168 fp32 with values, 251 MB, 37 us on the GPU (6.7 TB/s, part of them from the caches), 1536 x 2048 bf16 3.3 us.
#include "four_bit.h"

namespace emoe {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

template <typename T>
__device__ __forceinline__ void load8(const char *p, float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        const u32x4 r = *(const u32x4 *)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(r[i] << 16); v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u); }
    } else {
        const u32x4 r = *(const u32x4 *)p, s = *(const u32x4 *)(p + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(r[i]); v[4 + i] = __uint_as_float(s[i]); }
    }
}

// maximum over four neighbouring lanes, in all of them
__device__ __forceinline__ uint32_t lanes4_max(uint32_t v)
{
#define EMOE_DPP(ctrl) { const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false); v = o > v ? o : v; }
    EMOE_DPP(0xb1) EMOE_DPP(0x4e)
#undef EMOE_DPP
    return v;
}

// A wavefront's run is 64 threads' columns (512) of a row.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_four_quantize(FourRows j, int runs)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long items = (long long)j.rows * runs;
    for (long long item = (long long)blockIdx.x * kWaves + wave; item < items; item += (long long)gridDim.x * kWaves) {
        const int64_t r = item / runs;
        const int c = (int)(item - r * runs) * 64 + lane;         // of cols / 8
        if (c * 8 >= j.cols) continue;
        float v[8];
        load8<T>(j.x + r * j.ld_x + (int64_t)c * 8 * sizeof(T), v);
        uint32_t top = 0;                                        // magnitudes as integers: a NaN is larger than all else
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
            top = a > top ? a : top;
        }
        top = lanes4_max(top);
        const bool finite = top < 0x7f800000u;
        const int byte = finite ? max(0, (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u)) : 255;
        const float power = __uint_as_float((uint32_t)byte << 23);   // byte 0 is read as 2^-127
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], power, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], power, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], power, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], power, 3);
        if (!finite) q = 0;
        *(uint32_t *)(j.q + r * j.ld_q + (int64_t)c * 4) = q;
        if ((lane & 3) == 0) j.scale[r * j.ld_scale + c / 4] = (uint8_t)byte;
        if (j.values) {
            char *o = j.values + r * j.ld_values + (int64_t)c * 8 * sizeof(T);
            f32x2 f[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, power, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, power, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, power, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, power, 3)};
            u32x4 lo, hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2) lo[i] = (__float_as_uint(f[i][0]) >> 16) | (__float_as_uint(f[i][1]) & 0xffff0000u);   // exact: short numbers
                else if (i < 2) { lo[2 * i] = __float_as_uint(f[i][0]); lo[2 * i + 1] = __float_as_uint(f[i][1]); }
                else { hi[2 * i - 4] = __float_as_uint(f[i][0]); hi[2 * i - 3] = __float_as_uint(f[i][1]); }
            }
            *(u32x4 *)o = lo;
            if constexpr (sizeof(T) == 4) *(u32x4 *)(o + 16) = hi;
        }
    }
}

}  // namespace

hipError_t launch_four_quantize(const FourRows &j, bool bf16, hipStream_t st)
{
    const int runs = (j.cols / 8 + 63) / 64;
    const long long groups = ((long long)j.rows * runs + kWaves - 1) / kWaves;
    const dim3 grid((unsigned)(groups < 1 << 20 ? groups : 1 << 20));
    if (bf16) hipLaunchKernelGGL(k_four_quantize<uint16_t>, grid, dim3(kThreads), 0, st, j, runs);
    else      hipLaunchKernelGGL(k_four_quantize<float>, grid, dim3(kThreads), 0, st, j, runs);
    return hipGetLastError();
}

}  // namespace emoe
