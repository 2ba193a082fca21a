// RMS norm with the residual's addition, and quantising to e4m3.
//
//   r = x + residual,  y = r / sqrt(mean(r^2) + eps) * weight,
//   per 128 columns: a = max |y|, scale = a / 448, q = e4m3(448 y / a)
//
// A row stays in registers from its one reading to its last writing; r and y are not rounded on the way: the stored sum, the
// stored norm and the 8-bit values are each one rounding away from fp32.  Bound by memory: 8 operations an element against
// 3 to 9 bytes.  A lane holds chunks of 8 consecutive elements (16 bytes of bf16, whole lines per wavefront), so a group of 128
// columns is 16 lanes, one DPP row: its maximum takes four lane rotations and no shared memory.
#include "scaled.h"
#include "wave_ops.h"

namespace emoe {
namespace {

template <typename T> struct Vec8;   // 8 elements as they travel
template <> struct Vec8<uint16_t> {
    uint4 v;
    __device__ __forceinline__ void load(const uint16_t *p) { v = *(const uint4 *)p; }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ void put(uint16_t *p, const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16(f[2 * i]) | ((uint32_t)f32_to_bf16(f[2 * i + 1]) << 16);
        *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) { a = *(const float4 *)p; b = *(const float4 *)(p + 4); }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    static __device__ __forceinline__ void put(float *p, const float (&f)[8])
    {
        *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
        *(float4 *)(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
    }
};

// kWaves wavefronts per row, kChunks chunks of 8 elements per lane.  One wavefront a row: four rows share a workgroup.
template <typename T, int kWaves, int kChunks>
__global__ __launch_bounds__(kWaves == 1 ? 256 : kWaves * 64) void k_rows(RowsJob j)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = kWaves == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
    const int tid = kWaves == 1 ? lane : threadIdx.x;
    if (row >= j.rows) return;                       // whole wavefronts, and with several a row whole workgroups
    const int n = j.cols >> 3;                       // chunks of the row
    const T *x = (const T *)j.x + (size_t)row * j.ld_x;
    const T *res = j.residual ? (const T *)j.residual + (size_t)row * j.ld_residual : nullptr;
    Vec8<T> vx[kChunks], vr[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = tid + i * kWaves * 64;
        if (c < n) vx[i].load(x + c * 8);
    }
    if (res) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int c = tid + i * kWaves * 64;
            if (c < n) vr[i].load(res + c * 8);
        }
    }
    float v[kChunks][8];
    float sq = 0.f, scale_in = 1.f, eps = j.eps;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = tid + i * kWaves * 64;
        if (c < n) {
            vx[i].get(v[i]);
            if (res) {
                float r[8];
                vr[i].get(r);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] += r[e];
            }
            if (j.norm)
#pragma unroll
                for (int e = 0; e < 8; ++e) sq = fmaf(v[i][e], v[i][e], sq);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
    }
    if (j.norm) {
        sq = wave_sum_f32(sq);
        if (kWaves > 1) {
            __shared__ float part[kWaves > 1 ? kWaves : 1];
            if (lane == 0) part[wave] = sq;
            __syncthreads();                          // everyone has read its share of x and residual: sum and out may be those rows
            sq = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sq += part[w];
        }
    }
    if (j.norm) {
        // Squares that leave fp32 (magnitudes above some 2^63 / sqrt(cols); below 2^-60 where eps does not outweigh them): once more, of the row times the
        // power of two that brings its largest number to 1 .. 4.  The same for all wavefronts of the row: they all have its sum.
        // (The question costs one row of 7168 3.2 -> 3.4 us, 1024 rows 12.8 -> 13.0, 8192 nothing.)
        const float mean = sq / (float)j.cols + eps;
        if (mean < 0x1p-120f || mean == __builtin_inff()) {
            __shared__ uint32_t tops[kWaves];
            __shared__ float again[kWaves];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < kChunks; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[i][e]));
            top = wave_max_u32(top);
            if (kWaves > 1) {
                if (lane == 0) tops[wave] = top;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kWaves; ++w) top = max(top, tops[w]);
            }
            const uint32_t exponent = min(max(top >> 23, 1u), 253u);
            const float s = __uint_as_float((254u - exponent) << 23);
            if (top != 0 && top < 0x7f800000u && eps * s * s < __builtin_inff()) {      // no zeros, infinities or NaN, nor an eps that outweighs the row
                sq = 0.f;
#pragma unroll
                for (int i = 0; i < kChunks; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sq = fmaf(v[i][e] * s, v[i][e] * s, sq);
                sq = wave_sum_f32(sq);
                if (kWaves > 1) {
                    if (lane == 0) again[wave] = sq;
                    __syncthreads();
                    sq = 0.f;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) sq += again[w];
                }
                scale_in = s;
                eps = eps * s * s;
            }
        }
    }
    const float rstd = j.norm ? 1.f / sqrtf(sq / (float)j.cols + eps) : 1.f;
    const T *weight = (const T *)j.weight;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = tid + i * kWaves * 64;
        if (c - (tid & 15) >= n) continue;            // no chunk of this DPP row exists
        const bool live = c < n;
        if (j.sum && live) Vec8<T>::put((T *)j.sum + (size_t)row * j.ld_sum + c * 8, v[i]);
        if (j.norm) {
            float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            if (weight && live) {
                Vec8<T> vw;
                vw.load(weight + c * 8);
                vw.get(w);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * scale_in * rstd * w[e];
        }
        if (j.out && live) Vec8<T>::put((T *)j.out + (size_t)row * j.ld_out + c * 8, v[i]);
        if (j.q) {
            uint32_t top = 0;
            if (live)
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[i][e]));
            const float a = __uint_as_float(row16_max(top));
            const GroupScale s(a);
            if (live) {
                uint2 o;
                o.x = pack_e4m3(s.quotient(v[i][0]), s.quotient(v[i][1]), s.quotient(v[i][2]), s.quotient(v[i][3]));
                o.y = pack_e4m3(s.quotient(v[i][4]), s.quotient(v[i][5]), s.quotient(v[i][6]), s.quotient(v[i][7]));
                *(uint2 *)(j.q + (size_t)row * j.ld_q + c * 8) = o;
                if ((c & 15) == 0) j.scale[(size_t)row * j.ld_scale + (c >> 4)] = GroupScale::scale(a);
            }
        }
    }
}

// One workgroup per block of 128 x 128: 16 lanes a row of 128 columns, 8 rows a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_blocks(RowsJob j)
{
    const int lane16 = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const int col = blockIdx.x * kScaleBlock + lane16 * 8, row0 = blockIdx.y * kScaleBlock + r0;
    const bool live = col < j.cols;
    float v[8][8];
    Vec8<T> in[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (live && row0 + 16 * i < j.rows) in[i].load((const T *)j.x + (size_t)(row0 + 16 * i) * j.ld_x + col);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (live && row0 + 16 * i < j.rows) {
            in[i].get(v[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, magnitude(v[i][e]));
        }
    __shared__ uint32_t part[4];
    top = wave_max_u32(top);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    const float a = __uint_as_float(max(max(part[0], part[1]), max(part[2], part[3])));
    const GroupScale s(a);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (live && row0 + 16 * i < j.rows) {
            uint2 o;
            o.x = pack_e4m3(s.quotient(v[i][0]), s.quotient(v[i][1]), s.quotient(v[i][2]), s.quotient(v[i][3]));
            o.y = pack_e4m3(s.quotient(v[i][4]), s.quotient(v[i][5]), s.quotient(v[i][6]), s.quotient(v[i][7]));
            *(uint2 *)(j.q + (size_t)(row0 + 16 * i) * j.ld_q + col) = o;
        }
    if (threadIdx.x == 0) j.scale[(size_t)blockIdx.y * j.ld_scale + blockIdx.x] = GroupScale::scale(a);
}

// the scales of one slot (14 KB for the largest experts): a few workgroups move them word by word
__global__ __launch_bounds__(256) void k_fill_scales(float *dst13, const float *src13, size_t n13, float *dst2, const float *src2, size_t n2)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n13 + n2; i += (size_t)gridDim.x * 256) {
        if (i < n13) dst13[i] = src13[i];
        else         dst2[i - n13] = src2[i - n13];
    }
}

template <typename T, int kWaves>
void launch_rows_of(const RowsJob &j, hipStream_t st)
{
    const int chunks = ((j.cols >> 3) + kWaves * 64 - 1) / (kWaves * 64);
    const dim3 grid(kWaves == 1 ? (j.rows + 3) / 4 : j.rows), block(kWaves == 1 ? 256 : kWaves * 64);
    if (chunks <= 1) hipLaunchKernelGGL((k_rows<T, kWaves, 1>), grid, block, 0, st, j);
    else if (kWaves == 1 || chunks <= 2) hipLaunchKernelGGL((k_rows<T, kWaves, 2>), grid, block, 0, st, j);
    else if constexpr (kWaves > 1) hipLaunchKernelGGL((k_rows<T, kWaves, 4>), grid, block, 0, st, j);
}

template <typename T>
void launch_rows_t(const RowsJob &j, hipStream_t st)
{
    const int chunks = j.cols >> 3;
    // up to two workgroups a compute unit a row is shared out to more wavefronts: less in a row for each of them.  us, norm with all results / quantising, rows
    // of 7168: 1 row 5.2 / 3.6 -> 3.9 / 2.9, 64 5.7 / 3.9 -> 4.3 / 3.1, 512 8.7 / 4.7 -> 7.9 / 4.1, 1024 13.4 / 6.3 -> 14.0 / 5.7, 2048 21.0 -> 22.8; of
    // 4096: 1 3.9 -> 3.4, 512 5.9 -> 5.9, 2048 13.4 -> 15.3; of 768: 1 3.5 -> 3.1, 512 4.2 -> 3.7, 2048 5.4 -> 5.6
    const bool few = j.rows <= 512;
    if (chunks <= (few ? 64 : 128))        launch_rows_of<T, 1>(j, st);
    else if (chunks <= (few ? 256 : 1024)) launch_rows_of<T, 4>(j, st);
    else                                   launch_rows_of<T, 16>(j, st);
}

}  // namespace

hipError_t launch_rows(const RowsJob &j, bool bf16, hipStream_t st)
{
    if (j.rows == 0) return hipSuccess;
    if (bf16) launch_rows_t<uint16_t>(j, st);
    else      launch_rows_t<float>(j, st);
    return hipGetLastError();
}

hipError_t launch_fill_scales(float *dst13, const float *src13, size_t n13, float *dst2, const float *src2, size_t n2, hipStream_t st)
{
    hipLaunchKernelGGL(k_fill_scales, dim3(8), dim3(256), 0, st, dst13, src13, n13, dst2, src2, n2);
    return hipGetLastError();
}

hipError_t launch_quantize_blocks(const RowsJob &j, bool bf16, hipStream_t st)
{
    if (j.rows == 0) return hipSuccess;
    const dim3 grid(scale_blocks(j.cols), scale_blocks(j.rows));
    if (bf16) hipLaunchKernelGGL((k_quantize_blocks<uint16_t>), grid, dim3(256), 0, st, j);
    else      hipLaunchKernelGGL((k_quantize_blocks<float>), grid, dim3(256), 0, st, j);
    return hipGetLastError();
}

}  // namespace emoe
