// Un-permute and weighted combine of a layer with 8-bit experts: out[t] = sum_j w[t,j] y[inv[t,j]], in selection order (shared experts last, weight 1),
// in fp32 with one rounding at the end.  y are fp32 rows, or, in passes that take the 8-bit
// matrix instructions, 16-bit rows with a scale per 64 columns (Block16 in scaled.h).
//
// A workgroup owns one token and every gridDim.y-th run of 256 chunks of 8 columns.  Bound by memory: the rows of four assignments are
// requested before any is added.
#include "scaled.h"

namespace emoe {
namespace {

constexpr int kMaxKK = 36;   // top_k <= 32 plus <= 4 shared experts

template <bool kF32>
__global__ __launch_bounds__(256) void k_scaled_combine(Pass p, const float *scales)
{
    __shared__ int32_t rows[kMaxKK];
    __shared__ float wts[kMaxKK];
    __shared__ int32_t n_local;
    const int t = blockIdx.x;
    if (threadIdx.x < 64) {   // first wavefront: the token's local assignments, compacted, still in selection order
        const int j = threadIdx.x;
        int r = -1;
        float wv = 0.f;
        if (j < p.kk) {
            r = p.inv[(size_t)t * p.kk + j];
            wv = j < p.k ? p.w[(size_t)t * p.k + j] : 1.0f;
        }
        const unsigned long long m = __ballot(r >= 0);
        if (r >= 0) {
            const int at = __popcll(m & ((1ull << j) - 1ull));
            rows[at] = r;
            wts[at] = wv;
        }
        if (j == 0) n_local = __popcll(m);
    }
    __syncthreads();
    const int n = n_local, groups = scaled_out_groups(p.H);
    for (int c = (blockIdx.y * 256 + threadIdx.x) * 8; c < p.H; c += gridDim.y * 256 * 8) {
        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int i0 = 0; i0 < n; i0 += 4) {
            uint4 v[4][kF32 ? 2 : 1];
            float s[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i0 + u < n) {
                    const size_t r = rows[i0 + u];
                    if (kF32) {
                        v[u][0] = *(const uint4 *)((const float *)p.y + r * p.H + c);
                        v[u][kF32 ? 1 : 0] = *(const uint4 *)((const float *)p.y + r * p.H + c + 4);
                        s[u] = wts[i0 + u];
                    } else {
                        v[u][0] = *(const uint4 *)((const uint16_t *)p.y + r * p.H + c);
                        s[u] = wts[i0 + u] * scales[r * groups + (c >> 6)];
                    }
                }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i0 + u < n) {
                    const uint32_t a[4] = {v[u][0].x, v[u][0].y, v[u][0].z, v[u][0].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (kF32) {
                            const uint4 &h = v[u][kF32 ? 1 : 0];
                            const uint32_t b[4] = {h.x, h.y, h.z, h.w};
                            acc[e] = fmaf(s[u], __uint_as_float(a[e]), acc[e]);
                            acc[4 + e] = fmaf(s[u], __uint_as_float(b[e]), acc[4 + e]);
                        } else {
                            acc[2 * e] = fmaf(s[u], (float)(int16_t)(a[e] & 0xffffu), acc[2 * e]);
                            acc[2 * e + 1] = fmaf(s[u], (float)((int32_t)a[e] >> 16), acc[2 * e + 1]);
                        }
                    }
                }
        }
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (uint32_t)f32_to_bf16(acc[2 * e]) | ((uint32_t)f32_to_bf16(acc[2 * e + 1]) << 16);
        *(uint4 *)((uint16_t *)p.out + (size_t)t * p.H + c) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

}  // namespace

hipError_t launch_scaled_combine(const Pass &p, const float *scales, hipStream_t st)
{
    // a row is shared out over several workgroups only while there are too few tokens to fill the chip
    const int ny = p.T >= 1024 ? 1 : (p.H + 2047) / 2048;
    if (scales) hipLaunchKernelGGL((k_scaled_combine<false>), dim3(p.T, ny), dim3(256), 0, st, p, scales);
    else        hipLaunchKernelGGL((k_scaled_combine<true>), dim3(p.T, ny), dim3(256), 0, st, p, scales);
    return hipGetLastError();
}

}  // namespace emoe
