// Tokens sorted by expert and back: the order of the assignments, the tokens' rows in that order, their weighted sums, and the gradients.
//
//   g(a) = group of assignment a,  row(a) = #{a': g(a') < g(a)} + #{a' < a: g(a') = g(a)}
//   rows[row(a)] = x[a / k]        out[t] = sum_j w[t,j] y[row[t,j]]        dy[row[t,j]] = w[t,j] dout[t],  dw[t,j] = <dout[t], y[row[t,j]]>
//
// Assignments without a group count as group n_groups: their places are the rows behind the last one, so that "zero the rest" is a copy of zeros
// and every entry of source has exactly one writer.  Only counts are added by atomics; no place depends on their order.
// All kernels are bound by the rows they move.
#include "dispatch.h"
#include "wave_ops.h"

namespace emoe {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr long long kMostGroups = 1 << 20;   // workgroups of a launch: what is left is done by the same ones

__device__ __forceinline__ int group_of(const SortJob &s, int a)
{
    int g = s.ids[a];
    if (s.map) g = (unsigned)g < (unsigned)s.n_experts ? s.map[g] : -1;
    return (unsigned)g < (unsigned)s.n_groups ? g : s.n_groups;
}
// the assignments [lo, hi), shared out over the workgroup: their groups, eight of a thread on their way at once; f(a, g, whether there is one) by whole wavefronts
template <typename F>
__device__ __forceinline__ void each_group(const SortJob &s, int lo, int hi, F &&f)
{
    constexpr int U = 8;
    for (int a0 = lo + (threadIdx.x & ~63); a0 < hi; a0 += U * kThreads) {
        const int lane = threadIdx.x & 63;
        int g[U];
#pragma unroll
        for (int u = 0; u < U; ++u) g[u] = a0 + u * kThreads + lane < hi ? s.ids[a0 + u * kThreads + lane] : -1;
        if (s.map) {
#pragma unroll
            for (int u = 0; u < U; ++u) g[u] = (unsigned)g[u] < (unsigned)s.n_experts ? s.map[g[u]] : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (a0 + u * kThreads < hi) f(a0 + u * kThreads + lane, (unsigned)g[u] < (unsigned)s.n_groups ? g[u] : s.n_groups, a0 + u * kThreads + lane < hi);
    }
}
// Counts of assignments per group in LDS.  Those without a group, most of them where few experts are here, are added up by the wavefront first: additions to one
// address come one after the other (470 tokens of 7168 columns, one of eight assignments with a group: 24.6 -> 11.8 us).
struct Counter {
    int none = 0;
    __device__ __forceinline__ void add(int32_t *count, int g, bool is, int n_groups)
    {
        none += __popcll(__ballot(is && g == n_groups));
        if (is && g != n_groups) atomicAdd(&count[g], 1);
    }
    __device__ __forceinline__ void finish(int32_t *count, int n_groups) const
    {
        if ((threadIdx.x & 63) == 0 && none) atomicAdd(&count[n_groups], none);
    }
};

// counts of a block's assignments per group
__global__ __launch_bounds__(kThreads) void k_sort_count(SortJob s)
{
    extern __shared__ int32_t cnt[];      // [n_groups + 1]
    const int bins = s.n_groups + 1, A = s.tokens * s.top_k, a0 = blockIdx.x * kSortBlock;
    for (int g = threadIdx.x; g < bins; g += kThreads) cnt[g] = 0;
    __syncthreads();
    Counter c;
    each_group(s, a0, min(a0 + kSortBlock, A), [&](int, int g, bool is) { c.add(cnt, g, is, s.n_groups); });
    c.finish(cnt, s.n_groups);
    __syncthreads();
    for (int g = threadIdx.x; g < bins; g += kThreads) s.counts[(size_t)blockIdx.x * bins + g] = cnt[g];
}

// exclusive sums over the groups in place (LDS), total[bins] (+ more[bins]) -> first row of each group
__device__ __forceinline__ void scan_groups(int32_t *total, const int32_t *more, int bins, int32_t *scratch)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int carry = 0;
    for (int g0 = 0; g0 < bins; g0 += kThreads) {
        const int g = g0 + threadIdx.x;
        const int v = g < bins ? total[g] + (more ? more[g] : 0) : 0;
        const int incl = wave_incl_scan_i32(v);
        if (lane == 63) scratch[wave] = incl;
        __syncthreads();
        int base = carry;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) base += scratch[w];
            carry += scratch[w];
        }
        if (g < bins) total[g] = base + incl - v;
        __syncthreads();
    }
}

// One block's counts -> the place of its first assignment of every group: many assignments (more than the workgroups of k_sort_place add up
// themselves), one workgroup, block after block.  Bound by the latency of its loads: 65536 tokens, 8 rows of 4 KB each, 128 groups, 652 us for the sort, where
// adding up takes 515; 8 times the 59 us of 8192 tokens would be 475.
__global__ __launch_bounds__(kThreads) void k_sort_scan(SortJob s, int n_blocks)
{
    extern __shared__ int32_t total[];    // [n_groups + 1]
    __shared__ int32_t scratch[kWaves];
    const int bins = s.n_groups + 1;
    for (int g = threadIdx.x; g < bins; g += kThreads) {
        int sum = 0;
        for (int b = 0; b < n_blocks; ++b) sum += s.counts[(size_t)b * bins + g];
        total[g] = sum;
    }
    __syncthreads();
    scan_groups(total, nullptr, bins, scratch);
    for (int g = threadIdx.x; g < bins; g += kThreads) {
        int at = total[g];
        s.offsets[g] = at;
        for (int b = 0; b < n_blocks; ++b) {
            const size_t i = (size_t)b * bins + g;
            const int c = s.counts[i];
            s.counts[i] = at;
            at += c;
        }
    }
}

enum { kCountAll, kAddUp, kScanned };     // where the counts of the assignments in front come from

// A workgroup owns `per` tokens, at most 64 assignments, and every gridDim.y-th batch of `batch` runs of 64 16-byte columns of them: a wavefront has a batch of
// a token's row on its way (the first from the start, while the assignments are counted) and writes it row by row.  A run at a time, each of another token
// (and so of eight other rows): 5 us longer, 8192 tokens, 8 rows of 4 KB each, 302 MB, 63 us, 4.8 TB/s.  Stores that are not kept in the caches: 8 us less by
// themselves, but 8 more with the reader of the rows behind.
template <int kFrom>
__global__ __launch_bounds__(kThreads) void k_sort_place(SortJob s, int per, int batch, int n_blocks)
{
    extern __shared__ int32_t lds[];      // first[bins]: first rows of the groups, front[bins]: their assignments in front of this workgroup's
    __shared__ int32_t scratch[kWaves];
    __shared__ int32_t dest[64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int bins = s.n_groups + 1, A = s.tokens * s.top_k;
    const int t0 = blockIdx.x * per, nt = min(per, s.tokens - t0), a0 = t0 * s.top_k, mine = nt * s.top_k;
    int32_t *first = lds, *front = lds + bins;
    const int block = a0 / kSortBlock;
    constexpr int U = 4;                  // runs of a batch, at most
    const int runs = (s.chunks + 63) / 64, batches = (runs + batch - 1) / batch, items = nt * batches;
    u32x4 v[U];
    auto load = [&](int i) __attribute__((always_inline)) {
        const int t = i / batches, run = (i - t * batches) * batch;
        const char *from = s.x + (int64_t)(t0 + t) * s.ld_x;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = (run + u) * 64 + lane;
            if (u < batch && c < s.chunks) v[u] = *(const u32x4 *)(from + (int64_t)c * 16);
        }
    };
    const int stride = gridDim.y * kWaves, i0 = blockIdx.y * kWaves + wave;
    if (i0 < items) load(i0);
    const int g = wave == 0 && lane < mine ? group_of(s, a0 + lane) : -1;
    for (int g = tid; g < bins; g += kThreads) {
        first[g] = 0;
        front[g] = kFrom == kScanned ? s.counts[(size_t)block * bins + g] : 0;
    }
    __syncthreads();
    if (kFrom == kCountAll) {
        Counter before, behind;           // first: those behind for now
        each_group(s, 0, A, [&](int a, int g, bool is) {
            const unsigned long long out = __ballot(is && g == s.n_groups), in_front = __ballot(a < a0);
            before.none += __popcll(out & in_front);
            behind.none += __popcll(out & ~in_front);
            if (is && g != s.n_groups) atomicAdd(a < a0 ? &front[g] : &first[g], 1);
        });
        before.finish(front, s.n_groups);
        behind.finish(first, s.n_groups);
    } else {
        if (kFrom == kAddUp) {
            // all blocks' counts, four of a thread side by side and eight such on their way at once: other XCDs have just written them, a turn of waiting takes some 2 us
            // (a thread a group and block after block: 75 us where this takes 63)
            const int n = n_blocks * bins;
            const auto add = [&](int b, int g, int c) __attribute__((always_inline)) {
                if (c == 0) return;
                atomicAdd(&first[g], c);
                if (b < block) atomicAdd(&front[g], c);
            };
            constexpr int N = 8;
            for (int i0 = tid; i0 < n / 4; i0 += N * kThreads) {
                u32x4 c[N];
#pragma unroll
                for (int u = 0; u < N; ++u)
                    if (i0 + u * kThreads < n / 4) c[u] = *(const u32x4 *)(s.counts + (i0 + u * kThreads) * 4);
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    if (i0 + u * kThreads >= n / 4) break;
                    int b = (i0 + u * kThreads) * 4 / bins, g = (i0 + u * kThreads) * 4 - b * bins;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        add(b, g, (int)c[u][e]);
                        if (++g == bins) { g = 0; ++b; }
                    }
                }
            }
            if (tid < n % 4) {
                const int at = n - n % 4 + tid;
                add(at / bins, at % bins, s.counts[at]);
            }
        }
        Counter c;
        each_group(s, block * kSortBlock, a0, [&](int, int g, bool is) { c.add(front, g, is, s.n_groups); });
        c.finish(front, s.n_groups);
    }
    __syncthreads();
    if (kFrom != kScanned) {
        scan_groups(first, kFrom == kCountAll ? front : nullptr, bins, scratch);
        if (blockIdx.x == 0 && blockIdx.y == 0)
            for (int g = tid; g < bins; g += kThreads) s.offsets[g] = first[g];
    }
    if (wave == 0 && mine > 0) {
        // the lanes with the same group, bit by bit of its number
        unsigned long long same = __ballot(lane < mine);
        for (int b = 0; s.n_groups >> b; ++b) {
            const bool bit = (g >> b) & 1;
            const unsigned long long ones = __ballot(bit);
            same &= bit ? ones : ~ones;
        }
        if (lane < mine) {
            const int r = first[g] + front[g] + __popcll(same & ((1ull << lane) - 1ull));
            const bool here = g < s.n_groups;
            if (blockIdx.y == 0) {
                s.row[a0 + lane] = here ? r : -1;
                s.source[r] = here ? a0 + lane : -1;
            }
            dest[lane] = here ? r : (s.zero_rest ? ~r : (int)0x80000000);    // negative: not a row; ~r: zeros go there
        }
    }
    __syncthreads();
    for (int i = i0; i < items; i += stride) {
        const int t = i / batches, run = (i - t * batches) * batch;
        for (int k = 0; k < s.top_k; ++k) {
            const int d = __builtin_amdgcn_readfirstlane(dest[t * s.top_k + k]);
            if (d == (int)0x80000000) continue;
            char *to = s.rows + (int64_t)(d >= 0 ? d : ~d) * s.ld_rows;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = (run + u) * 64 + lane;
                if (u < batch && c < s.chunks) *(u32x4 *)(to + (int64_t)c * 16) = d >= 0 ? v[u] : (u32x4){0, 0, 0, 0};
            }
        }
        if (i + stride < items) load(i + stride);
    }
}

template <typename T> constexpr int kPer = 16 / sizeof(T);   // values of 16 bytes

template <typename T>
__device__ __forceinline__ float value(const u32x4 &v, int i)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[i]);
    else return __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
}
template <typename T>
__device__ __forceinline__ u32x4 packed(const float (&f)[kPer<T>])
{
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = __float_as_uint(f[i]);
        else v[i] = (uint32_t)f32_to_bf16(f[2 * i]) | ((uint32_t)f32_to_bf16(f[2 * i + 1]) << 16);
    }
    return v;
}

// A wavefront owns 64 16-byte columns of a token: the rows of eight assignments are requested before any is added.  They are read for the last time and not
// kept in the caches: 65536 rows of 4 KB behind as many written ones 87 us -> 57 (302 MB, 5.3 TB/s), 33 MB the same as without.  Whole rows a wavefront,
// rather than a quarter of eight rows at a time: no difference.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_combine_rows(CombineJob p, int runs)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int A = p.tokens * p.top_k;
    for (long long item = (long long)blockIdx.x * kWaves + wave; item < (long long)p.tokens * runs; item += (long long)gridDim.x * kWaves) {
        const int t = (int)(item / runs), c = (int)(item - (long long)t * runs) * 64 + lane;
        int r = -1;
        float w = 1.f;
        if (lane < p.top_k) {
            r = p.row[(size_t)t * p.top_k + lane];
            if (p.weights) w = p.weights[(size_t)t * p.top_k + lane];
        }
        unsigned long long live = __ballot((unsigned)r < (unsigned)A);
        float acc[kPer<T>];
#pragma unroll
        for (int i = 0; i < kPer<T>; ++i) acc[i] = 0.f;
        constexpr int U = 8;
        while (live) {
            u32x4 v[U];
            float wj[U];
            int n = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!live) break;
                const int j = __builtin_ctzll(live);
                live &= live - 1;
                const int rj = __builtin_amdgcn_readlane(r, j);
                wj[u] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j));
                v[u] = (u32x4){0, 0, 0, 0};
                if (c < p.chunks) v[u] = __builtin_nontemporal_load((const u32x4 *)(p.y + (int64_t)rj * p.ld_y + (int64_t)c * 16));
                n = u + 1;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= n) break;
#pragma unroll
                for (int i = 0; i < kPer<T>; ++i) acc[i] = fmaf(wj[u], value<T>(v[u], i), acc[i]);
            }
        }
        if (c < p.chunks) *(u32x4 *)(p.out + (int64_t)t * p.ld_out + (int64_t)c * 16) = packed<T>(acc);
    }
}

// A wavefront owns an assignment: its row of dy, its dot product (fp32, one rounding for each element of dy).  A token's wavefronts share its row of dout through
// the caches; rows of y are read for the last time.  40008 rows of 4 KB, 348 MB: 61 us, 5.7 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_combine_rows_backward(CombineJob p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int A = p.tokens * p.top_k;
    for (int64_t a = (int64_t)blockIdx.x * kWaves + wave; a < A; a += (int64_t)gridDim.x * kWaves) {
        if (p.grad_y && p.source) {       // row a, if it is nobody's
            const int of = p.source[a];
            if ((unsigned)of >= (unsigned)A || p.row[of] != (int)a)
                for (int c = lane; c < p.chunks; c += 64) *(u32x4 *)(p.grad_y + a * p.ld_grad_y + (int64_t)c * 16) = (u32x4){0, 0, 0, 0};
        }
        const int r = p.row[a];
        if ((unsigned)r >= (unsigned)A) {
            if (p.grad_weights && lane == 0) p.grad_weights[a] = 0.f;
            continue;
        }
        const float w = p.weights ? p.weights[a] : 1.f;
        const char *g = p.grad_out + (a / p.top_k) * p.ld_grad_out, *y = p.y + (int64_t)r * p.ld_y;
        char *dy = p.grad_y + (int64_t)r * p.ld_grad_y;
        float dot = 0.f;
        constexpr int U = 4;
        for (int c0 = lane; c0 < p.chunks; c0 += 64 * U) {
            u32x4 gv[U], yv[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * 64;
                gv[u] = yv[u] = (u32x4){0, 0, 0, 0};
                if (c < p.chunks) {
                    gv[u] = *(const u32x4 *)(g + (int64_t)c * 16);
                    if (p.grad_weights) yv[u] = __builtin_nontemporal_load((const u32x4 *)(y + (int64_t)c * 16));
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * 64;
                if (c >= p.chunks) continue;
                float d[kPer<T>];
#pragma unroll
                for (int i = 0; i < kPer<T>; ++i) {
                    const float gi = value<T>(gv[u], i);
                    d[i] = w * gi;
                    if (p.grad_weights) dot = fmaf(gi, value<T>(yv[u], i), dot);
                }
                if (p.grad_y) *(u32x4 *)(dy + (int64_t)c * 16) = packed<T>(d);
            }
        }
        if (p.grad_weights) {
            dot = wave_sum_f32(dot);
            if (lane == 0) p.grad_weights[a] = dot;
        }
    }
}

}  // namespace

int sort_blocks(int tokens, int top_k)
{
    const long long A = (long long)tokens * top_k;
    return A <= kSortOneLaunch ? 0 : (int)((A + kSortBlock - 1) / kSortBlock);
}

hipError_t launch_sort_tokens(const SortJob &j, hipStream_t st)
{
    const int bins = j.n_groups + 1, n_blocks = sort_blocks(j.tokens, j.top_k);
    int per = 64 / j.top_k;
    const int runs = (j.chunks + 63) / 64;
    // few tokens: fewer of them to a workgroup, then shorter batches on more workgroups.  us (a quarter of the limit, four times as much), 8 assignments a token, 128 groups:
    //   512 workgroups: 2048 tokens of 256 columns 11.1 (11.1, 15.3), 8192 20.1 (20.1, 24.3), 2048 of 7168 52 (54, 49), 512 of 256 8.3 (7.6, 8.3)
    //   4096 batches: 8192 tokens of 2048 columns 59.7 (59.3, 66.0), 2048 of 7168 50.6 (51.3, 57.5), 256 of 7168 11.2 (10.1, 11.1)
    //   512 workgroups in all: 128 tokens of 7168 columns 8.1 (11.5, 8.1), 64 6.6 (7.9, 6.5), 512 17.9 (17.9, 19.0)
    while (per > 1 && (j.tokens + per - 1) / per < 512) per = (per + 1) / 2;
    const int gx = j.tokens > 0 ? (j.tokens + per - 1) / per : 1;
    int batch = 4;
    while (batch > 1 && (long long)gx * per * ((runs + batch - 1) / batch) < 4096) batch /= 2;
    const int batches = (runs + batch - 1) / batch;
    int gy = 1;
    while (gy * kWaves < batches * per && gx * gy < 512) gy *= 2;
    const dim3 grid(gx, gy);
    const size_t lds = 2 * bins * sizeof(int32_t);
    if (n_blocks == 0) {
        hipLaunchKernelGGL(k_sort_place<kCountAll>, grid, dim3(kThreads), lds, st, j, per, batch, 0);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(k_sort_count, dim3(n_blocks), dim3(kThreads), bins * sizeof(int32_t), st, j);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if ((long long)n_blocks * bins <= kSortSums) {
        hipLaunchKernelGGL(k_sort_place<kAddUp>, grid, dim3(kThreads), lds, st, j, per, batch, n_blocks);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(k_sort_scan, dim3(1), dim3(kThreads), bins * sizeof(int32_t), st, j, n_blocks);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_sort_place<kScanned>, grid, dim3(kThreads), lds, st, j, per, batch, n_blocks);
    return hipGetLastError();
}

hipError_t launch_combine_tokens(const CombineJob &j, bool bf16, hipStream_t st)
{
    const int runs = (j.chunks + 63) / 64;
    const long long groups = ((long long)j.tokens * runs + kWaves - 1) / kWaves;
    const dim3 grid((unsigned)(groups < kMostGroups ? groups : kMostGroups));
    if (bf16) hipLaunchKernelGGL(k_combine_rows<uint16_t>, grid, dim3(kThreads), 0, st, j, runs);
    else      hipLaunchKernelGGL(k_combine_rows<float>, grid, dim3(kThreads), 0, st, j, runs);
    return hipGetLastError();
}

hipError_t launch_combine_tokens_backward(const CombineJob &j, bool bf16, hipStream_t st)
{
    const long long groups = ((long long)j.tokens * j.top_k + kWaves - 1) / kWaves;
    if (bf16) hipLaunchKernelGGL(k_combine_rows_backward<uint16_t>, dim3((unsigned)(groups < kMostGroups ? groups : kMostGroups)), dim3(kThreads), 0, st, j);
    else      hipLaunchKernelGGL(k_combine_rows_backward<float>, dim3((unsigned)(groups < kMostGroups ? groups : kMostGroups)), dim3(kThreads), 0, st, j);
    return hipGetLastError();
}

}  // namespace emoe
