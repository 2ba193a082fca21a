// Products of bf16 rows with 4-bit weights, the weights streamed straight into the matrix cores' operands.
//
//   out[r, c] = sum_k a[r, k] code[c, k] 2^p[c, k / 32]
//
// A code times its power of two is a bf16 number, 2^-128 .. 1.5 * 2^127 in magnitude, and infinite from 2^128 on (powers 2^126 and 2^127 alone): the conversion
// instruction makes two of them from a byte and the power, the products are exact and the sums fp32's.
// A K-step is a line of a weight row, 128 bytes or 256 columns, in two halves: of half h lane (quad, l15) has the 16 bytes of row l15 that hold the columns
// 128 h + 32 quad .. + 31, one group with one power, and instruction i takes the eight from 8 i, of the activation row the same.  Which k an instruction pairs
// with which does not matter: both sides agree.  Weight rows are the first operand, so that a lane holds neighbouring columns of one row of the result:
// tile t's row 4 q + e is the wavefront's column 4 (q WT + t) + e, which makes them 4 WT.
//
// A workgroup is NW wavefronts along the weight rows times KW along K (wavefront kw takes the lines kw, kw + KW, ..., their sums are added in that order
// through LDS), each on WT tiles of 16 weight rows (with swiglu WT of gate and WT of up rows) and all MT tiles of 16 rows, whose columns they share in LDS:
// KC of them at a time in two buffers, or (KC 0) all of them.  Weights go from memory to registers, D lines ahead; both halves of a line are requested
// together (half a line at a time, the other half by another wavefront: 142 us where this takes 106, DeepSeek-V3-shaped first products, 64 tokens, 468 MB).
// Their powers are read a line's eight at a time, or, where rows are long, 64 at a time by way of LDS: eight at a time the lines of the powers, of which a
// step needs a sixteenth, push each other out of the first cache (106 us -> 87).
#pragma once
#include <atomic>

#include "four_tiles.h"

namespace emoe {
namespace {

constexpr int kLine = 256;                // columns of a line of a weight row
constexpr int kPowers = 72;               // bytes in LDS from one weight row's powers to the next: 64 of them and a gap against bank conflicts
constexpr size_t kMostLds = 160 * 1024;

// The n-th group (lo, hi: its rows), -1 if it has none; where there are more groups than twice the rows (sparse) the n-th that has some: every workgroup looks for
// itself, and groups without rows cost none then.
__device__ __forceinline__ int nth_group(const FourGemm &g, int n, int &lo, int &hi)
{
    lo = 0; hi = g.m;
    if (!g.offsets) return n == 0 ? 0 : -1;
    if (n >= g.groups) return -1;
    if (!g.sparse) {
        lo = max(g.offsets[n], 0);
        hi = min(g.offsets[n + 1], g.m);
        return hi > lo ? n : -1;
    }
    const int lane = threadIdx.x & 63;
    constexpr int U = 4;
    for (int g0 = 0; g0 < g.groups; g0 += 64 * U) {
        int a[U], b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = g0 + u * 64 + lane;
            a[u] = b[u] = 0;
            if (e < g.groups) { a[u] = max(g.offsets[e], 0); b[u] = min(g.offsets[e + 1], g.m); }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned long long some = __ballot(b[u] > a[u]);
            const int here = __popcll(some);
            if (n >= here) { n -= here; continue; }
            const int at = __builtin_ctzll(__ballot(b[u] > a[u] && __popcll(some & ((1ull << lane) - 1ull)) == n));
            lo = __builtin_amdgcn_readlane(a[u], at);
            hi = __builtin_amdgcn_readlane(b[u], at);
            return g0 + u * 64 + at;
        }
    }
    return -1;
}

// kWhole: k is whole lines.  kDirect: powers a line at a time, straight from memory.
template <bool kSwiglu, int NW, int KW, int MT, int WT, int D, int KC, int kWavesPerSimd, bool kDirect, bool kWhole, typename TOut>
__global__ __launch_bounds__(NW * KW * 64) __attribute__((amdgpu_waves_per_eu(kWavesPerSimd, kWavesPerSimd))) void k_four_rows(FourGemm g, int slices, int row_tiles, int together)
{
    constexpr int LT = kSwiglu ? 2 * WT : WT, W = NW * KW, kThreads = W * 64;
    constexpr int XJ = KC ? MT * 2 * KC / kThreads : 1;                 // 16-byte pieces of a chunk's rows a thread
    constexpr int STRIDE = LT * 16 + 4;                                 // floats of a row's partial sums
    static_assert(KC % (kLine * KW) == 0 && (KC == 0 || (KC / kLine / KW % D == 0 && 2048 % KC == 0 && XJ * kThreads == MT * 2 * KC)), "chunks are whole turns of the loops");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, quad = lane >> 4, kw = wave % KW, nw = wave / KW;
    char *ss = lds + wave * (LT * 16 * kPowers), *xs = lds + (kDirect ? 0 : W * LT * 16 * kPowers);

    // `together` slices' row tiles one after the other (a multiple of eight, so that a slice's tiles run on one XCD: workgroup b on XCD b mod 8)
    const int turn = blockIdx.x / (together * row_tiles), in_turn = blockIdx.x - turn * together * row_tiles;
    const int first_tile = in_turn / together, at = turn * together + in_turn - first_tile * together;
    const int slice = at % slices, n0 = (slice * NW + nw) * WT * 16;
    int lo, hi;
    const int group = nth_group(g, at / slices, lo, hi);
    if (group < 0) return;
    const int lines = (g.k + kLine - 1) / kLine, powers = g.k / kFourGroup;
    const int cols = KC ? KC : lines * kLine, chunks = KC ? (g.k + KC - 1) / KC : 1, turns = cols / kLine / KW + (KC ? 0 : 1);   // of a chunk in LDS; lines of a wavefront's
    // addresses: a scalar of the wavefront's first row (of gate and of up rows) and 32 bits of this lane's row from there
    const size_t w_row = (size_t)group * (kSwiglu ? 2 : 1) * g.n + min(n0, g.n - 1);
    const uint8_t *wb[kSwiglu ? 2 : 1], *sb[kSwiglu ? 2 : 1];
#pragma unroll
    for (int u = 0; u < (kSwiglu ? 2 : 1); ++u) {
        wb[u] = g.w + (w_row + (size_t)u * g.n) * (g.k / 2);
        sb[u] = g.ws + (w_row + (size_t)u * g.n) * powers;
    }
    uint32_t wo[WT], so[WT];
#pragma unroll
    for (int t = 0; t < WT; ++t) {
        const uint32_t row = max(min((l15 >> 2) * (WT * 4) + t * 4 + (l15 & 3), g.n - 1 - n0), 0);
        wo[t] = row * (uint32_t)(g.k / 2) + quad * 16;
        so[t] = row * (uint32_t)powers;
    }
    // n bytes of a weight row's powers from `at` on: behind the row's end the next row's (they meet zeros), but nothing behind the last row of a group
    const bool near_end = n0 + WT * 16 + 16 > g.n;
    auto fetch_powers = [&](uint32_t *to, int t, int at, int n) __attribute__((always_inline)) {
        const uint8_t *p = sb[t / WT];
        const uint32_t o = so[t % WT] + at;
        if (!near_end || (kWhole && n == 8) || at + n <= powers) {
            if (n == 16) __builtin_memcpy(to, p + o, 16);
            else __builtin_memcpy(to, p + o, 8);
            return;
        }
        unsigned long long v[2] = {0, 0};
        if (powers >= n) {                  // the row's last n bytes, shifted
            __builtin_memcpy(v, p + so[t % WT] + (powers - n), n == 16 ? 16 : 8);
            const int bits = 8 * (at + n - powers);
            if (n == 8) v[0] >>= bits;
            else if (bits >= 64) { v[0] = v[1] >> (bits - 64); v[1] = 0; }
            else { v[0] = (v[0] >> bits) | (v[1] << (64 - bits)); v[1] >>= bits; }
        } else {
#pragma unroll 1
            for (int i = powers - 1; i >= at; --i) {
                v[1] = (v[1] << 8) | (v[0] >> 56);
                v[0] = (v[0] << 8) | p[so[t % WT] + i];
            }
        }
        for (int i = 0; i < n / 4; ++i) to[i] = (uint32_t)(v[i / 2] >> (32 * (i % 2)));
    };

    for (int r0 = lo + first_tile * MT * 16; r0 < hi; r0 += row_tiles * MT * 16) {
        const int rows = min(MT * 16, hi - r0), live = (rows + 15) >> 4;
        // the 16-byte pieces of a row lie in LDS with the low four bits of their number xored with the row's: a half-wavefront reads 16 rows' pieces of
        // one number, from 16 different bank groups
        auto piece = [&](int row, int at) __attribute__((always_inline)) { return xs + (size_t)row * (cols * 2) + ((at & ~15) | ((at ^ row) & 15)) * 16; };
        u32x4 xr[XJ];
        auto load_x = [&](int c) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < XJ; ++j) {
                constexpr int P = KC ? KC / 8 : 1, R = kThreads / P;    // pieces of a row, rows of a turn
                static_assert(kThreads % P == 0, "a thread has the same piece of several rows");
                const int row = threadIdx.x / P, col = threadIdx.x % P * 8;
                const char *from = (const char *)(g.a + (r0 + j * R) * g.ld_a + c * KC);
                xr[j] = (u32x4){0, 0, 0, 0};
                if (row + j * R < rows && c * KC + col < g.k) xr[j] = *(const u32x4 *)(from + (uint32_t)(row * (int)g.ld_a + col) * 2u);
            }
        };
        auto store_x = [&](int c) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < XJ; ++j) {
                const int p = threadIdx.x + j * kThreads, row = p / (KC ? KC / 8 : 1);
                if (row < rows) *(u32x4 *)(piece(row, p % (KC ? KC / 8 : 1)) + (c & 1) * (MT * 32 * KC)) = xr[j];
            }
        };
        auto copy_x = [&]() __attribute__((always_inline)) {            // all of the rows: runs of 64 pieces, eight of a wavefront on their way
            constexpr int U = 8;
            const int runs = (cols / 8 + 63) / 64, n = rows * runs;
            for (int i0 = wave; i0 < n; i0 += W * U) {
                u32x4 v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * W, row = i / runs, at = (i - row * runs) * 64 + lane;
                    v[u] = (u32x4){0, 0, 0, 0};
                    if (i < n && at * 8 < g.k) v[u] = *(const u32x4 *)(g.a + (r0 + row) * g.ld_a + at * 8);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * W, row = i / runs, at = (i - row * runs) * 64 + lane;
                    if (i < n && at < cols / 8) *(u32x4 *)piece(row, at) = v[u];
                }
            }
        };
        u32x4 sr[LT];                                                   // the powers of 2048 columns: lane (quad, l15) fetches 16 of row l15
        auto load_s = [&](int c) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < LT; ++t) {
                sr[t] = (u32x4){0, 0, 0, 0};
                uint32_t s[4];
                if (c * 64 + quad * 16 < powers) {
                    fetch_powers(s, t, c * 64 + quad * 16, 16);
                    sr[t] = (u32x4){s[0], s[1], s[2], s[3]};
                }
            }
        };
        auto store_s = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < LT; ++t) {
                u32x2 *p = (u32x2 *)(ss + (t * 16 + l15) * kPowers + quad * 16);
                p[0] = (u32x2){sr[t][0], sr[t][1]};
                p[1] = (u32x2){sr[t][2], sr[t][3]};
            }
        };
        u32x4 wf[D][LT][2];
        uint32_t df[D][LT][2];
        auto request = [&](int d, int b) __attribute__((always_inline)) {
            if (b >= lines) return;
            const bool whole = kWhole || (b + 1) * kLine <= g.k;
#pragma unroll
            for (int t = 0; t < LT; ++t) {
                if (kDirect) fetch_powers(df[d][t], t, b * 8, 8);
                const uint8_t *p = wb[t / WT] + (size_t)b * (kLine / 2);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (whole) wf[d][t][h] = *(const u32x4 *)(p + h * 64 + wo[t % WT]);
                    else {
                        wf[d][t][h] = (u32x4){0, 0, 0, 0};
                        if (b * kLine + h * 128 + quad * 32 < g.k) wf[d][t][h] = *(const u32x4 *)(p + h * 64 + wo[t % WT]);
                    }
                }
            }
        };
        f32x4 acc[LT][MT];
#pragma unroll
        for (int t = 0; t < LT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[t][m] = (f32x4){0.f, 0.f, 0.f, 0.f};
        int xrow[MT];                                                   // rows that do not exist: anything, but where LDS has no place for them the last one
#pragma unroll
        for (int m = 0; m < MT; ++m) xrow[m] = KC ? m * 16 + l15 : min(m * 16 + l15, rows - 1);

        if (KC) load_x(0);
        if (!kDirect) load_s(0);
#pragma unroll
        for (int d = 0; d < D; ++d) request(d, d * KW + kw);
        if (KC) store_x(0);
        else copy_x();
        __syncthreads();
        for (int c = 0; c < chunks; ++c) {
            if (KC && c + 1 < chunks) load_x(c + 1);
            if (!kDirect && (KC == 0 || c % (2048 / (KC ? KC : 2048)) == 0)) {
                store_s();
                if ((c * KC / 2048 + 1) * 2048 < g.k) load_s(c * KC / 2048 + 1);
            }
            const char *xb = xs + (KC ? (c & 1) * (MT * 32 * KC) : 0);
#pragma unroll
            for (int i0 = 0; i0 < (KC ? KC / kLine / KW : turns); i0 += D) {
#pragma unroll
                for (int d = 0; d < D; ++d) {
                    const int l = (i0 + d) * KW + kw, b = (KC ? c * (KC / kLine) : 0) + l;
                    if (b >= lines) continue;
                    const bool whole = kWhole || (b + 1) * kLine <= g.k;
                    uint32_t sf[LT][2];
#pragma unroll
                    for (int t = 0; t < LT; ++t) {
                        if (kDirect) { sf[t][0] = df[d][t][0]; sf[t][1] = df[d][t][1]; }
                        else {
                            const u32x2 s = *(const u32x2 *)(ss + (t * 16 + l15) * kPowers + (b & 7) * 8);
                            sf[t][0] = s[0]; sf[t][1] = s[1];
                        }
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        bf16x8 x[MT][4];
#pragma unroll
                        for (int m = 0; m < MT; ++m)
                            if (m < live)
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    x[m][i] = *(const bf16x8 *)(xb + xrow[m] * (cols * 2) + ((l * 2 + h) * 16 + ((quad * 4 + i) ^ (KC ? l15 : xrow[m] & 15))) * 16);
                        const bool in = whole || b * kLine + h * 128 + quad * 32 < g.k;
#pragma unroll
                        for (int t = 0; t < LT; ++t) {
                            const uint32_t byte = (sf[t][h] >> (8 * quad)) & 255;
                            const float power = __uint_as_float((in ? byte : 0) << 23);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const bf16x8 w = weights8(wf[d][t][h][i], power);
#pragma unroll
                                for (int m = 0; m < MT; ++m)
                                    if (m < live) acc[t][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[m][i], acc[t][m], 0, 0, 0);
                            }
                        }
                    }
                    request(d, b + D * KW);
                }
            }
            if (KC && c + 1 < chunks) store_x(c + 1);
            __syncthreads();
        }

        if constexpr (KW == 1) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (m * 16 + l15 >= rows) continue;
                const size_t r = r0 + m * 16 + l15;
                const int col = n0 + quad * (WT * 4);
#pragma unroll
                for (int t = 0; t < WT; t += 2) {
                    if (WT > 1 && sizeof(TOut) == 2 && col + t * 4 + 8 <= g.n)
                        finish8<kSwiglu>(g, r, col + t * 4, acc[t][m], acc[(t + 1) % LT][m], acc[kSwiglu ? t + WT : t][m], acc[kSwiglu ? (t + 1) % WT + WT : t][m]);
                    else {
                        if (col + t * 4 < g.n) finish<kSwiglu, TOut>(g, r, col + t * 4, acc[t][m], acc[kSwiglu ? t + WT : t][m]);
                        if (WT > 1 && col + t * 4 + 4 < g.n) finish<kSwiglu, TOut>(g, r, col + t * 4 + 4, acc[(t + 1) % LT][m], acc[kSwiglu ? (t + 1) % WT + WT : t][m]);
                    }
                }
            }
        } else {
            float *red = (float *)xs;                                   // [wavefronts][16][STRIDE]
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (m >= live) break;
                if (m > 0) __syncthreads();
#pragma unroll
                for (int t = 0; t < LT; ++t) *(f32x4 *)&red[(wave * 16 + l15) * STRIDE + t / WT * WT * 16 + quad * (WT * 4) + t % WT * 4] = acc[t][m];
                __syncthreads();
                const int mine = min(16, rows - m * 16);
                for (int i = threadIdx.x; i < NW * 16 * WT * 4; i += kThreads) {
                    const int c4 = i % (WT * 4) * 4, row = i / (WT * 4) % 16, of = i / (WT * 64);
                    const int col = (slice * NW + of) * WT * 16 + c4;
                    if (row >= mine || col >= g.n) continue;
                    f32x4 s[kSwiglu ? 2 : 1];
#pragma unroll
                    for (int h = 0; h < (kSwiglu ? 2 : 1); ++h) {
                        s[h] = *(const f32x4 *)&red[(of * KW * 16 + row) * STRIDE + h * WT * 16 + c4];
#pragma unroll
                        for (int w = 1; w < KW; ++w) s[h] += *(const f32x4 *)&red[((of * KW + w) * 16 + row) * STRIDE + h * WT * 16 + c4];
                    }
                    finish<kSwiglu, TOut>(g, r0 + m * 16 + row, col, s[0], s[kSwiglu ? 1 : 0]);
                }
            }
            __syncthreads();
        }
    }
}

int slices_of(const FourGemm &g, int cols) { return (g.n + cols - 1) / cols; }
// groups that get workgroups: where many have no rows, one for every row at most
int groups_of(const FourGemm &g) { return g.sparse && g.m < g.groups ? g.m : g.groups; }

// LDS of a workgroup
template <bool kSwiglu, int NW, int KW, int MT, int WT, int KC, bool kDirect>
size_t lds_of(const FourGemm &g)
{
    constexpr int LT = kSwiglu ? 2 * WT : WT;
    const size_t line_cols = (size_t)(g.k + kLine - 1) / kLine * kLine, rows = g.m < MT * 16 ? g.m : MT * 16;
    const size_t x = KC ? (size_t)MT * 32 * KC * (g.k > KC ? 2 : 1) : rows * line_cols * 2;
    const size_t red = KW > 1 ? (size_t)NW * KW * 16 * (LT * 16 + 4) * 4 : 0;
    return (kDirect ? 0 : (size_t)NW * KW * LT * 16 * kPowers) + (x > red ? x : red);
}

// More than 64 KB of LDS are asked for once for each kernel and device (a bit of `allowed`).
hipError_t allow_lds(const void *kernel, size_t lds, std::atomic<unsigned long long> &allowed)
{
    if (lds <= 64 * 1024) return hipSuccess;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
    if (allowed.load(std::memory_order_relaxed) & bit) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMostLds);
    if (e == hipSuccess) allowed.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <bool kSwiglu, int NW, int KW, int MT, int WT, int D, int KC, int kOcc, bool kDirect, bool kWhole, typename TOut>
hipError_t launch_whole(const FourGemm &g, int row_tiles, hipStream_t st)
{
    static_assert(KC || kDirect, "powers by way of LDS are turned over with the chunks");
    const auto kernel = k_four_rows<kSwiglu, NW, KW, MT, WT, D, KC, kOcc, kDirect, kWhole, TOut>;
    const size_t lds = lds_of<kSwiglu, NW, KW, MT, WT, KC, kDirect>(g);
    static std::atomic<unsigned long long> allowed{0};
    const hipError_t e = allow_lds((const void *)kernel, lds, allowed);
    if (e != hipSuccess) return e;
    const int slices = slices_of(g, NW * WT * 16);
    // A slice's row tiles read the same weights and run side by side.  Of sorted rows nobody knows which tiles have none: those workgroups end at once, and
    // come last.  Between the others they upset how these are dealt out to the chip (in turn with eight others 309 us for 163, with 264 169 for 102).
    const long long all = ((long long)slices * groups_of(g) + 7) / 8 * 8;
    const int together = !g.offsets ? 8 : (int)all;
    const long long units = (all + together - 1) / together * together, most = kMostThreads / (NW * KW * 64) / units;
    // workgroups go on to further row tiles of theirs where a launch could not have one for each
    const int tiles = (int)(most < row_tiles ? most : row_tiles);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(units * tiles)), dim3(NW * KW * 64), lds, st, g, slices, tiles, together);
    return hipGetLastError();
}
template <bool kSwiglu, int NW, int KW, int MT, int WT, int D, int KC, int kOcc, bool kDirect, typename TOut>
hipError_t launch_as(const FourGemm &g, int row_tiles, hipStream_t st)
{
    if (g.k % kLine == 0) return launch_whole<kSwiglu, NW, KW, MT, WT, D, KC, kOcc, kDirect, true, TOut>(g, row_tiles, st);
    return launch_whole<kSwiglu, NW, KW, MT, WT, D, KC, kOcc, kDirect, false, TOut>(g, row_tiles, st);
}
// rows of a group, if all get as many
int rows_each(const FourGemm &g) { return (g.m + groups_of(g) - 1) / groups_of(g); }
int row_tiles(const FourGemm &g, int rows)
{
    if (!g.offsets) return (g.m + rows - 1) / rows;
    const int tiles = (rows_each(g) * 3 / 2 + rows - 1) / rows;  // some groups have more than others; the workgroups of those with still more go on
    return tiles < 1 ? 1 : tiles > 8 ? 8 : tiles;
}
long long workgroups(const FourGemm &g, int cols, int rows) { return (long long)slices_of(g, cols) * groups_of(g) * row_tiles(g, rows); }

}  // namespace
}  // namespace emoe
