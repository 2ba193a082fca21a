// Block-scaled e4m3 products of many rows: tiles of up to 128 rows, with the 8-bit matrix instructions 256, times 256 weight rows (with swiglu 128 gate and
// 128 up rows).
//
//   out[r, c] = sum_b as[r, b] ws[c / 128, b] sum_{k in block b} a[r, k] w[c, k]
//
// A K-step is one scale block: 128 bytes of every row of the tile, one cache line each.  Both operands travel straight from global
// memory into an LDS ring (16 bytes per lane, the XOR swizzle of swz8 applied on the global side), together with the step's
// scales, four steps at a time.  The block's sums come out of the matrix cores with a zero start and are added to the
// fp32 accumulators times as * ws: four multiply-adds a lane for the 256 sums of 16 x 16, beside the one 8-bit or four bf16 matrix instructions of the
// next 16 x 16.  Exact products (through bf16) are bound by the bf16 matrix rate and the conversions, matrix cores busy 40 to 46 % of a prefill's
// products; a decode batch by its weights (GEMM-1 of a DeepSeek-V3-shaped rank, 64 tokens, 138 us for 0.91 GB; with the 8-bit instructions 134).
//
// Workgroup: 8 wavefronts as 2 (rows) x 4 (weights).  Wavefront (wm, wn) owns weight rows [64 wn, 64 wn + 64) and the 16-row tiles
// wm, wm + 2, ... of the rows.  A tile with fewer rows runs a body for fewer of them, whose ring is deeper.
// Weight rows are the first operand, so that a lane holds four neighbouring columns of one row of the result.  With swiglu
// 16 gate rows and the 16 matching up rows alternate: a lane has both values of a column in neighbouring accumulators, and the
// 128 columns of a tile are one scale group of the 8-bit result, whose maximum is found over the four weight wavefronts through LDS.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "scaled.h"

namespace emoe {
namespace {

constexpr int kThreads = 512;
constexpr int kBN = 256;                       // weight rows of a tile
constexpr int kRowBytes = kScaleBlock;         // bytes of a row in a K-step
constexpr int kWStage = kBN * kRowBytes;       // 32 KB
constexpr int kLds = 160 * 1024;
constexpr int kXcds = 8;
constexpr int kGroup = 4;                      // steps whose scales travel together

// NT 16-row tiles per wavefront: 32 NT rows, staged in whole 64.  NW stages of weights, NX of rows: as many as there is room for, weights first,
// which come from memory while the rows are found in L2.
template <int NT_> struct Ring {
    static constexpr int NT = NT_, BM = NT == 1 ? 32 : (NT + 1) / 2 * 64, XStage = BM * kRowBytes;
    static constexpr int NW = NT == 1 ? 4 : NT <= 6 ? 3 : 2, NX = NT == 1 ? 4 : NT <= 4 ? 3 : 2;
    static constexpr bool WeightsFirst = NT <= 2;              // of a step's copies: where everybody waits for the weights
    static constexpr int WP = 4, XP = NT >= 2 ? BM / 64 : 1;     // 1 KB pieces (8 rows) per wavefront and step
    static constexpr int XBase = NW * kWStage, Scales = XBase + NX * XStage, ScaleBytes = 2 * kGroup * BM * 4;
    static constexpr int WScales = Scales + ScaleBytes, WScaleBytes = 2 * 256;
    // Copies that may be on their way when step b is needed, all steps up to b + NW - 2 being there: in the order in which they go out (the rows of a step
    // before its weights) those behind the rows of b, or with as many stages of both behind its weights.  A wavefront that issues more waits for more.
    static constexpr int P = NT >= 2 ? WP + XP : WP;
    static constexpr int Young = (NX - 2) * P + (NW > NX ? WP : 0);
    static_assert(NW == NX || (NW == NX + 1 && !WeightsFirst), "Young");
    static_assert(WScales + WScaleBytes <= kLds, "LDS");
};

struct Ctx {
    const uint8_t *wbase, *abase;
    size_t up;                     // bytes from a gate row to its up row
    uint32_t woff[4], xoff[4];     // this lane's byte offsets of the pieces it stages, k = 0
    uint32_t soff;                 // and of its row's scales (wavefronts below BM / 64)
    const float *sbase, *wsbase;
    uint32_t wsoff;                // this lane's weight scale of a group: 4 steps of 2 blocks
    int wave, lane, wm, wn, l15, quad;
    int k, kb;
    bool wide;                     // scales of a group travel as 16 bytes
    bool once;                     // no other tile reads these weights
};

__device__ __forceinline__ uint32_t lds_addr(const void *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p; }
// global -> LDS: lane i's bytes land at lds + its width * i.  Issued as assembly so that the compiler does not hold later LDS reads for
// copies of a later stage; wait_loads() waits for them.
__device__ __forceinline__ void dma16(const void *base, uint32_t off, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
// The same for the wavefronts of a mask that is all ones or zero (nothing is copied), without a branch.  Called where all lanes are active, and they are again
// behind it.
// kOnce: the line is marked as read once.
template <bool kOnce>
__device__ __forceinline__ void dma16_masked(const void *base, uint32_t off, uint32_t lds, int mask)
{
    mask = __builtin_amdgcn_readfirstlane(mask);
    if (kOnce) asm volatile("s_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt\n\ts_mov_b64 exec, -1" ::"s"(lds), "v"(off), "s"(base), "s"(mask) : "memory", "m0");
    else       asm volatile("s_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1" ::"s"(lds), "v"(off), "s"(base), "s"(mask) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void *base, uint32_t off, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
template <int n>
__device__ __forceinline__ void wait_loads()
{
    static_assert(n < 64, "vmcnt has 6 bits");
    __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8));
}

// Copy i of this wavefront's for a K-step: rows of step b + NX - 1, then weights of step b + NW - 1 (step b is the one that is multiplied meanwhile).
// A last step that ends inside the block fetches the last 128 columns: what comes before its own is zeroed in LDS before use.  Of a contraction shorter
// than a block (kShort) chunks behind the row's end repeat the first one, and are zeroed.
template <typename R, bool kSwiglu, bool kShort, int i>
__device__ __forceinline__ void issue_copy(const Ctx &c, uint32_t lds, int wstage, int xstage, int b)
{
    constexpr bool weights = R::WeightsFirst ? i < R::WP : i >= R::XP;
    constexpr int n = !weights ? (R::WeightsFirst ? i - R::WP : i) : R::WeightsFirst ? i : i - R::XP;    // the how-manieth of its kind
    const int step = b + (weights ? R::NW : R::NX) - 1;
    int mask = step >= 0 && step < c.kb ? -1 : 0;
    if constexpr (!weights && R::NT < 2) mask = c.wave < 4 ? mask : 0;
    const int pc = c.wave * (weights ? R::WP : R::XP) + n;
    uint32_t off = weights ? c.woff[weights ? n : 0] : c.xoff[weights ? 0 : n];
    if (kShort) {
        const int chunk = ((c.lane & 7) ^ swz8(pc * 8 + (c.lane >> 3))) * 16;
        if (chunk >= c.k) off -= chunk;
    }
    const uint8_t *from = (weights ? kSwiglu && (pc & 2) ? c.wbase + c.up : c.wbase : c.abase) + (kShort ? 0 : min(step * kRowBytes, c.k - kRowBytes));
    const uint32_t to = lds + (weights ? wstage * kWStage : R::XBase + xstage * R::XStage) + pc * 1024;
    if (weights && R::NT <= 2 && c.once) dma16_masked<true>(from, off, to, mask);
    else                                 dma16_masked<false>(from, off, to, mask);
}
template <typename R, bool kSwiglu, bool kShort, int i = 0>
__device__ __forceinline__ void issue_copies(const Ctx &c, uint32_t lds, int wstage, int xstage, int b)
{
    if constexpr (i < R::WP + R::XP) {
        issue_copy<R, kSwiglu, kShort, i>(c, lds, wstage, xstage, b);
        issue_copies<R, kSwiglu, kShort, i + 1>(c, lds, wstage, xstage, b);
    }
}
// The copies of a step go out behind the first row tiles' matrix instructions, two at a time: a compute unit accepts 64 bytes a cycle, and a
// wavefront that issues all of its copies at once stands still meanwhile.  Tiles of up to 64 rows, which wait for weights, issue them first.
template <typename R, bool kSwiglu, int i = 0>
__device__ __forceinline__ void issue_between(const Ctx &c, uint32_t lds, int wstage, int xstage, int b, int t)
{
    if constexpr (i < R::WP + R::XP) {
        if (R::NT <= 2 ? t == 0 : i / 2 == t || (t == R::NT - 1 && i / 2 > t)) issue_copy<R, kSwiglu, false, i>(c, lds, wstage, xstage, b);
        issue_between<R, kSwiglu, i + 1>(c, lds, wstage, xstage, b, t);
    }
}
// The scales of steps 4 g .. 4 g + 3 into half g & 1 of their buffers (steps that do not exist repeat the last one).
template <typename R>
__device__ __forceinline__ void issue_scales(const Ctx &c, uint32_t ring, int g)
{
    const int b0 = g * kGroup;
    if (b0 >= c.kb) return;
    const uint32_t half = ring + R::Scales + (g & 1) * (R::ScaleBytes / 2);
    if (c.wave < (R::BM + 63) / 64) {      // 64 rows a wavefront (a tile of 32 rows: the upper lanes repeat the last row, behind its own half)
        if (c.wide) {
            if (R::BM >= 64 || c.lane < R::BM) dma16(c.sbase + b0, c.soff, half + c.wave * 1024);
        } else {
#pragma unroll
            for (int j = 0; j < kGroup; ++j)
                if (R::BM >= 64 || c.lane < R::BM) dma4(c.sbase + min(b0 + j, c.kb - 1), c.soff, half + j * R::BM * 4 + c.wave * 256);
        }
    }
    if (c.wave == 7) dma4(c.wsbase + b0, c.wsoff + 4 * min(c.lane & 3, c.kb - 1 - b0), ring + R::WScales + (g & 1) * 256);
}

// One K-step: NT tiles of 16 rows x 4 tiles of 16 weight rows.  Exact: through bf16, see scaled.h.  between(t) runs behind the
// matrix instructions of row tile t.
template <int NT, bool kSwiglu, bool kExact, typename Between>
__device__ __forceinline__ void multiply_step(const Ctx &c, const char *Ws, const char *Xs, const float *sa, int sa_row, float sw0, float sw1, f32x4 (&acc)[4][NT],
                                              Between between)
{
    const int lo = ((c.quad ^ swz8(c.l15)) << 4), hi = (((4 + c.quad) ^ swz8(c.l15)) << 4);   // rows 16 apart have the same swizzle but for bit 3 of the row, which l15 holds
    auto fetch = [&](const char *base, int row16) __attribute__((always_inline)) {
        const char *p = base + (row16 * 16 + c.l15) * kRowBytes;
        Bytes32 f;
        f.lo = *(const uint4 *)(p + lo);
        f.hi = *(const uint4 *)(p + hi);
        return f;
    };
    if (NT <= 2) between(0);
    Bytes32 wf[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) wf[a] = fetch(Ws, c.wn * 4 + a);
    const auto scale_of = [&](int t) __attribute__((always_inline)) { return sa[((2 * t + c.wm) * 16 + c.l15) * sa_row]; };
    float s[2] = {scale_of(0), 0.f};
    Bytes32 xf[2];
    xf[0] = fetch(Xs, c.wm);
    Bf16x32 w[kExact ? 4 : 1], x[kExact ? 2 : 1];
    if constexpr (kExact) x[0].from(xf[0]);
    // two sets of block sums: those of row tile t - 1 are added between the matrix instructions of t.  (Added in front of them, on one set of
    // registers, both wavefronts of a SIMD add at the same time, and the matrix cores wait.)
    f32x4 d[2][4];
    auto add = [&](int t, int a, float f) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[a][t][e] = fmaf(d[t & 1][a][e], f, acc[a][t][e]);
    };
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (t + 1 < NT) xf[(t + 1) & 1] = fetch(Xs, 2 * (t + 1) + c.wm);
        const float f0 = s[(t + 1) & 1] * sw0, f1 = kSwiglu ? s[(t + 1) & 1] * sw1 : f0;
        // a wavefront on its matrix instructions goes first: the other one's copies and reads fill the gaps (8192^3, 8-bit instructions, 464 -> 450 us, SwiGLU 4096 x 2048 x 7168 208 -> 201)
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            if constexpr (kExact) {
                // the conversions stand between the matrix instructions too: of the weights at their first use, of the next rows under these ones'
                if (t == 0) w[a].from(wf[a]);
                d[t & 1][a] = multiply_exact(w[a], x[t & 1]);
                if (t + 1 < NT && a == 2) { x[(t + 1) & 1].template from_quarter<0>(xf[(t + 1) & 1]); x[(t + 1) & 1].template from_quarter<1>(xf[(t + 1) & 1]); }
                if (t + 1 < NT && a == 3) { x[(t + 1) & 1].template from_quarter<2>(xf[(t + 1) & 1]); x[(t + 1) & 1].template from_quarter<3>(xf[(t + 1) & 1]); }
            } else {
                d[t & 1][a] = multiply_fast(wf[a], xf[t & 1]);
            }
            if (t > 0) add(t - 1, a, a & 1 ? f1 : f0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (t + 1 < NT) s[(t + 1) & 1] = scale_of(t + 1);
        __builtin_amdgcn_s_setprio(0);
        if (NT > 2) between(t);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int a = 0; a < 4; ++a) add(NT - 1, a, s[(NT - 1) & 1] * (a & 1 ? sw1 : sw0));
}

// Rows of the result through a wavefront's own LDS region: 16 rows of 64 fp32 columns, then whole row segments.  Block16: the wavefront's 64
// columns of a row become 16-bit numbers with a common scale.
template <int NT, typename TOut>
__device__ __forceinline__ void store_rows(const SGemm &g, const Ctx &c, const MTile &mt, int n0, char *ring, const f32x4 (&acc)[4][NT])
{
    constexpr int STRIDE = 64 + 4;
    float *mine = (float *)ring + c.wave * 16 * STRIDE;
    const int col = n0 + c.wn * 64 + (c.lane & 7) * 8, lr = c.lane >> 3;
    const bool whole = col + 8 <= g.n;
    // what is added is requested for all rows before the first are stored
    constexpr bool kBlock = std::is_same<TOut, Block16>::value;
    constexpr int W = sizeof(TOut) / 2;                        // 16-byte pieces of 8 columns
    uint4 av[NT][2][W];
    if (!kBlock && g.add) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = (2 * t + c.wm) * 16 + h * 8 + lr;
                if (row < mt.rows && whole)
#pragma unroll
                    for (int w = 0; w < W; ++w) av[t][h][w] = *(const uint4 *)((const TOut *)g.add + ((size_t)mt.row_begin + row) * g.ld_add + col + w * 4);
            }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int a = 0; a < 4; ++a) *(f32x4 *)(mine + c.l15 * STRIDE + a * 16 + c.quad * 4) = acc[a][t];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = (2 * t + c.wm) * 16 + h * 8 + lr;
            float v[8];
            *(f32x4 *)v = *(const f32x4 *)(mine + (h * 8 + lr) * STRIDE + (c.lane & 7) * 8);
            *(f32x4 *)(v + 4) = *(const f32x4 *)(mine + (h * 8 + lr) * STRIDE + (c.lane & 7) * 8 + 4);
            const size_t r = (size_t)mt.row_begin + row;
            if constexpr (kBlock) {
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, whole ? magnitude(v[e]) : 0u);
                top = lanes8_max(top);
                const Block16Scale b(__uint_as_float(top));
                if (row < mt.rows && whole) {                  // n is a multiple of 16
                    *(uint4 *)((uint16_t *)g.out + r * g.ld_out + col) = make_uint4(b.pack(v[0], v[1]), b.pack(v[2], v[3]), b.pack(v[4], v[5]), b.pack(v[6], v[7]));
                    if ((c.lane & 7) == 0) g.os[r * g.ld_os + (col >> 6)] = b.scale;
                }
                continue;
            }
            if (row >= mt.rows || col >= g.n) continue;
            TOut *o = (TOut *)g.out + r * g.ld_out + col;
            if (whole) {
                if (g.add) {
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        const uint32_t x[4] = {av[t][h][w].x, av[t][h][w].y, av[t][h][w].z, av[t][h][w].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if constexpr (W == 2) v[w * 4 + i] += __uint_as_float(x[i]);
                            else { v[2 * i] += __uint_as_float(x[i] << 16); v[2 * i + 1] += __uint_as_float(x[i] & 0xffff0000u); }
                        }
                    }
                }
                if constexpr (W == 2) {
                    *(float4 *)o = make_float4(v[0], v[1], v[2], v[3]);
                    *(float4 *)(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
                } else {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16(v[2 * i]) | ((uint32_t)f32_to_bf16(v[2 * i + 1]) << 16);
                    *(uint4 *)o = make_uint4(w[0], w[1], w[2], w[3]);
                }
            } else if constexpr (!kBlock) {
                const TOut *add = (const TOut *)g.add + r * g.ld_add + col;
                for (int e = 0; e < g.n - col; ++e) store_f32<TOut>(o, e, v[e] + (g.add ? load_f32<TOut>(add, e) : 0.f));
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
}

// silu(gate) * up, quantised per row over the tile's 128 columns
template <int NT>
__device__ __forceinline__ void store_quantized(const SGemm &g, const Ctx &c, const MTile &mt, int n0, char *ring, f32x4 (&acc)[4][NT])
{
    constexpr int BM = NT * 32, STRIDE = 128 + 16;
    uint32_t *top = (uint32_t *)(ring + BM * STRIDE);          // [BM][4]
    static_assert(BM * STRIDE + BM * 16 <= kLds, "LDS");
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        uint32_t m = 0;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const bool live = n0 + c.wn * 32 + p * 16 < g.n;      // inter is a multiple of 16
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float h = silu_mul(acc[2 * p][t][e], acc[2 * p + 1][t][e]);
                acc[2 * p][t][e] = h;
                m = max(m, live ? magnitude(h) : 0u);
            }
        }
        m = max(m, (uint32_t)__shfl_xor((int)m, 16));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32));
        if (c.quad == 0) top[((2 * t + c.wm) * 16 + c.l15) * 4 + c.wn] = m;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = (2 * t + c.wm) * 16 + c.l15;
        const uint4 m = *(const uint4 *)(top + row * 4);
        const GroupScale s(__uint_as_float(max(max(m.x, m.y), max(m.z, m.w))));
#pragma unroll
        for (int p = 0; p < 2; ++p)
            *(uint32_t *)(ring + row * STRIDE + c.wn * 32 + p * 16 + c.quad * 4) =
                pack_e4m3(s.quotient(acc[2 * p][t][0]), s.quotient(acc[2 * p][t][1]), s.quotient(acc[2 * p][t][2]), s.quotient(acc[2 * p][t][3]));
    }
    __syncthreads();
    const int nb = n0 / kScaleBlock;
    for (int i = threadIdx.x; i < mt.rows * 16; i += kThreads) {
        const int row = i >> 4, col = n0 + (i & 15) * 8;
        if (col >= g.n) continue;
        *(uint2 *)(g.q + ((size_t)mt.row_begin + row) * g.ld_q + col) = *(const uint2 *)(ring + row * STRIDE + (i & 15) * 8);
    }
    for (int row = threadIdx.x; row < mt.rows; row += kThreads) {
        const uint4 m = *(const uint4 *)(top + row * 4);
        g.qs[((size_t)mt.row_begin + row) * g.ld_qs + nb] = GroupScale::scale(__uint_as_float(max(max(m.x, m.y), max(m.z, m.w))));
    }
}

template <int NT, bool kSwiglu, bool kExact, typename TOut>
__device__ __forceinline__ void run_tile(const SGemm &g, Ctx &c, const MTile &mt, int n0, char *ring)
{
    using R = Ring<NT>;
    // ---- what this lane copies ----
#pragma unroll
    for (int i = 0; i < R::WP; ++i) {
        const int row = (c.wave * R::WP + i) * 8 + (c.lane >> 3);
        const int chunk = (c.lane & 7) ^ swz8(row);
        int col;
        if (kSwiglu) col = min(n0 + (row >> 5) * 16 + (row & 15), g.n - 1);     // 16 gate rows, 16 up rows, ...
        else         col = min(n0 + row, g.n - 1);
        c.woff[i] = (uint32_t)(col - n0) * g.k + chunk * 16;
    }
    auto source = [&](int row) { const int r = mt.row_begin + min(row, mt.rows - 1); return g.perm ? g.perm[r] : r; };
    const int first = g.perm ? 0 : mt.row_begin;           // rows that follow each other are addressed from the tile's first
    c.abase = g.a + (size_t)first * g.ld_a;
    c.sbase = g.as + (size_t)first * g.ld_as;
#pragma unroll
    for (int i = 0; i < R::XP; ++i) {
        const int row = (c.wave * R::XP + i) * 8 + (c.lane >> 3);
        const int chunk = (c.lane & 7) ^ swz8(row);
        c.xoff[i] = (uint32_t)(source(row) - first) * (uint32_t)g.ld_a + chunk * 16;
    }
    c.soff = (uint32_t)(source(c.wave * 64 + c.lane) - first) * (uint32_t)g.ld_as * 4;

    const uint32_t lds = lds_addr(ring);
    f32x4 acc[4][NT];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[a][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    issue_scales<R>(c, lds, 0);
    // as the steps before the first would have done: step -1 fills the last stage but one of the weights and of the rows
    if (c.k < kRowBytes) {
        issue_copies<R, kSwiglu, true>(c, lds, 0, 0, 1 - R::NW);              // the weights of step 0, and with as many stages its rows
        if (R::NX != R::NW) issue_copies<R, kSwiglu, true>(c, lds, 1, 0, 1 - R::NX);
    } else {
#pragma unroll
        for (int b = 1 - R::NW; b < 0; ++b) issue_copies<R, kSwiglu, false>(c, lds, b + R::NW - 1, max(0, b + R::NX - 1), b);
    }
    int wat = 0, xat = 0, wfill = R::NW - 1, xfill = R::NX - 1;     // stages of step b, and of those that are fetched meanwhile
    const int sa_row = c.wide ? kGroup : 1, sa_step = c.wide ? 1 : R::BM;
    for (int b = 0; b < c.kb; ++b) {
        if (b + R::NW - 2 < c.kb) wait_loads<R::Young>();
        else                      wait_loads<0>();
        __syncthreads();   // everyone's share of step b is in LDS, and everyone is done with step b - 1
        char *ws = ring + wat * kWStage, *xs = ring + R::XBase + xat * R::XStage;
        if (c.k - b * kRowBytes < kRowBytes) {
            // a block that ends early: zero what is not its own, on both sides (fetched were the last 128 columns, or the first where there are no 128)
            const int own = (c.k - b * kRowBytes) / 16;
            for (int i = threadIdx.x; i < (kBN + R::BM) * 8; i += kThreads) {
                const int r = i >> 3, row = r < kBN ? r : r - kBN;
                if (c.k < kRowBytes ? (i & 7) >= own : (i & 7) < 8 - own)
                    *(uint4 *)((r < kBN ? ws : xs) + row * kRowBytes + (((i & 7) ^ swz8(row)) << 4)) = make_uint4(0, 0, 0, 0);
            }
            __syncthreads();
        }
        if ((b & (kGroup - 1)) == 0) issue_scales<R>(c, lds, b / kGroup + 1);
        const int half = (b / kGroup) & 1, j = b & (kGroup - 1);
        const float *sa = (const float *)(ring + R::Scales + half * (R::ScaleBytes / 2)) + j * sa_step;
        const float *sw = (const float *)(ring + R::WScales + half * 256) + j;
        const float sw0 = sw[kSwiglu ? 0 : (c.wn >> 1) * 4], sw1 = kSwiglu ? sw[4] : sw0;
        // (no branch around the copies: across one the compiler lets the multiply-adds slide to the step's end, and their operands out of the registers)
        multiply_step<NT, kSwiglu, kExact>(c, ws, xs, sa, sa_row, sw0, sw1, acc,
                                           [&](int t) __attribute__((always_inline)) { issue_between<R, kSwiglu>(c, lds, wfill, xfill, b, t); });
        wat = wat + 1 == R::NW ? 0 : wat + 1;
        xat = xat + 1 == R::NX ? 0 : xat + 1;
        wfill = wfill + 1 == R::NW ? 0 : wfill + 1;
        xfill = xfill + 1 == R::NX ? 0 : xfill + 1;
    }
    __syncthreads();   // all reads are done: the ring is the epilogue's
    if constexpr (kSwiglu) store_quantized<NT>(g, c, mt, n0, ring, acc);
    else                   store_rows<NT, TOut>(g, c, mt, n0, ring, acc);
}

// the body for nt parts of 32 rows
template <int NT, int kMaxNT, bool kSwiglu, bool kExact, typename TOut>
__device__ __forceinline__ void run_nt(int nt, const SGemm &g, Ctx &c, const MTile &mt, int n0, char *ring)
{
    if constexpr (NT == kMaxNT) run_tile<NT, kSwiglu, kExact, TOut>(g, c, mt, n0, ring);
    else if (nt <= NT) run_tile<NT, kSwiglu, kExact, TOut>(g, c, mt, n0, ring);
    else run_nt<NT + 1, kMaxNT, kSwiglu, kExact, TOut>(nt, g, c, mt, n0, ring);
}

// The items of a launch are (tile, slice of the weights); workgroup b works for XCD b % 8, whose share is a run of items.  Tiles are
// taken `together` at a time, slice by slice, so that a slice's weights are read by that many workgroups of one XCD while they are in its L2.
// us, 1, 2, 4 at a time, exact products (8-bit instructions): 8192^3 975, 935, 926 (509, 464, 454), 8192 x 7168 x 2048 241, 231, 224 (125, 120, 117);
// layers, where as many belong together as a slot has tiles of 128 (256) rows: DeepSeek-V3-shaped rank 8192 routed tokens, three (one), 1284, 1303, 1277 (818, 785,
// 787), 3000 tokens, one, 573, 590, 573 (410, 419, 428); Qwen3 shape 4096 tokens, two (one), 493, 493, 503 (313, 326, 355).
//
// A compute unit runs one workgroup at a time, so that a last round that is not full costs a whole one.  Where it fills half of an XCD's `cus` units or less, the
// rows of its tiles are shared out to two to four workgroups (parts of whole 32 rows; a row's sums are the same whichever runs it).  cus 0: never.
// us, whole -> shared out, exact (8-bit): 8192 x 7168 x 2048 227 -> 223 (123 -> 118), 3000 x 1408 x 7168 96 -> 97 (72 -> 49), swiglu of 3000 rows 1408 x 7168 195 -> 158;
// layers: DeepSeek-V3-shaped rank 3000 tokens 567 -> 577 (427 -> 410), 8192 1212 -> 1225 (798 -> 785), 16 of its experts 6000 tokens 837 -> 819 (491 -> 457),
// DeepSeek-V2-Lite shape 1777 tokens 320 -> 323 (214 -> 202), Qwen3 shape 4096 tokens 497 -> 492 (312 -> 314).
template <bool kSwiglu, bool kExact, int kMaxNT, typename TOut>
__global__ __launch_bounds__(kThreads, 1) void k_scaled_tiles(SGemm g, int slices, int tile_rows, int together, int cus)
{
    __shared__ __attribute__((aligned(1024))) char ring[kLds];
    const int tiles = g.tiles ? *g.n_tiles : (g.m + tile_rows - 1) / tile_rows;
    // (32 bits hold the items: a launch has fewer workgroups than that)
    const unsigned items = (unsigned)tiles * (unsigned)slices, share = (items + kXcds - 1) / kXcds;
    unsigned j = blockIdx.x / kXcds, parts = 1, part = 0;
    if (cus > 0) {
        const unsigned left = share % (unsigned)cus, whole = share - left;
        if (j >= whole) {
            parts = left > 0 ? max(1u, min(4u, (unsigned)cus / left)) : 1;
            part = (j - whole) % parts;
            j = whole + (j - whole) / parts;
        }
    }
    const unsigned i = (blockIdx.x % kXcds) * share + j;
    if (j >= share || i >= items) return;
    const int set = (int)(i / ((unsigned)together * (unsigned)slices)) * together, width = min(together, tiles - set);
    const int in_set = (int)(i - (unsigned)set * (unsigned)slices);
    const int tile = set + in_set % width, n0 = in_set / width * (kSwiglu ? kBN / 2 : kBN);
    MTile mt = {0, tile * tile_rows, min(tile_rows, g.m - tile * tile_rows), 0};
    if (g.tiles) {
        const MTile m = g.tiles[tile];
        mt = {__builtin_amdgcn_readfirstlane(m.slot), __builtin_amdgcn_readfirstlane(m.row_begin), __builtin_amdgcn_readfirstlane(m.rows),
              __builtin_amdgcn_readfirstlane(m.single)};
    }
    if (parts > 1) {
        const int rows = ((mt.rows + (int)parts - 1) / (int)parts + 31) & ~31, begin = (int)part * rows;
        if (begin >= mt.rows) return;
        mt.row_begin += begin;
        mt.rows = min(rows, mt.rows - begin);
    }

    Ctx c;
    c.lane = threadIdx.x & 63;
    c.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    c.wm = c.wave >> 2; c.wn = c.wave & 3;
    c.l15 = c.lane & 15; c.quad = c.lane >> 4;
    c.k = g.k; c.kb = g.kb;
    c.wbase = g.w + (size_t)mt.slot * g.w_slot + (size_t)n0 * g.k;
    c.up = (size_t)g.n * g.k;
    const int nb = scale_blocks(g.n), nb0 = n0 / kScaleBlock;
    c.wsbase = g.ws + (size_t)mt.slot * g.ws_slot + (size_t)nb0 * g.kb;
    c.wsoff = (c.lane & 4) ? (uint32_t)(kSwiglu ? nb : min(1, nb - 1 - nb0)) * (uint32_t)g.kb * 4 : 0;
    c.wide = g.kb % kGroup == 0 && g.ld_as % kGroup == 0 && ((uintptr_t)g.as & 15) == 0;
    c.once = parts == 1 && (g.tiles ? mt.single != 0 : tiles == 1);
    const int nt = (mt.rows + 31) >> 5;
    run_nt<1, kMaxNT, kSwiglu, kExact, TOut>(nt, g, c, mt, n0, ring);
}

int tail_parts(long long left, int cus) { return left > 0 ? (int)std::max(1ll, std::min(4ll, cus / left)) : 1; }

// compute units of an XCD of the current device (looked up once per device)
int cus_per_xcd()
{
    static std::atomic<int> cus_of[64] = {};
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 32;
    n = cus_of[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < kXcds) n = 32 * kXcds;
        n /= kXcds;
        cus_of[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

template <bool kSwiglu, bool kExact, int kMaxNT, typename TOut>
void launch_as(const SGemm &g, int tile_rows, hipStream_t st)
{
    const int slices = tiles_slices(g.n, kSwiglu);
    const long long tiles = g.tiles ? g.max_tiles : (g.m + tile_rows - 1) / tile_rows;
    const long long share = (tiles * slices + kXcds - 1) / kXcds;
    const int cus = g.split_tail ? cus_per_xcd() : 0;
    const long long blocks = !cus ? share : g.tiles ? share + cus : share / cus * cus + (share % cus ? (share % cus) * tail_parts(share % cus, cus) : 0);
    hipLaunchKernelGGL((k_scaled_tiles<kSwiglu, kExact, kMaxNT, TOut>), dim3((unsigned)(blocks * kXcds)), dim3(kThreads), 0, st, g, slices, tile_rows, g.together, cus);
}

}  // namespace

int tiles_slices(int n, bool swiglu) { return (n + (swiglu ? kBN / 2 : kBN) - 1) / (swiglu ? kBN / 2 : kBN); }

// Rounds of the chip times the time of a workgroup: its K-steps and 4 to 6 us for the first copies and the stores.  us a K-step by the tile's 32-row
// parts, of launches that leave compute units idle .. fill the chip: 1 0.62, 2 0.81, 4 1.0 .. 1.19, 6 1.31 .. 1.55, 8 1.5 .. 2.0; exact products 1 1.08, 2 1.36, 4 1.78.
// The last round's tiles may be shared out (see the kernel).  (Without a GPU, where refusals are tested: 32 units.)
double tiles_us(long long tiles, int tile_rows, int n, int k, bool swiglu, bool exact)
{
    const auto workgroup = [&](int rows) {
        const int nt = (rows + 31) / 32;
        const double step = exact ? (nt <= 1 ? 1.08 : nt <= 2 ? 1.36 : 1.78) : nt <= 1 ? 0.62 : nt <= 2 ? 0.81 : nt <= 4 ? 1.1 : nt <= 6 ? 1.45 : 1.85;
        return scale_blocks(k) * step + 3.5 + 0.25 * nt;
    };
    constexpr int kCus = 32;
    const long long share = (tiles * tiles_slices(n, swiglu) + kXcds - 1) / kXcds, left = share % kCus;
    const int parts = tile_rows > 64 ? tail_parts(left, kCus) : 1;
    return (double)(share / kCus) * workgroup(tile_rows) + (left ? workgroup((tile_rows + parts - 1) / parts) : 0.0);
}

hipError_t launch_scaled_tiles(const SGemm &g, TilesOut out, int tile_rows, hipStream_t st)
{
    switch (out) {
    case TilesOut::bf16:         launch_as<false, true, 4, uint16_t>(g, tile_rows, st); break;
    case TilesOut::f32:          launch_as<false, true, 4, float>(g, tile_rows, st); break;
    case TilesOut::fast_bf16:    launch_as<false, false, 8, uint16_t>(g, tile_rows, st); break;
    case TilesOut::block16:      launch_as<false, false, 8, Block16>(g, tile_rows, st); break;
    case TilesOut::swiglu:       launch_as<true, false, 8, float>(g, tile_rows, st); break;
    case TilesOut::swiglu_exact: launch_as<true, true, 4, float>(g, tile_rows, st); break;
    }
    return hipGetLastError();
}

}  // namespace emoe
