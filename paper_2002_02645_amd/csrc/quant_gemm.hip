// The dense layer on rows held in 8 bits (gfx950 / CDNA4):
//
//     y[r, c] = act(bias[c] + sum_B 2^(Ex[r, B] + Ew[c, B]) sum_{i in B} x8[r, i] w8[c, i])
//
// A k-step is a block of 128 codes: 128 bytes a row, copied as they are into LDS (direct loads) with the scale bytes of the four
// blocks it belongs to; both operands are laid out so that a stage is a run of memory (QuantRows).  Two forms of the inner product:
//   - fp32 outputs (and small tiles): codes widen to bf16 in registers, their scale applied by the same instruction, exactly;
//     bf16 matrix instructions, exact products summed in fp32.
//   - bf16 outputs of tiles of 256 rows (F8): the 8-bit matrix instructions with their scales, at twice the rate.  They cut the products
//     of eight neighbours off 13 bits below the largest's exponent: measured against 64 bits 1.4e-5 of the result's
//     norm on normal values, 8e-5 with a few channels far larger.  A bf16 output is rounded by 1.7e-3; an fp32 one is not
//     worth its bits then, which is why it does not go this way.
// Work: the flattened (tile, k-step) space in ranges, whole tiles where they fill the chip, else even ranges whose cut tiles
// leave their sums in slots, added in order by quant_sum_kernel.
#include "../../include/freeze.h"
#include "quantised.h"

#include <algorithm>
#include <type_traits>
#include <utility>

namespace fz {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((address_space(3))) void *lds_void_ptr;

namespace {

// four codes of a word times 2^(exponent of s): four bf16, exact
__device__ __forceinline__ u32x2 widen(uint32_t codes, float s)
{
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes, s, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes, s, true))};
}
__device__ __forceinline__ bf16x8 widen8(uint32_t c0, uint32_t c1, float s)
{
    const u32x2 a = widen(c0, s), b = widen(c1, s);
    return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) { return (uint32_t)bf16_rne(a) | ((uint32_t)bf16_rne(b) << 16); }

// outputs col .. col + 3 of a row
__device__ __forceinline__ void store_outputs(const QuantProduct &p, int64_t row, int64_t col, f32x4 v)
{
    if (col >= p.m) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (p.bias) v[e] += p.bias[col + e < p.m ? col + e : p.m - 1];
        if (p.relu) v[e] = __builtin_fmaxf(v[e], 0.f);
    }
    const int64_t at = row * p.out_stride + col;
    if (p.vec && col + 4 <= p.m) {
        if (p.out_bf16) *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(p.out) + at) = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        else *reinterpret_cast<f32x4 *>(static_cast<float *>(p.out) + at) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (col + e >= p.m) continue;
            if (p.out_bf16) static_cast<uint16_t *>(p.out)[at + e] = bf16_rne(v[e]);
            else static_cast<float *>(p.out)[at + e] = v[e];
        }
    }
}

// Tiles in the order in which ranges take them: four tiles of x rows side by side, so that the workgroups of an XCD, which
// are at neighbouring places of that order, share both operands in its L2.
constexpr int kTileGroup = 4;
__device__ __forceinline__ void tile_place(const QuantProduct &p, int64_t tile, int *xt, int *wt)
{
    const int64_t group = tile / (kTileGroup * (int64_t)p.w_tiles);
    const int first = (int)group * kTileGroup, wide = p.x_tiles - first < kTileGroup ? p.x_tiles - first : kTileGroup;
    const int r = (int)(tile - group * kTileGroup * p.w_tiles);
    *xt = first + r % wide;
    *wt = r / wide;
}

// LDS-direct loads to a constant distance behind a wave's place (formed in M0 itself: as many places as a stage has loads, kept over
// the loop, would not fit the scalar registers).  Stages are runs of memory: a wave's load is 1 KiB at lane * 16, or 256 bytes at lane * 4.
template <int TO>
__device__ __forceinline__ void load16_to_lds_at(uint64_t sbase, uint32_t voff, uint32_t lds)
{
    asm volatile("s_add_u32 m0, %0, %3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(sbase), "n"(TO) : "memory", "m0", "scc");
}
template <int TO>
__device__ __forceinline__ void load4_to_lds_at(uint64_t sbase, uint32_t voff, uint32_t lds)
{
    asm volatile("s_add_u32 m0, %0, %3\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(voff), "s"(sbase), "n"(TO) : "memory", "m0", "scc");
}
template <int... I, class F>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F f)
{
    (f(std::integral_constant<int, I>{}), ...);
}

// A wave's sums: the matrix instructions take w as their rows, so a lane holds four consecutive outputs (from col on, and 16 j behind)
// of one x row (row, and 16 i behind).
template <int XB, int NB, int BM, int BN>
__device__ __forceinline__ void tile_out(const QuantProduct &p, const f32x4 (&acc)[XB][NB], int64_t range, int64_t tile, bool whole, int row, int col,
                                         int64_t x0, int64_t w0, int x_last)
{
    if (whole) {   // uniform
        each(std::make_integer_sequence<int, XB * NB>{}, [&](auto ij) {
            constexpr int i = decltype(ij)::value / NB, j = decltype(ij)::value % NB;
            if (row + 16 * i <= x_last) store_outputs(p, x0 + row + 16 * i, w0 + col + 16 * j, acc[i][j]);
        });
    } else {
        const int slot = (int)(range - tile * p.nk / p.len);   // how many ranges before this one touch the tile
        float *dst = p.part + ((tile * p.slots + slot) * BM + row) * BN + col;
        each(std::make_integer_sequence<int, XB * NB>{}, [&](auto ij) {
            constexpr int i = decltype(ij)::value / NB, j = decltype(ij)::value % NB;
            *reinterpret_cast<f32x4 *>(dst + i * 16 * BN + j * 16) = acc[i][j];
        });
    }
}

// Batches of few rows: eight waves of XB x NB blocks of 16 x 16 outputs, WX of them along x; NS stages.  Bound by the memory that the
// weights come from: what counts is how many bytes are on their way.
template <int WX, int WN, int XB, int NB, int NS>
__global__ __launch_bounds__(512, 2) void quant_gemm_kernel(QuantProduct p)
{
    static_assert(WX * WN == 8, "eight waves");
    constexpr int BM = WX * XB * 16, BN = WN * NB * 16;
    constexpr int kX = BN * 128, kS = kX + BM * 128, kStage = kS + (BN + (BM < 64 ? 64 : BM)) * 4;
    constexpr int IW = BN / 64, LX = BM / 8, IX = (LX + 7) / 8;        // load instructions: of a wave, of all, of a wave
    constexpr int LS = BN / 64 + (BM + 63) / 64, NL = IW + IX + 1;
    static_assert(kQuantTile % BN == 0 && LS <= 8 && NS * kStage <= 163840 && (NS - 2) * NL <= 63, "");
    __shared__ __attribute__((aligned(16))) unsigned char smem[NS * kStage];

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wx = w / WN, wn = w % WN;
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_void_ptr)smem;
    const int nk = p.nk;

    const int64_t range = p.xcd_share ? (int64_t)(blockIdx.x & 7) * p.xcd_share + (blockIdx.x >> 3) : blockIdx.x;
    const int64_t total = (int64_t)p.x_tiles * p.w_tiles * nk;
    const int64_t g_begin = range * p.len, g_end = g_begin + p.len < total ? g_begin + p.len : total;

    const int g4 = lane >> 4;
    const int rX = wx * XB * 16 + (lane & 15), rW = wn * NB * 16 + (lane & 15);   // + 16 i: leaves the swizzle as it is
    const int swX = row128_swizzle(rX), swW = row128_swizzle(rW);
    // the wave's loads (where there are fewer than waves, the last ones repeat one)
    const int lx = w < LX ? w : LX - 1, ls = w < LS ? w : LS - 1;
    const uint32_t off16 = lane * 16;
    // (of fewer rows than lanes the last row's scales are loaded again)
    const uint32_t off4 = (ls < BN / 64 || BM >= 64 || lane < BM ? lane : BM - 1) * 4;

    for (int64_t g = g_begin; g < g_end;) {
        const int64_t tile = g / nk;
        const int ka = (int)(g - tile * nk);
        const int kb = g_end - tile * nk < nk ? (int)(g_end - tile * nk) : nk;
        int xt, wt;
        tile_place(p, tile, &xt, &wt);
        const int64_t x0 = (int64_t)xt * BM, w0 = (int64_t)wt * BN;
        const int x_last = (int)(p.b - x0 < BM ? p.b - x0 : BM) - 1;
        const int64_t wbig = w0 / kQuantTile * kQuantTile, win = w0 - wbig;   // the tile of the weights, the place within it
        const uint64_t gX = uniform_u64((uint64_t)(uintptr_t)(p.x + x0 * p.d_pad) + lx * 1024);
        const uint64_t gW = uniform_u64((uint64_t)(uintptr_t)(p.w + wbig * p.d_pad + win * 128) + w * 1024);
        const uint64_t gS = uniform_u64((uint64_t)(uintptr_t)(ls < BN / 64 ? p.ws + wbig * p.sd + win * 4 + ls * 256 : p.xs + x0 * p.sd + (ls - BN / 64) * 256));
        const uint32_t s_rows = ls < BN / 64 ? kQuantTile * 4 : BM * 4;
        auto issue = [&](int buf, int kt) {
            const uint32_t to = smem_base + buf * kStage;
            const uint64_t kw = gW + (uint64_t)kt * (kQuantTile * 128), kx = gX + (uint64_t)kt * (BM * 128);
            each(std::make_integer_sequence<int, IW>{}, [&](auto i) {
                load16_to_lds_at<decltype(i)::value * 8192>(kw + decltype(i)::value * 8192, off16, to + w * 1024);
            });
            each(std::make_integer_sequence<int, IX>{}, [&](auto i) {
                load16_to_lds_at<kX + decltype(i)::value * 8192>(kx + decltype(i)::value * 8192, off16, to + lx * 1024);
            });
            load4_to_lds_at<kS>(gS + (uint64_t)(kt >> 2) * s_rows, off4, to + ls * 256);
        };

        f32x4 acc[XB][NB];
#pragma unroll
        for (int i = 0; i < XB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

        const int klast = kb - 1;
        __syncthreads();   // the LDS is free (a range's previous tile)
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) issue(s, ka + s < klast ? ka + s : klast);
        int st = 0;
        for (int kt = ka; kt < kb; ++kt) {
            wait_global_loads_le<(NS - 2) * NL>();
            __syncthreads();   // this step's stage is there, the one before has been read
            const int fill = st == 0 ? NS - 1 : st - 1;
            issue(fill, kt + NS - 1 < klast ? kt + NS - 1 : klast);
            const unsigned char *stage = smem + st * kStage;
            const u32x4 *tw = reinterpret_cast<const u32x4 *>(stage), *tx = reinterpret_cast<const u32x4 *>(stage + kX);
            const uint32_t *sw = reinterpret_cast<const uint32_t *>(stage + kS), *sx = sw + BN;
            const int sh = 8 * (kt & 3);
            float fx[XB], fw[NB];
#pragma unroll
            for (int i = 0; i < XB; ++i) fx[i] = __uint_as_float((sx[rX + 16 * i] >> sh & 255u) << 23);
#pragma unroll
            for (int j = 0; j < NB; ++j) fw[j] = __uint_as_float((sw[rW + 16 * j] >> sh & 255u) << 23);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 xa[2][XB];
#pragma unroll
                for (int i = 0; i < XB; ++i) {
                    const u32x4 a = tx[(rX + 16 * i) * 8 + ((2 * g4 + h) ^ swX)];
                    xa[0][i] = widen8(a[0], a[1], fx[i]);
                    xa[1][i] = widen8(a[2], a[3], fx[i]);
                }
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const u32x4 a = tw[(rW + 16 * j) * 8 + ((2 * g4 + h) ^ swW)];
                    const bf16x8 w0v = widen8(a[0], a[1], fw[j]), w1v = widen8(a[2], a[3], fw[j]);
#pragma unroll
                    for (int i = 0; i < XB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w0v, xa[0][i], acc[i][j], 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < XB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w1v, xa[1][i], acc[i][j], 0, 0, 0);
                }
            }
            st = st + 1 == NS ? 0 : st + 1;
        }
        wait_global_loads_le<0>();   // the refills past the last k-step
        tile_out<XB, NB, BM, BN>(p, acc, range, tile, ka == 0 && kb == nk, wx * XB * 16 + (lane & 15), wn * NB * 16 + g4 * 4, x0, w0, x_last);
        g = tile * nk + kb;
    }
}

// Tiles of 256 x 256 for the batches that the matrix pipes bound.  A wave forms 16 XB x 128 outputs: 8-bit form XB = 8, four waves, one a
// SIMD (the sums take half of its registers; a k-step reads 128 KiB of fragments out of LDS, with eight waves it would be 192 in
// half the time of the bf16 form); bf16 form XB = 4, eight waves, so that one of a SIMD's widens codes while the other's matrix instructions run.  A
// step goes through its blocks of 16 w rows, in the bf16 form twice (64 codes each); fragments are read kAhead blocks ahead.  The step's
// barrier comes before its last kAhead blocks of matrix instructions, which need nothing newer: it publishes the
// next step's stage and frees this one, which is refilled from there on.
template <bool F8, int XB>
__global__ __launch_bounds__(2048 / XB, 8 / XB) void quant_tile_kernel(QuantProduct p)
{
    using frag = std::conditional_t<F8, i32x8, u32x4>;
    constexpr int BM = 256, BN = 256, NB = 8, kWaves = 32 / XB;
    static_assert(BM == kQuantTile && BN == kQuantTile, "a stage is a run of memory");
    constexpr int kX = BN * 128, kS = kX + BM * 128, kStage = kS + (BN + BM) * 4;
    constexpr int kHalves = F8 ? 1 : 2, kAhead = 2, kRing = 4;
    constexpr int NC = 32 / kWaves, NS = 8 / kWaves, NL = 2 * NC + NS;   // load instructions of a wave and step: codes of an operand, scales, all
    constexpr int kPerGroup = (NL + kAhead - 1) / kAhead;
    static_assert(2 * kStage <= 163840 && NB % kRing == 0, "");
    __shared__ __attribute__((aligned(16))) unsigned char smem[2 * kStage];

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wx = w >> 1, wn = w & 1;
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_void_ptr)smem;
    const int nk = p.nk;

    const int64_t range = p.xcd_share ? (int64_t)(blockIdx.x & 7) * p.xcd_share + (blockIdx.x >> 3) : blockIdx.x;
    const int64_t total = (int64_t)p.x_tiles * p.w_tiles * nk;
    const int64_t g_begin = range * p.len, g_end = g_begin + p.len < total ? g_begin + p.len : total;

    const int g4 = lane >> 4;
    const int rX = wx * 16 * XB + (lane & 15), rW = wn * 128 + (lane & 15);   // + 16 i: leaves the swizzle as it is
    const int swX = row128_swizzle(rX), swW = row128_swizzle(rW);
    const uint32_t off16 = lane * 16, off4 = lane * 4;
    const uint32_t lds16 = smem_base + w * 1024, lds4 = smem_base + w * 256;

    for (int64_t g = g_begin; g < g_end;) {
        const int64_t tile = g / nk;
        const int ka = (int)(g - tile * nk);
        const int kb = g_end - tile * nk < nk ? (int)(g_end - tile * nk) : nk;
        int xt, wt;
        tile_place(p, tile, &xt, &wt);
        const int64_t x0 = (int64_t)xt * BM, w0 = (int64_t)wt * BN;
        const int x_last = (int)(p.b - x0 < BM ? p.b - x0 : BM) - 1;
        const uint64_t gX = uniform_u64((uint64_t)(uintptr_t)(p.x + x0 * p.d_pad) + w * 1024), gW = uniform_u64((uint64_t)(uintptr_t)(p.w + w0 * p.d_pad) + w * 1024);
        // scales: four waves bring both operands', or four each one's
        const bool s_of_w = NS == 2 || w < 4;
        const uint64_t gS = uniform_u64((uint64_t)(uintptr_t)(s_of_w ? p.ws + w0 * p.sd : p.xs + x0 * p.sd) + (w & 3) * 256);
        const uint64_t gS2 = uniform_u64((uint64_t)(uintptr_t)(p.xs + x0 * p.sd) + (w & 3) * 256);
        // load l of k-step kt's stage
        auto issue = [&](int buf, int kt, auto l_) {
            constexpr int l = decltype(l_)::value;
            const uint32_t st = buf * kStage;
            const uint64_t k = (uint64_t)kt * 32768, q = (uint64_t)(kt >> 2) * 1024;
            if constexpr (l < NC) load16_to_lds_at<l * kWaves * 1024>(gW + k + l * kWaves * 1024, off16, lds16 + st);
            else if constexpr (l < 2 * NC) load16_to_lds_at<kX + (l - NC) * kWaves * 1024>(gX + k + (l - NC) * kWaves * 1024, off16, lds16 + st);
            else if constexpr (l == 2 * NC) load4_to_lds_at<kS>(gS + q, off4, lds4 + st);   // (eight waves: the second four's lie behind the first's)
            else if constexpr (l < NL) load4_to_lds_at<kS + BN * 4>(gS2 + q, off4, lds4 + st);
        };

        f32x4 acc[XB][NB];
#pragma unroll
        for (int i = 0; i < XB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

        frag wr[kRing];            // fragments of w ahead, with the scale bytes of their rows
        uint32_t ew[kRing];
        frag xr[XB];               // of x: 8-bit form, this step's; bf16 form, the next 64 codes
        bf16x8 xa[F8 ? 1 : XB][2];
        uint32_t ex[XB];
        auto read = [&](frag &to, const unsigned char *base, int row, int sw, int h) {
            const u32x4 *t = reinterpret_cast<const u32x4 *>(base) + row * 8;
            if constexpr (F8) {
                const u32x4 a = t[(2 * g4) ^ sw], b = t[(2 * g4 + 1) ^ sw];
                to = i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
            } else {
                to = t[(2 * g4 + h) ^ sw];
            }
        };
        auto read_w = [&](int set, int buf, int j, int h) {
            read(wr[set], smem + buf * kStage, rW + 16 * j, swW, h);
            ew[set] = *reinterpret_cast<const uint32_t *>(smem + buf * kStage + kS + (rW + 16 * j) * 4);
        };
        auto read_x = [&](int buf, int i, int h) { read(xr[i], smem + buf * kStage + kX, rX + 16 * i, swX, h); };
        auto read_xs = [&](int buf, int i) { ex[i] = *reinterpret_cast<const uint32_t *>(smem + buf * kStage + kS + (BN + rX + 16 * i) * 4); };

        const int klast = kb - 1;
        auto at_most = [&](int kt) { return kt < klast ? kt : klast; };
        __syncthreads();   // the LDS is free (a range's previous tile)
        each(std::make_integer_sequence<int, NL>{}, [&](auto l) { issue(0, ka, l); });
        each(std::make_integer_sequence<int, NL>{}, [&](auto l) { issue(1, at_most(ka + 1), l); });
        wait_global_loads_le<NL>();
        __syncthreads();
#pragma unroll
        for (int i = 0; i < XB; ++i) {
            read_x(0, i, 0);
            read_xs(0, i);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) read_w(j, 0, j, 0);
        int st = 0;
        for (int kt = ka; kt < kb; ++kt) {
            const int nst = st ^ 1, sh = 8 * (kt & 3);
            if constexpr (F8) {
#pragma unroll
                for (int i = 0; i < XB; ++i) ex[i] >>= sh;
            }
            each(std::make_integer_sequence<int, kHalves * NB>{}, [&](auto hj) {
                constexpr int h = decltype(hj)::value / NB, j = decltype(hj)::value % NB;
                constexpr bool last_half = h == kHalves - 1;
                if constexpr (last_half && j == NB - kAhead) {
                    wait_global_loads_le<0>();
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    __syncthreads();
                }
                if constexpr (j + kAhead < NB) read_w((j + kAhead) % kRing, st, j + kAhead, h);
                else read_w((j + kAhead) % kRing, last_half ? nst : st, j + kAhead - NB, last_half ? 0 : h + 1);
                if constexpr (!F8 && j >= NB - kAhead) {
#pragma unroll
                    for (int i = (j - NB + kAhead) * XB / kAhead; i < (j - NB + kAhead + 1) * XB / kAhead; ++i) {
                        read_x(last_half ? nst : st, i, last_half ? 0 : h + 1);
                        if (last_half) read_xs(nst, i);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (last_half && j >= NB - kAhead)
                    each(std::make_integer_sequence<int, kPerGroup>{}, [&](auto l) {
                        issue(st, at_most(kt + 2), std::integral_constant<int, (j - NB + kAhead) * kPerGroup + decltype(l)::value>{});
                    });
                if constexpr (F8) {
                    const int e = (int)(ew[j % kRing] >> sh);
#pragma unroll
                    for (int i = 0; i < XB; ++i) {
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wr[j % kRing], xr[i], acc[i][j], 0, 0, 0, e, 0, (int)ex[i]);
                        if constexpr (j == NB - 1) {   // the block's last use: the next step's takes its place
                            read_x(nst, i, 0);
                            read_xs(nst, i);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                } else {
                    const float fw = __uint_as_float((ew[j % kRing] >> sh & 255u) << 23);
                    const u32x4 a = wr[j % kRing];
                    const bf16x8 w0v = widen8(a[0], a[1], fw), w1v = widen8(a[2], a[3], fw);
#pragma unroll
                    for (int i = 0; i < XB; ++i) {
                        if constexpr (j == 0) {
                            const float fx = __uint_as_float((ex[i] >> sh & 255u) << 23);
                            xa[i][0] = widen8(xr[i][0], xr[i][1], fx);
                            xa[i][1] = widen8(xr[i][2], xr[i][3], fx);
                        }
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w0v, xa[i][0], acc[i][j], 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < XB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w1v, xa[i][1], acc[i][j], 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            st = nst;
        }
        wait_global_loads_le<0>();   // the refills past the last k-step
        tile_out<XB, NB, BM, BN>(p, acc, range, tile, ka == 0 && kb == nk, rX, wn * 128 + g4 * 4, x0, w0, x_last);
        g = tile * nk + kb;
    }
}

// The outputs of cut tiles: the sums of a tile's slots in order, 256 threads for 1,024 outputs.
__global__ __launch_bounds__(256) void quant_sum_kernel(QuantProduct p, int bm, int bn)
{
    const int per_tile = bm * bn / 1024;
    const int64_t tile = blockIdx.x / per_tile;
    const int64_t first = tile * p.nk / p.len, last = (tile * p.nk + p.nk - 1) / p.len;
    if (first == last) return;   // uniform: written by its range
    int xt, wt;
    tile_place(p, tile, &xt, &wt);
    const int at = (int)(blockIdx.x % per_tile) * 1024 + threadIdx.x * 4, row = at / bn, col = at % bn;
    if ((int64_t)xt * bm + row >= p.b) return;
    const float *src = p.part + (tile * p.slots) * bm * bn + at;
    const int ns = (int)(last - first) + 1;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < ns; s += 4) {   // four in flight, and summed before they are added
        f32x4 t[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            t[u] = *reinterpret_cast<const f32x4 *>(src + (int64_t)(s + u < ns ? s + u : s) * bm * bn);
            if (s + u >= ns) t[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        v += (t[0] + t[1]) + (t[2] + t[3]);
    }
    store_outputs(p, (int64_t)xt * bm + row, (int64_t)wt * bn + col, v);
}

struct Variant {
    int bm, bn, per_cu;
    float step_us;   // of a k-step of a workgroup, all CUs at work
    void (*kernel)(QuantProduct);
    int threads;
};
const Variant kVariants[] = {
    {16, 128, 2, 1.2f, quant_gemm_kernel<1, 8, 1, 1, 4>, 512},
    {32, 128, 2, 1.2f, quant_gemm_kernel<1, 8, 2, 1, 3>, 512},
    {64, 128, 2, 1.3f, quant_gemm_kernel<1, 8, 4, 1, 3>, 512},
    {128, 256, 1, 1.5f, quant_gemm_kernel<2, 4, 4, 4, 3>, 512},
    {256, 256, 1, 2.2f, quant_tile_kernel<false, 4>, 512},
    {256, 256, 1, 1.2f, quant_tile_kernel<true, 4>, 512},
};

}  // namespace

QuantPlan plan_quant_product(int64_t b, int64_t m, int64_t d_pad, bool out_bf16, int num_cus)
{
    QuantPlan pl{};
    pl.variant = b <= 16 ? 0 : (b <= 32 ? 1 : (b <= 64 ? 2 : (b <= 128 ? 3 : (out_bf16 ? 5 : 4))));
    const Variant &v = kVariants[pl.variant];
    pl.bm = v.bm;
    pl.bn = v.bn;
    pl.x_tiles = (int)((b + v.bm - 1) / v.bm);
    pl.w_tiles = (int)((m + v.bn - 1) / v.bn);
    pl.nk = (int)(d_pad / kQuantBlock);
    const int64_t tiles = (int64_t)pl.x_tiles * pl.w_tiles, total = tiles * pl.nk, wgs = (int64_t)num_cus * v.per_cu;
    // Whole tiles, or even ranges with the sums of cut tiles through memory (written and read at 4 TB/s, and a launch).
    const int64_t whole = (tiles + wgs - 1) / wgs * pl.nk;
    int64_t even = (total + wgs - 1) / wgs;
    even = even < 4 ? 4 : even;
    const double join_us = 5.0 + 2.0 * 4.0 * (double)std::min<int64_t>(tiles, wgs) * v.bm * v.bn * (even < pl.nk ? (double)pl.nk / even : 1.0) / 4e6;
    pl.len = (double)whole * v.step_us <= (double)even * v.step_us + join_us ? pl.nk : even;   // (whole tiles: a workgroup each)
    pl.wgs = (int)((total + pl.len - 1) / pl.len);
    if (pl.len % pl.nk != 0) {
        pl.slots = (int)((pl.nk - 1) / pl.len + 2);
        pl.part = (size_t)tiles * pl.slots * v.bm * v.bn;
    }
    return pl;
}

hipError_t launch_quant_product(const QuantPlan &pl, QuantProduct p, hipStream_t s)
{
    p.len = pl.len;
    p.nk = pl.nk;
    p.x_tiles = pl.x_tiles;
    p.w_tiles = pl.w_tiles;
    p.slots = pl.slots;
    p.xcd_share = pl.wgs % 8 == 0 ? pl.wgs / 8 : 0;
    const int size = p.out_bf16 ? 2 : 4;
    p.vec = p.out_stride % 4 == 0 && reinterpret_cast<uintptr_t>(p.out) % (4 * size) == 0;
    const Variant &v = kVariants[pl.variant];
    hipLaunchKernelGGL(v.kernel, dim3((unsigned)pl.wgs), dim3((unsigned)v.threads), 0, s, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || pl.part == 0) return e;
    const int64_t tiles = (int64_t)pl.x_tiles * pl.w_tiles;
    hipLaunchKernelGGL(quant_sum_kernel, dim3((unsigned)(tiles * (pl.bm * pl.bn / 1024))), dim3(256), 0, s, p, pl.bm, pl.bn);
    return hipGetLastError();
}

}  // namespace fz
