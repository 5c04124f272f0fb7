// The dense layer on rows held in 8 bits (gfx950 / CDNA4):
//
//     y[r, c] = act(bias[c] + sum_B 2^(Ex[r, B] + Ew[c, B]) sum_{i in B} x8[r, i] w8[c, i])
//
// A k-step is a block of 128 codes: 128 bytes a row, copied as they are into LDS (direct loads, NS stages) with the scale bytes
// of the four blocks it belongs to.  Two forms of the inner product:
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

// WX x WN waves, each XB x NB blocks of 16 x 16 outputs (x rows, w rows); NS stages
template <int WX, int WN, int XB, int NB, int NS, bool F8>
__global__ __launch_bounds__(512, 2) void quant_gemm_kernel(QuantProduct p)
{
    static_assert(WX * WN == 8, "eight waves");
    constexpr int BM = WX * XB * 16, BN = WN * NB * 16;
    constexpr int kXScales = (BM + 63) / 64 * 64;   // a load instruction brings those of 64 rows
    constexpr int kX = BN * 128, kS = kX + BM * 128, kStage = kS + (BN + kXScales) * 4;
    constexpr int IW = BN / 64, IX = (BM / 8 + 7) / 8, IS = BN / 64 + kXScales / 64;   // load instructions: of a wave, of a wave, of all
    constexpr int NL = IW + IX + 1;
    static_assert(IS <= 8 && NS * kStage <= 163840 && (NS - 2) * NL <= 63, "");
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

    for (int64_t g = g_begin; g < g_end;) {
        const int64_t tile = g / nk;
        const int ka = (int)(g - tile * nk);
        const int kb = g_end - tile * nk < nk ? (int)(g_end - tile * nk) : nk;
        int xt, wt;
        tile_place(p, tile, &xt, &wt);
        const int64_t x0 = (int64_t)xt * BM, w0 = (int64_t)wt * BN;
        const int x_last = (int)(p.b - x0 < BM ? p.b - x0 : BM) - 1, w_last = (int)(p.m - w0 < BN ? p.m - w0 : BN) - 1;
        const uint64_t gX = uniform_u64((uint64_t)(uintptr_t)(p.x + x0 * p.d_pad)), gW = uniform_u64((uint64_t)(uintptr_t)(p.w + w0 * p.d_pad));
        // a lane's place in each load: rows behind the last one are met by that row again
        uint32_t offX[IX], offW[IW], offS;
        uint32_t toX[IX];
#pragma unroll
        for (int i = 0; i < IX; ++i) {
            int id = i * 8 + w;
            id = id < BM / 8 ? id : BM / 8 - 1;   // (the last waves of a small tile repeat a load)
            const int r = id * 8 + (lane >> 3);
            offX[i] = (uint32_t)(r < x_last ? r : x_last) * (uint32_t)p.d_pad + (uint32_t)(((lane & 7) ^ row128_swizzle(r)) * 16);
            toX[i] = kX + id * 1024;
        }
#pragma unroll
        for (int i = 0; i < IW; ++i) {
            const int r = (i * 8 + w) * 8 + (lane >> 3);
            offW[i] = (uint32_t)(r < w_last ? r : w_last) * (uint32_t)p.d_pad + (uint32_t)(((lane & 7) ^ row128_swizzle(r)) * 16);
        }
        const int sid = w < IS ? w : IS - 1;
        const bool s_of_w = sid < BN / 64;
        const uint64_t gS = uniform_u64((uint64_t)(uintptr_t)(s_of_w ? p.ws + w0 * p.sd : p.xs + x0 * p.sd));
        {
            const int r = (s_of_w ? sid : sid - BN / 64) * 64 + lane, last = s_of_w ? w_last : x_last;
            offS = (uint32_t)(r < last ? r : last) * (uint32_t)p.sd;
        }
        auto issue = [&](int buf, int kt) {
            const uint32_t to = smem_base + buf * kStage;
            const uint64_t k = (uint64_t)kt * 128;
#pragma unroll
            for (int i = 0; i < IW; ++i) load16_global_to_lds(gW + k, offW[i], to + (i * 8 + w) * 1024);
#pragma unroll
            for (int i = 0; i < IX; ++i) load16_global_to_lds(gX + k, offX[i], to + toX[i]);
            load4_global_to_lds(gS + (uint64_t)(kt >> 2) * 4, offS, to + kS + sid * 256);
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
            if constexpr (F8) {
                i32x8 xa[XB];
                uint32_t ex[XB];
#pragma unroll
                for (int i = 0; i < XB; ++i) {
                    const u32x4 a = tx[(rX + 16 * i) * 8 + ((2 * g4) ^ swX)], b = tx[(rX + 16 * i) * 8 + ((2 * g4 + 1) ^ swX)];
                    xa[i] = i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
                    ex[i] = sx[rX + 16 * i] >> sh;
                }
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const u32x4 a = tw[(rW + 16 * j) * 8 + ((2 * g4) ^ swW)], b = tw[(rW + 16 * j) * 8 + ((2 * g4 + 1) ^ swW)];
                    const i32x8 wa = i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
                    const uint32_t ew = sw[rW + 16 * j] >> sh;
#pragma unroll
                    for (int i = 0; i < XB; ++i)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, xa[i], acc[i][j], 0, 0, 0, (int)ew, 0, (int)ex[i]);
                }
            } else {
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
            }
            st = st + 1 == NS ? 0 : st + 1;
        }
        wait_global_loads_le<0>();   // the refills past the last k-step
        // the matrix instructions take w as their rows: a lane holds four consecutive outputs of one x row
        const int row = wx * XB * 16 + (lane & 15), col = wn * NB * 16 + g4 * 4;
        if (ka == 0 && kb == nk) {   // uniform: the whole tile
#pragma unroll
            for (int i = 0; i < XB; ++i)
                if (row + 16 * i <= x_last)
#pragma unroll
                    for (int j = 0; j < NB; ++j) store_outputs(p, x0 + row + 16 * i, w0 + col + 16 * j, acc[i][j]);
        } else {
            const int slot = (int)(range - tile * nk / p.len);   // how many ranges before this one touch the tile
            float *dst = p.part + ((tile * p.slots + slot) * BM + row) * BN + col;
#pragma unroll
            for (int i = 0; i < XB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) *reinterpret_cast<f32x4 *>(dst + i * 16 * BN + j * 16) = acc[i][j];
        }
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
};
const Variant kVariants[] = {
    {16, 128, 2, 1.2f, quant_gemm_kernel<1, 8, 1, 1, 4, false>},
    {32, 128, 2, 1.2f, quant_gemm_kernel<1, 8, 2, 1, 3, false>},
    {64, 128, 2, 1.3f, quant_gemm_kernel<1, 8, 4, 1, 3, false>},
    {128, 256, 1, 1.5f, quant_gemm_kernel<2, 4, 4, 4, 3, false>},
    {256, 256, 1, 2.2f, quant_gemm_kernel<4, 2, 4, 8, 2, false>},
    {256, 256, 1, 1.2f, quant_gemm_kernel<4, 2, 4, 8, 2, true>},
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
    pl.len = (double)whole * v.step_us <= (double)even * v.step_us + join_us ? whole : even;
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
    hipLaunchKernelGGL(v.kernel, dim3((unsigned)pl.wgs), dim3(512), 0, s, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || pl.part == 0) return e;
    const int64_t tiles = (int64_t)pl.x_tiles * pl.w_tiles;
    hipLaunchKernelGGL(quant_sum_kernel, dim3((unsigned)(tiles * (pl.bm * pl.bn / 1024))), dim3(256), 0, s, p, pl.bm, pl.bn);
    return hipGetLastError();
}

}  // namespace fz
