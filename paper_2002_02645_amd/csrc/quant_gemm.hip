// The dense layer on rows held in 8 bits (gfx950 / CDNA4):
//
//     y[r, c] = act(bias[c] + sum_B 2^(Ex[r, B] + Ew[c, B]) sum_{i in B} x8[r, i] w8[c, i])
//
// A k-step is a block of 128 codes: 128 bytes a row, copied as they are into LDS (direct loads) with the scale bytes of the four
// blocks it belongs to; both operands are laid out so that a stage is a run of memory (QuantRows).  Codes widen to bf16 in registers, their
// scale applied by the same instruction; bf16 matrix instructions, exact products (see widen) summed in fp32.  (The 8-bit matrix instructions have twice the
// rate, but cut the products of eight neighbours off 13 bits below the largest's exponent: up to 8e-5 of the result's norm, and where large terms
// cancel nothing is left of the small ones.  Not even a bf16 output is worth its bits then: 2.9 % of them were a step off at
// 4,096 x 2,048 -> 2,048.)
// Work: the flattened (tile, k-step) space in ranges, whole tiles where they fill the chip, else even ranges whose cut tiles
// leave their sums in slots, added in order by quant_sum_kernel.
#include "../../include/freeze.h"
#include "quantised.h"

#include <type_traits>
#include <utility>

namespace fz {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((address_space(3))) void *lds_void_ptr;

namespace {

// four codes of a word times 2^(exponent of s): four bf16, exact from 2^-126 on; below that to the nearest multiple of 2^-133, where codes of the
// lowest exponents reach 2^-135.  (The matrix instructions take such numbers as they are.)  256 * 2^120 is infinite.
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

// two bf16, to nearest even
__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// no number stays what it is
__device__ __forceinline__ float relu_of(float v) { return v <= 0.f ? 0.f : v; }

// outputs col .. col + 3 of a row
__device__ __forceinline__ void store_outputs(const QuantProduct &p, int64_t row, int64_t col, f32x4 v)
{
    if (col >= p.m) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (p.bias) v[e] += p.bias[col + e < p.m ? col + e : p.m - 1];
        if (p.relu) v[e] = relu_of(v[e]);
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

// What a workgroup forms: a tile, or the k-steps [ka, kb) of it.  Units are in order of (cut, group of four tiles of x rows, tile of w
// rows, x tile), and each XCD (block id modulo 8) takes a run of them: its workgroups are in the same k-steps at about the same time and
// share the rows of both operands in its L2.  (Ranges one after the other along a tile's depth shared nothing: 256 x 8,192 -> 8,192 55 us.)
constexpr int kTileGroup = 4;
struct Unit {
    int xt, wt, ka, kb;
    uint32_t slot;   // of the sums: tile * splits + cut
};
__device__ __forceinline__ void tile_place(const QuantProduct &p, uint32_t tile, int *xt, int *wt)
{
    const uint32_t group = tile / (uint32_t)(kTileGroup * p.w_tiles);
    const int first = (int)group * kTileGroup, wide = p.x_tiles - first < kTileGroup ? p.x_tiles - first : kTileGroup;
    const int r = (int)(tile - group * (uint32_t)(kTileGroup * p.w_tiles));
    *wt = r / wide;
    *xt = first + r - *wt * wide;
}
__device__ __forceinline__ Unit unit_of(const QuantProduct &p)
{
    const uint32_t n = gridDim.x, share = n >> 3, more = n & 7, xcd = blockIdx.x & 7, at = blockIdx.x >> 3;
    const uint32_t id = xcd * share + (xcd < more ? xcd : more) + at;   // the first `more` XCDs have one unit more
    const uint32_t tiles = (uint32_t)p.x_tiles * (uint32_t)p.w_tiles, cut = id / tiles, tile = id - cut * tiles;
    Unit u;
    tile_place(p, tile, &u.xt, &u.wt);
    u.ka = (int)((int64_t)p.nk * cut / p.splits);
    u.kb = (int)((int64_t)p.nk * (cut + 1) / p.splits);
    u.slot = tile * (uint32_t)p.splits + cut;
    return u;
}

// LDS-direct loads to a constant distance behind a wave's place (formed in M0 itself: as many places as a stage has loads, kept over
// the loop, would not fit the scalar registers).  Stages are runs of memory: a wave's load is 1 KiB at lane * 16, or 256 bytes at lane * 4.
template <int TO>
__device__ __forceinline__ void load16_to_lds_at(uint64_t sbase, uint32_t voff, uint32_t lds)
{
    asm volatile("s_add_u32 m0, %0, %3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(sbase), "n"(TO) : "memory", "m0", "scc");
}
// of memory that nobody else reads soon: not kept in L2
template <int TO>
__device__ __forceinline__ void load16_once_to_lds_at(uint64_t sbase, uint32_t voff, uint32_t lds)
{
    asm volatile("s_add_u32 m0, %0, %3\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(voff), "s"(sbase), "n"(TO) : "memory", "m0", "scc");
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

// A wave's sums: the matrix instructions take w as their rows, so a lane holds four consecutive outputs (from col on, and 16 j behind) of one
// x row (row, and 16 i behind).  Two blocks' bf16 outputs change places between a lane and the one 16 further, so that each has eight in a row.
template <int XB, int NB, int BM, int BN>
__device__ __forceinline__ void tile_out(const QuantProduct &p, const f32x4 (&acc)[XB][NB], const Unit &u, int row, int wave_col, int g4, int64_t x0,
                                         int64_t w0, int x_last)
{
    const int col = wave_col + 4 * g4;
    if (p.splits > 1) {   // uniform
        float *dst = p.part + ((int64_t)u.slot * BM + row) * BN + col;
        each(std::make_integer_sequence<int, XB * NB>{}, [&](auto ij) {
            constexpr int i = decltype(ij)::value / NB, j = decltype(ij)::value % NB;
            if (row + 16 * i <= x_last) *reinterpret_cast<f32x4 *>(dst + i * 16 * BN + j * 16) = acc[i][j];
        });
        return;
    }
    if (p.vec && w0 + wave_col + 16 * NB <= p.m) {   // uniform in the wave
        f32x4 bias[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) bias[j][e] = p.bias ? p.bias[w0 + col + 16 * j + e] : 0.f;
        each(std::make_integer_sequence<int, XB>{}, [&](auto i_) {
            constexpr int i = decltype(i_)::value;
            const int64_t to = (x0 + row + 16 * i) * p.out_stride + w0 + wave_col;
            const bool in = row + 16 * i <= x_last;
            f32x4 v[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                v[j] = acc[i][j] + bias[j];
                if (p.relu)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[j][e] = relu_of(v[j][e]);
            }
            if (!p.out_bf16) {
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    if (in) *reinterpret_cast<f32x4 *>(static_cast<float *>(p.out) + to + 4 * g4 + 16 * j) = v[j];
                return;
            }
            uint32_t h[NB][2];
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) h[j][e] = bf16_pair(v[j][2 * e], v[j][2 * e + 1]);
            uint16_t *out = static_cast<uint16_t *>(p.out) + to;
            if (p.vec > 1 && NB % 2 == 0) {
#pragma unroll
                for (int j = 0; j + 1 < NB; j += 2) {
                    u32x4 t;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const auto s = __builtin_amdgcn_permlane16_swap(h[j][e], h[j + 1][e], false, false);
                        t[e] = s[0];
                        t[2 + e] = s[1];
                    }
                    if (in) *reinterpret_cast<u32x4 *>(out + 16 * (j + (g4 & 1)) + 8 * (g4 >> 1)) = t;
                }
            } else {
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    if (in) *reinterpret_cast<u32x2 *>(out + 4 * g4 + 16 * j) = u32x2{h[j][0], h[j][1]};
            }
        });
    } else {
        each(std::make_integer_sequence<int, XB * NB>{}, [&](auto ij) {
            constexpr int i = decltype(ij)::value / NB, j = decltype(ij)::value % NB;
            if (row + 16 * i <= x_last) store_outputs(p, x0 + row + 16 * i, w0 + col + 16 * j, acc[i][j]);
        });
    }
}

// Batches of few rows: eight waves of XB x NB blocks of 16 x 16 outputs, WX of them along x; NS stages.  Bound by the memory that the
// weights come from: what counts is how many bytes are on their way.  Weights that one workgroup reads and that L2 cannot hold until the
// next call pass it by: 134 MB (1 x 4,096 -> 32,768) in 21.2 us against 25.5, 1.07 GB (32 x 8,192 -> 131,072) in 172.7 against 190.7,
// 6.2 - 6.9 TB/s.  Not so where tiles of x share them (300 rows of x: 25.1 us against 23.8), nor where L2 holds them: 16.8 MB 6.9 against 5.8.
// RAW: the few rows of x are quantised by every workgroup for itself, for the k-steps it takes, while its first weights are on their way; they stay
// in LDS as a whole.  As many as that holds: 1 x 4,096 -> 32,768 21.9 us a call, with a launch of its own for the row 24.3.
constexpr int kRawBytes = 14336;   // beside four stages, twice in a CU
constexpr int kRawSteps = kRawBytes / 129;   // k-steps of a row: 128 codes and a scale byte
template <int WX, int WN, int XB, int NB, int NS, bool RAW = false>
__global__ __launch_bounds__(kQuantThreads, 2) void quant_gemm_kernel(QuantProduct p)
{
    static_assert(!RAW || (WX == 1 && XB == 1), "one block of x rows");
    static_assert(WX * WN == 8, "eight waves");
    constexpr int BM = WX * XB * 16, BN = WN * NB * 16;
    constexpr int kX = BN * 128, kS = kX + (RAW ? 0 : BM * 128), kStage = kS + (BN + (RAW ? 0 : BM < 64 ? 64 : BM)) * 4;
    constexpr int IW = BN / 64, LX = BM / 8, IX = RAW ? 0 : (LX + 7) / 8;        // load instructions: of a wave, of all, of a wave
    constexpr int LS = BN / 64 + (RAW ? 0 : (BM + 63) / 64), NL = IW + IX + 1;
    static_assert(kQuantTile % BN == 0 && LS <= 8 && NS * kStage + (RAW ? kRawBytes : 0) <= 163840 && (NS - 2) * NL <= 63, "");
    __shared__ __attribute__((aligned(16))) unsigned char smem[NS * kStage + (RAW ? kRawBytes : 0)];

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wx = w / WN, wn = w % WN;
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_void_ptr)smem;
    const Unit u = unit_of(p);
    const int ka = u.ka, kb = u.kb;

    const int g4 = lane >> 4;
    const int rX = wx * XB * 16 + (lane & 15), rW = wn * NB * 16 + (lane & 15);   // + 16 i: leaves the swizzle as it is
    const int swX = row128_swizzle(rX), swW = row128_swizzle(rW);
    // the wave's loads (where there are fewer than waves, the last ones repeat one)
    const int lx = w < LX ? w : LX - 1, ls = w < LS ? w : LS - 1;
    const uint32_t off16 = lane * 16;
    // (of fewer rows than lanes the last row's scales are loaded again)
    const uint32_t off4 = (ls < BN / 64 || BM >= 64 || lane < BM ? lane : BM - 1) * 4;

    const int64_t x0 = (int64_t)u.xt * BM, w0 = (int64_t)u.wt * BN;
    const int x_last = (int)(p.b - x0 < BM ? p.b - x0 : BM) - 1;
    const int64_t wbig = w0 / kQuantTile * kQuantTile, win = w0 - wbig;   // the tile of the weights, the place within it
    const uint64_t gX = uniform_u64((uint64_t)(uintptr_t)(p.x + x0 * p.d_pad) + lx * 1024);
    const uint64_t gW = uniform_u64((uint64_t)(uintptr_t)(p.w + wbig * p.d_pad + win * 128) + w * 1024);
    const uint64_t gS = uniform_u64((uint64_t)(uintptr_t)(ls < BN / 64 ? p.ws + wbig * p.sd + win * 4 + ls * 256 : p.xs + x0 * p.sd + (ls - BN / 64) * 256));
    const int steps = kb - ka;
    const int rows = (int)(p.b < BM ? p.b : BM), own = rX < rows ? rX : rows - 1;   // RAW: one tile of x rows
    unsigned char *const held = smem + NS * kStage, *const held_scales = held + rows * steps * 128;
    const uint32_t s_rows = ls < BN / 64 ? kQuantTile * 4 : BM * 4;
    auto issue = [&](int buf, int kt) {
        const uint32_t to = smem_base + buf * kStage;
        const uint64_t kw = gW + (uint64_t)kt * (kQuantTile * 128), kx = gX + (uint64_t)kt * (BM * 128);
        each(std::make_integer_sequence<int, IW>{}, [&](auto i) {
            if (p.w_once) load16_once_to_lds_at<decltype(i)::value * 8192>(kw + decltype(i)::value * 8192, off16, to + w * 1024);   // uniform
            else load16_to_lds_at<decltype(i)::value * 8192>(kw + decltype(i)::value * 8192, off16, to + w * 1024);
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
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) issue(s, ka + s < klast ? ka + s : klast);
    if constexpr (RAW) {
        // sixteen values a thread, eight threads a block; chunk c of row r at c ^ (r & 7)
        const int per_row = steps * 8, n = rows * per_row;   // (a multiple of 8)
        for (int t = tid; t < n; t += 512) {
            const int r = t / per_row, chunk = t - r * per_row;
            const int64_t c = (int64_t)ka * 128 + chunk * 16;
            float v[16];
            if (c >= p.d) {
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = 0.f;
            } else if (p.raw_bf16) {   // uniform
                sixteen_of(static_cast<const uint16_t *>(p.raw) + r * p.raw_stride + c, v);
            } else {
                sixteen_of(static_cast<const float *>(p.raw) + r * p.raw_stride + c, v);
            }
            int ex;
            const u32x4 codes = codes_of(v, &ex);
            const int step = r * steps + (chunk >> 3);
            *reinterpret_cast<u32x4 *>(held + step * 128 + ((chunk & 7) ^ (r & 7)) * 16) = codes;
            if ((chunk & 7) == 0) held_scales[step] = (unsigned char)(ex + 127);
        }
    }
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
        for (int i = 0; i < XB; ++i)
            fx[i] = __uint_as_float((RAW ? (uint32_t)held_scales[own * steps + kt - ka] : sx[rX + 16 * i] >> sh & 255u) << 23);
        const u32x4 *const hx = reinterpret_cast<const u32x4 *>(held + (own * steps + kt - ka) * 128);
#pragma unroll
        for (int j = 0; j < NB; ++j) fw[j] = __uint_as_float((sw[rW + 16 * j] >> sh & 255u) << 23);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8 xa[2][XB];
#pragma unroll
            for (int i = 0; i < XB; ++i) {
                const u32x4 a = RAW ? hx[(2 * g4 + h) ^ (own & 7)] : tx[(rX + 16 * i) * 8 + ((2 * g4 + h) ^ swX)];
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
    tile_out<XB, NB, BM, BN>(p, acc, u, rX, wn * NB * 16, g4, x0, w0, x_last);
}

// Larger batches, which the matrix pipes bound: tiles of 32 XB x rows by 256 w rows, eight waves of 16 XB x 64 outputs, two stages.  A wave
// keeps its four blocks of w rows' fragments (16 rows each) for half a step (64 codes) and goes through its XB blocks of x rows, a group of
// matrix instructions each; their codes are read kAhead groups ahead.  The step's barrier comes
// before its last kAhead groups, which need nothing newer: it publishes the next step's stage and frees this one, which is refilled from there on.
// 10,000 x 8,192 -> 1,024 128 - 140 us by card, 1.2 - 1.3 PFLOP/s, the matrix pipes busy 55 % of all cycles; 4,096 x 8,192 -> 8,192 399 us, 1.38 PFLOP/s, 66 %.
template <int XB>
__global__ __launch_bounds__(kQuantThreads, 2) void quant_tile_kernel(QuantProduct p)
{
    constexpr int BM = 32 * XB, BN = 256, NB = 4;
    static_assert(BN == kQuantTile, "a stage of the weights is a run of memory");
    constexpr int kX = BN * 128, kS = kX + BM * 128, kStage = kS + (BN + (BM + 63) / 64 * 64) * 4;
    constexpr int kGroups = 2 * XB, kAhead = 3;
    constexpr int kRing = kGroups % 4 == 0 ? 4 : (kGroups % 5 == 0 ? 5 : 6);   // fragments ahead, in step with the groups
    constexpr int IW = BN / 64, LX = BM / 8, IX = (LX + 7) / 8, LS = BN / 64 + (BM + 63) / 64, NL = IW + IX + 1;   // load instructions: see above
    constexpr int kPerGroup = (NL + kAhead - 1) / kAhead;   // loads that each of the step's last groups issues
    static_assert(2 * kStage <= 163840 && kGroups % kRing == 0 && kRing > kAhead && LS <= 8, "");
    __shared__ __attribute__((aligned(16))) unsigned char smem[2 * kStage];

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wx = w >> 2, wn = w & 3;
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_void_ptr)smem;
    const Unit u = unit_of(p);
    const int ka = u.ka, kb = u.kb;

    const int g4 = lane >> 4;
    const int rX = wx * 16 * XB + (lane & 15), rW = wn * 64 + (lane & 15);   // + 16 i: leaves the swizzle as it is
    const int swX = row128_swizzle(rX), swW = row128_swizzle(rW);
    const uint32_t off16 = lane * 16;
    const int lx_last = (IX - 1) * 8 + w < LX ? (IX - 1) * 8 + w : LX - 1, ls = w < LS ? w : LS - 1;   // (surplus waves repeat a load)
    // (of fewer rows than lanes the last row's scales are loaded again)
    const int x_scales = BM - (ls - BN / 64) * 64;
    const uint32_t off4 = (ls < BN / 64 || lane < x_scales ? lane : x_scales - 1) * 4;
    const uint32_t lds16 = smem_base + w * 1024;

    const int64_t x0 = (int64_t)u.xt * BM, w0 = (int64_t)u.wt * BN;
    const int x_last = (int)(p.b - x0 < BM ? p.b - x0 : BM) - 1;
    const uint64_t gX = uniform_u64((uint64_t)(uintptr_t)(p.x + x0 * p.d_pad)), gW = uniform_u64((uint64_t)(uintptr_t)(p.w + w0 * p.d_pad) + w * 1024);
    const uint64_t gS = uniform_u64((uint64_t)(uintptr_t)(ls < BN / 64 ? p.ws + w0 * p.sd + ls * 256 : p.xs + x0 * p.sd + (ls - BN / 64) * 256));
    const uint32_t s_rows = ls < BN / 64 ? BN * 4 : BM * 4;
    // load l of k-step kt's stage
    auto issue = [&](int buf, int kt, auto l_) {
        constexpr int l = decltype(l_)::value;
        const uint32_t st = buf * kStage;
        if constexpr (l < IW) load16_to_lds_at<l * 8192>(gW + (uint64_t)kt * (BN * 128) + l * 8192, off16, lds16 + st);
        else if constexpr (l < IW + IX - 1) load16_to_lds_at<kX + (l - IW) * 8192>(gX + (uint64_t)kt * (BM * 128) + (l - IW) * 8192 + w * 1024, off16, lds16 + st);
        else if constexpr (l == IW + IX - 1) load16_to_lds_at<kX>(gX + (uint64_t)kt * (BM * 128) + lx_last * 1024, off16, smem_base + lx_last * 1024 + st);
        else if constexpr (l == NL - 1) load4_to_lds_at<kS>(gS + (uint64_t)(kt >> 2) * s_rows, off4, smem_base + ls * 256 + st);
    };

    f32x4 acc[XB][NB];
#pragma unroll
    for (int i = 0; i < XB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    u32x4 xr[kRing], wr[NB];   // codes yet to be widened: of x, ahead; of w
    uint32_t ex[kRing], ew[NB];   // with the scale bytes of their rows
    auto read = [&](u32x4 &to, const unsigned char *base, int row, int sw, int h) { to = (reinterpret_cast<const u32x4 *>(base) + row * 8)[(2 * g4 + h) ^ sw]; };
    auto read_x = [&](int set, int buf, int i, int h) {
        read(xr[set], smem + buf * kStage + kX, rX + 16 * i, swX, h);
        ex[set] = *reinterpret_cast<const uint32_t *>(smem + buf * kStage + kS + (BN + rX + 16 * i) * 4);
    };
    auto read_w = [&](int buf, int j, int h) { read(wr[j], smem + buf * kStage, rW + 16 * j, swW, h); };
    auto read_ws = [&](int buf, int j) { ew[j] = *reinterpret_cast<const uint32_t *>(smem + buf * kStage + kS + (rW + 16 * j) * 4); };

    const int klast = kb - 1;
    auto at_most = [&](int kt) { return kt < klast ? kt : klast; };
    each(std::make_integer_sequence<int, NL>{}, [&](auto l) { issue(0, ka, l); });
    each(std::make_integer_sequence<int, NL>{}, [&](auto l) { issue(1, at_most(ka + 1), l); });
    wait_global_loads_le<NL>();
    __syncthreads();
    each(std::make_integer_sequence<int, NB>{}, [&](auto j) {
        read_w(0, decltype(j)::value, 0);
        read_ws(0, decltype(j)::value);
    });
    each(std::make_integer_sequence<int, kAhead>{}, [&](auto i) { read_x(decltype(i)::value, 0, decltype(i)::value, 0); });
    // group g of a step: its barriers, the loads that they make room for, the reads of the group kAhead further
    auto group_head = [&](int kt, int st, auto g_) {
        constexpr int g = decltype(g_)::value, ahead = g + kAhead;
        if constexpr (g == kGroups - kAhead) {
            wait_global_loads_le<0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __syncthreads();
        }
        read_x(ahead % kRing, ahead < kGroups ? st : st ^ 1, ahead % XB, ahead / XB % 2);
        if constexpr (g >= kGroups - kAhead)
            each(std::make_integer_sequence<int, kPerGroup>{}, [&](auto l) {
                issue(st, at_most(kt + 2), std::integral_constant<int, (g - kGroups + kAhead) * kPerGroup + decltype(l)::value>{});
            });
    };
    int st = 0;
    // Codes are widened between the matrix instructions of the group before, a word or two behind each: one after the other, the two kinds
    // hardly overlap, not even those of a SIMD's two waves (measured: 8 matrix and 16 conversion instructions a wave 359 cycles in blocks,
    // 307 interleaved, 295 without the conversions).
    u32x4 wa[2][NB][2], xc[2][2];
    const auto word = [](u32x4 &to, int half, uint32_t codes, uint32_t e) {
        const u32x2 v = widen(codes, __uint_as_float(e));
        to[2 * half] = v[0];
        to[2 * half + 1] = v[1];
    };
    const auto scale = [](uint32_t e, int sh) { return (e >> sh & 255u) << 23; };
    each(std::make_integer_sequence<int, 4 * NB>{}, [&](auto t_) {
        constexpr int t = decltype(t_)::value;
        word(wa[0][t / 4][t % 4 / 2], t % 2, wr[t / 4][t % 4], scale(ew[t / 4], 8 * (ka & 3)));
    });
    each(std::make_integer_sequence<int, 4>{}, [&](auto t_) {
        constexpr int t = decltype(t_)::value;
        word(xc[0][t / 2], t % 2, xr[0][t], scale(ex[0], 8 * (ka & 3)));
    });
    for (int kt = ka; kt < kb; ++kt) {
        const int sh = 8 * (kt & 3), nsh = 8 * ((kt + 1) & 3);
        each(std::make_integer_sequence<int, kGroups>{}, [&](auto g_) {
            constexpr int g = decltype(g_)::value, h = g / XB, i = g % XB;
            group_head(kt, st, g_);
            // w blocks of the other half: of this step early in its first half, of the next one when its stage is there
            if constexpr (g < 2) {
                read_w(st, 2 * g, 1);
                read_w(st, 2 * g + 1, 1);
            } else if constexpr (g == kGroups - 3 || g == kGroups - 2) {
                constexpr int j = 2 * (g - kGroups + 3);
                read_w(st ^ 1, j, 0);
                read_ws(st ^ 1, j);
                read_w(st ^ 1, j + 1, 0);
                read_ws(st ^ 1, j + 1);
            }
            // ... and those of them that are widened in this group: the first half ends with one a group (of four groups, the last takes two)
            constexpr int late = XB == 4 ? 1 : XB - 4;
            constexpr int w_first = h == 0 ? i - late : 2 * (g - kGroups + 2);
            constexpr int w_count = h == 0 ? (i < late ? 0 : (XB == 4 && i == 3 ? 2 : 1)) : (g >= kGroups - 2 ? 2 : 0);
            constexpr int words = 4 + 4 * w_count;
            const uint32_t fx = scale(ex[(g + 1) % kRing], g + 1 < kGroups ? sh : nsh);
            uint32_t fw[2];
            each(std::make_integer_sequence<int, w_count>{}, [&](auto n) { fw[decltype(n)::value] = scale(ew[w_first + decltype(n)::value], h == 0 ? sh : nsh); });
            __builtin_amdgcn_sched_barrier(0);
            each(std::make_integer_sequence<int, 2 * NB>{}, [&](auto q_) {
                constexpr int q = decltype(q_)::value, j = q % NB, half = q / NB;
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wa[h][j][half]), __builtin_bit_cast(bf16x8, xc[g & 1][half]),
                                                                    acc[i][j], 0, 0, 0);
                each(std::make_integer_sequence<int, words>{}, [&](auto t_) {
                    constexpr int t = decltype(t_)::value;
                    if constexpr (t * 2 * NB / words == q) {
                        if constexpr (t < 4) {
                            word(xc[(g + 1) & 1][t / 2], t % 2, xr[(g + 1) % kRing][t], fx);
                        } else {
                            constexpr int n = t - 4, wj = w_first + n / 4;
                            word(wa[h ^ 1][wj][n % 4 / 2], n % 2, wr[wj][n % 4], fw[n / 4]);
                        }
                    }
                });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        st ^= 1;
    }
    wait_global_loads_le<0>();   // the refills past the last k-step
    tile_out<XB, NB, BM, BN>(p, acc, u, rX, wn * 64, g4, x0, w0, x_last);
}

// The outputs of cut tiles: the sums of a tile's cuts in order, 256 threads for 1,024 outputs.
__global__ __launch_bounds__(256) void quant_sum_kernel(QuantProduct p, int bm, int bn)
{
    const uint32_t per_tile = (uint32_t)(bm * bn) / 1024, tile = blockIdx.x / per_tile;
    int xt, wt;
    tile_place(p, tile, &xt, &wt);
    const int at = (int)(blockIdx.x - tile * per_tile) * 1024 + threadIdx.x * 4, row = at / bn, col = at % bn;
    if ((int64_t)xt * bm + row >= p.b || (int64_t)wt * bn + col >= p.m) return;
    const int64_t step = (int64_t)bm * bn;
    const float *src = p.part + (int64_t)tile * p.splits * step + at;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](int s, auto n_) {   // n cuts, all on their way at once, summed in pairs before they are added
        constexpr int n = decltype(n_)::value;
        f32x4 t[n];
#pragma unroll
        for (int e = 0; e < n; ++e) t[e] = s + e < p.splits ? *reinterpret_cast<const f32x4 *>(src + (s + e) * step) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 1; d < n; d <<= 1)
#pragma unroll
            for (int e = 0; e < n; e += 2 * d) t[e] += t[e + d];
        v += t[0];
    };
    int s = 0;
    for (; p.splits - s > 4; s += 16) add(s, std::integral_constant<int, 16>{});
    if (s < p.splits) add(s, std::integral_constant<int, 4>{});
    store_outputs(p, (int64_t)xt * bm + row, (int64_t)wt * bn + col, v);
}

// The kernels of kQuantVariants.
struct Variant {
    void (*kernel)(QuantProduct);
    void (*raw)(QuantProduct);   // the form that quantises its rows itself
};
const Variant kVariants[] = {
    {quant_gemm_kernel<1, 8, 1, 1, 4>, quant_gemm_kernel<1, 8, 1, 1, 4, true>},
    {quant_gemm_kernel<1, 8, 2, 1, 3>, nullptr},
    {quant_gemm_kernel<1, 8, 4, 1, 3>, nullptr},
    {quant_gemm_kernel<1, 8, 1, 2, 4>, quant_gemm_kernel<1, 8, 1, 2, 4, true>},
    {quant_gemm_kernel<1, 8, 2, 2, 4>, nullptr},
    {quant_gemm_kernel<1, 8, 4, 2, 3>, nullptr},
    {quant_tile_kernel<4>, nullptr},
    {quant_tile_kernel<5>, nullptr},
    {quant_tile_kernel<6>, nullptr},
    {quant_tile_kernel<8>, nullptr},
};
static_assert(sizeof kVariants / sizeof kVariants[0] == kQuantNumVariants, "a kernel for each");
}  // namespace

bool quant_takes_values(const QuantPlan &pl, const void *x, int dtype, int64_t b, int64_t d, int64_t row_stride)
{
    const int64_t size = dtype == FREEZE_F32 ? 4 : 2;
    return kVariants[pl.variant].raw && pl.x_tiles == 1 && b * ((pl.nk + pl.splits - 1) / pl.splits) <= kRawSteps && d % 16 == 0 &&
           reinterpret_cast<uintptr_t>(x) % 16 == 0 && row_stride * size % 16 == 0;
}

hipError_t launch_quant_product(const QuantPlan &pl, QuantProduct p, hipStream_t s)
{
    p.nk = pl.nk;
    p.x_tiles = pl.x_tiles;
    p.w_tiles = pl.w_tiles;
    p.splits = pl.splits;
    const int size = p.out_bf16 ? 2 : 4;
    p.vec = p.out_stride % 4 == 0 && reinterpret_cast<uintptr_t>(p.out) % (4 * size) == 0;
    if (p.vec && p.out_stride % 8 == 0 && reinterpret_cast<uintptr_t>(p.out) % 16 == 0) p.vec = 2;
    p.w_once = pl.x_tiles == 1 && p.m * p.d_pad > kL2Bytes;
    const Variant &v = kVariants[pl.variant];
    hipLaunchKernelGGL(p.raw ? v.raw : v.kernel, dim3((unsigned)pl.wgs), dim3(kQuantThreads), 0, s, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || pl.part == 0) return e;
    const int64_t tiles = (int64_t)pl.x_tiles * pl.w_tiles;   // (cut ones: a few rounds)
    hipLaunchKernelGGL(quant_sum_kernel, dim3((unsigned)(tiles * (pl.bm * pl.bn / 1024))), dim3(256), 0, s, p, pl.bm, pl.bn);
    return hipGetLastError();
}

}  // namespace fz
