// Attention over pages of 8 bits: one block of tokens against the columns of a wave, in registers.  Not part of the C ABI.
#pragma once
#include "pages.h"

namespace fz {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

struct AttendArgs {
    PageView v;
    const void *q;
    void *out;
    int64_t q_token, q_head, out_token, out_head;   // strides
    int64_t tokens, most, window;
    const int32_t *starts;
    int64_t least_cols, most_cols;                  // of a row that the kernel takes: others are another launch's
    int group, q_vec, out_bf16, out_vec;            // *_vec: 16-byte loads of q, 8-byte (bf16) or 16-byte stores of out
    float scale_log2;                               // the scale times log2(e): weights are powers of two
    // work split over the tokens
    int workers;
    int whole;                                      // no tile is split
    struct SplitTile *split;                        // [workers]: the tile that a worker has the first piece of and others go on with
    float *part_o, *part_ml;                        // [workers][2] pieces of tiles
};
struct SplitTile {
    int64_t first;                                  // of the row's new tokens
    int32_t columns;                                // of the row
    int32_t col0, head, pieces, slot;               // pieces 0: none; slot: of the first one, the others' are their workers' first
};

// What a row asks for: its new tokens, its length, the blocks that the first to the last of them see.
struct RowWork {
    NewTokens n;
    int len, lo, blocks, tiles;
};
__device__ __forceinline__ RowWork row_work(const AttendArgs &p, int row, int cols, int *floor)
{
    RowWork w;
    w.n = new_tokens(p.starts, row, p.tokens, p.most, floor);
    w.len = p.v.length_of(row);
    const int64_t seen = p.window > 0 ? (int64_t)w.len - w.n.count - p.window + 1 : 0;   // first place of the first token
    w.lo = seen > 0 ? (int)(seen / kPageBlock) : 0;
    w.blocks = w.n.count > 0 ? (w.len + kPageBlock - 1) / kPageBlock - w.lo : 0;
    w.blocks = w.blocks < 0 ? 0 : w.blocks;
    const int64_t own = (int64_t)w.n.count * p.group;
    w.tiles = own >= p.least_cols && own <= p.most_cols ? (int)((own + cols - 1) / cols) : 0;
    return w;
}

// What is the same in every lane, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)(((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32) | (uint32_t)uniform((int)x));
}
__device__ __forceinline__ RowWork uniform(const RowWork &w)
{
    return RowWork{{uniform(w.n.count), uniform(w.n.first)}, uniform(w.len), uniform(w.lo), uniform(w.blocks), uniform(w.tiles)};
}

__device__ __forceinline__ bf16x8 values_of(uint32_t a, uint32_t b, float scale)
{
    union {
        bf16x2 h[4];
        bf16x8 v;
    } u;
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
    return u.v;
}

// bytes 0x7f where a code is no number, 0 elsewhere (bit 7 alone)
__device__ __forceinline__ uint32_t no_numbers(uint32_t codes) { return ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// 1 where no_numbers() has a bit
__device__ __forceinline__ bf16x8 ones_where(uint32_t a, uint32_t b)
{
    union {
        uint32_t w[4];
        bf16x8 v;
    } u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t pair = __builtin_amdgcn_perm(0, e < 2 ? a : b, e & 1 ? 0x0c030c02u : 0x0c010c00u);   // two bytes to two halves
        u.w[e] = (pair >> 7) * 0x3f80u;
    }
    return u.v;
}

// x as NS numbers of 8 bits each
template <int NS>
__device__ __forceinline__ void parts_of(const float (&x)[8], bf16x8 (&out)[NS])
{
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            out[n][e] = (__bf16)r[e];
            if (n + 1 < NS) r[e] -= (float)out[n][e];
        }
}

// The running softmax of 16 * CT columns (a column: one head of one new token) in a wave.  A lane has column lane & 15 of each 16; weights and sums
// belong to the lane's own tokens, outputs are elements 32 c + 16 u + 4 (lane >> 4) + i of o[.][2 c + u].
__device__ __forceinline__ float largest(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));   // (fmaxf quiets its operands first)
    return r;
}
template <int CT>
__device__ __forceinline__ float largest_of(const f32x4 (&s)[CT][2], int ct)
{
    return largest(largest(s[ct][0][0], s[ct][0][1], s[ct][0][2]), largest(s[ct][0][3], s[ct][1][0], s[ct][1][1]), fmaxf(s[ct][1][2], s[ct][1][3]));
}
template <int DC, int CT>
struct Running {
    f32x4 o[CT][2 * DC];
    float m[CT], l[CT];   // m: the column's reference (no smaller than its largest score less kSlack), the same in its four lanes; l: the lane's own sum

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            m[t] = -INFINITY;
            l[t] = 0.f;
#pragma unroll
            for (int f = 0; f < 2 * DC; ++f) o[t][f] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
};
// Scores may pass the reference by this many powers of two before it follows: weights up to 2^8 cost no digit, and the reference
// (a reduction over four lanes, all outputs scaled) seldom moves.
constexpr float kSlack = 8.f;

// The queries of kCols columns from col0 on into LDS, [NS][kCols] rows of 32 DC + 8 bf16 (the 16 bytes more keep a wave's reads off each other's banks), zeros behind
// the last column and element.
template <int DC>
constexpr int kQueryRow = 32 * DC + 8;
template <int DC, int NS, int THREADS>
__device__ __forceinline__ void stage_queries(const AttendArgs &p, const RowWork &w, int head, int col0, int cols, uint16_t *to)
{
    const int there = w.n.count * p.group;
    for (int i = threadIdx.x; i < cols * (4 * DC); i += THREADS) {
        const int c = i / (4 * DC), d = i % (4 * DC) * 8, col = col0 + c;
        bf16x8 parts[NS];
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
        if (col < there) {
            const int token = col / p.group;
            const int64_t at = (w.n.first + token) * p.q_token + (head * p.group + col - token * p.group) * p.q_head + d;
            if (p.q_vec && d < p.v.head_dim) {
                if constexpr (NS == 1) {
                    const u32x4 u = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p.q) + at);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const f32x4 u = reinterpret_cast<const f32x4 *>(static_cast<const float *>(p.q) + at)[h];
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[4 * h + e] = u[e];
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (d + e < p.v.head_dim) {
                        if constexpr (NS == 1) x[e] = __uint_as_float((uint32_t)static_cast<const uint16_t *>(p.q)[at + e] << 16);
                        else x[e] = static_cast<const float *>(p.q)[at + e];
                    }
            }
        }
        parts_of<NS>(x, parts);
#pragma unroll
        for (int n = 0; n < NS; ++n) *reinterpret_cast<bf16x8 *>(to + (n * cols + c) * kQueryRow<DC> + d) = parts[n];
    }
}
// a lane's part of the 16 columns from c0 on
template <int DC, int NS>
__device__ __forceinline__ void take_queries(const uint16_t *from, int cols, int c0, bf16x8 (&q)[NS][DC])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
        for (int c = 0; c < DC; ++c) q[n][c] = *reinterpret_cast<const bf16x8 *>(from + (n * cols + c0 + (lane & 15)) * kQueryRow<DC> + 32 * c + 8 * (lane >> 4));
}

// Sums over the workgroup's threads before this one, of two numbers, and over all.  WAVES: of the workgroup.
constexpr int64_t kFalls = (int64_t)1 << 48;   // beside a sum below it: how many rows end before they begin
template <int WAVES>
struct TwoSums {
    int64_t before[2], all[2];
};
template <int WAVES>
__device__ __forceinline__ TwoSums<WAVES> two_sums(int64_t a, int64_t b, int64_t *lds /* [2 WAVES] */)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x = a, y = b;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t u = __shfl_up(x, o), w = __shfl_up(y, o);
        if (lane >= o) {
            x += u;
            y += w;
        }
    }
    if (lane == 63) {
        lds[wave] = x;
        lds[WAVES + wave] = y;
    }
    __syncthreads();
    TwoSums<WAVES> s{{x - a, y - b}, {0, 0}};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) {
            s.before[0] += lds[w];
            s.before[1] += lds[WAVES + w];
        }
        s.all[0] += lds[w];
        s.all[1] += lds[WAVES + w];
    }
    return s;
}

// The blocks of a row for one head, by their number in the row.
struct Blocks {
    const int32_t *table;
    const uint8_t *codes, *scales;          // of the head in page 0
    uint32_t page_bytes, page_scales;       // from page to page
    uint32_t block_bytes;
    int log2, mask, num_pages;
    __device__ __forceinline__ Blocks(const PageView &v, int row, int head)
        : table(v.tables + row * v.max_pages), codes(v.codes + v.block_at(0, head, 0)), scales(v.scales + v.scale_at(0, head, 0)),
          page_bytes((uint32_t)v.block_at(1, 0, 0)), page_scales((uint32_t)v.scale_at(1, 0, 0)), block_bytes(64 * v.width), log2(v.page_log2 - 5),
          mask(v.per_page - 1), num_pages(v.num_pages)
    {
    }
    __device__ __forceinline__ int page(int b) const { return table[b >> log2]; }   // (a load: uniform() of it a step later, not to wait for it here)
    __device__ __forceinline__ bool there(int page) const { return (unsigned)page < (unsigned)num_pages; }
    __device__ __forceinline__ const uint8_t *at(int page, int b) const
    {
        return codes + ((uint64_t)(uint32_t)page * page_bytes + (uint32_t)(b & mask) * block_bytes);
    }
    __device__ __forceinline__ uint32_t scale_bytes(int page, int b) const
    {
        return *reinterpret_cast<const uint16_t *>(scales + ((uint64_t)(uint32_t)page * page_scales + (uint32_t)(b & mask) * 2));
    }
};

// Scores of the block's 32 tokens: token 16 t + 4 (lane >> 4) + i against the lane's column.
template <int DC, int CT, int NS>
__device__ __forceinline__ void scores_of(const u32x4 (&k)[DC], const bf16x8 (&q)[CT][NS][DC], f32x4 (&s)[CT][2])
{
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) s[ct][0] = s[ct][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const bf16x8 f = values_of(k[c][2 * t], k[c][2 * t + 1], 1.f);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int n = 0; n < NS; ++n) s[ct][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[ct][n][c], s[ct][t], 0, 0, 0);
        }
}

// The factor of a block's scores, from its scale bytes: not below the smallest normal number, where scores are as good as 0, so that hidden ones stay -inf; nor infinite, so that
// scores of 0 stay 0.
__device__ __forceinline__ float score_factor(float scale_log2, uint32_t bytes)
{
    return __builtin_amdgcn_fmed3f(scale_log2 * __uint_as_float((bytes & 0xffu) << 23), 1.17549435e-38f, 3.40282347e38f);
}
__device__ __forceinline__ float value_factor(uint32_t bytes) { return __uint_as_float((bytes >> 8) << 23); }

// What a lane's columns see: the places behind `before` up to `place` (below 0: a column of nobody).
template <int CT>
struct Sight {
    int place[CT], before[CT];
    __device__ __forceinline__ void set(int ct, int at, int64_t window)
    {
        place[ct] = at;
        before[ct] = window > 0 ? (int)(at - window) : -1;   // (a window has less than 2^31 places)
    }
    // the token of weight e (0 .. 7: scores [e / 4][e % 4]) of the block that begins with `first`
    __device__ __forceinline__ bool sees(int ct, int first, int e) const
    {
        const int token = first + 16 * (e >> 2) + 4 * ((threadIdx.x & 63) >> 4) + (e & 3);
        return token <= place[ct] && token > before[ct];
    }
};
template <int CT>
__device__ __forceinline__ void hide(f32x4 (&s)[CT][2], int first, const Sight<CT> &sight)
{
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (!sight.sees(ct, first, e)) s[ct][e >> 2][e & 3] = -INFINITY;
            __builtin_amdgcn_sched_barrier(0);   // (one at a time: their masks together would push the loop's own scalars out of their registers)
        }
}

// Codes that are no number, in a block that some columns do not see all of (or that nobody wrote all of): they are taken out of the values, and the
// outputs of the columns that see them become NaN.
template <int DC, int CT>
__device__ __forceinline__ void take_out_strange(f32x4 (&o)[CT][2 * DC], u32x4 (&v)[DC], int first, const Sight<CT> &sight)
{
    uint32_t any = 0;
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) any |= no_numbers(v[c][e]);
    if (!__any(any != 0)) return;
    bf16x8 seen[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            seen[ct][e] = sight.sees(ct, first, e) ? (__bf16)1.f : (__bf16)0.f;
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t a = no_numbers(v[c][2 * u]), b = no_numbers(v[c][2 * u + 1]);
            v[c][2 * u] &= ~((a >> 7) * 0xffu);
            v[c][2 * u + 1] &= ~((b >> 7) * 0xffu);
            const bf16x8 bad = ones_where(a, b);
            __builtin_amdgcn_sched_barrier(0);   // (one at a time: seldom run, and not to cost the others registers)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const f32x4 count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, seen[ct], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (count[i] > 0.f) o[ct][2 * c + u][i] = __uint_as_float(0x7fc00000u);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
}

// Scores to weights.  first: the block's first token, edge: some column does not see all of the block.
template <int DC, int CT>
__device__ __forceinline__ void weigh(Running<DC, CT> &r, f32x4 (&s)[CT][2], float scale, bool edge, int first, const Sight<CT> &sight)
{
    if (edge) hide<CT>(s, first, sight);
    float top[CT];
    bool follow = false;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        top[ct] = largest_of(s, ct) * scale;
        follow |= top[ct] > r.m[ct] + kSlack;
    }
    if (__any(follow)) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            float m = fmaxf(top[ct], __shfl_xor(top[ct], 16));
            m = fmaxf(r.m[ct], fmaxf(m, __shfl_xor(m, 32)));
            const float a = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(r.m[ct] - m);
            r.m[ct] = m;
            r.l[ct] *= a;
#pragma unroll
            for (int f = 0; f < 2 * DC; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) r.o[ct][f][i] *= a;
        }
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const float m = r.m[ct] == -INFINITY ? 0.f : r.m[ct];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[ct][t][i] = __builtin_amdgcn_exp2f(fmaf(s[ct][t][i], scale, -m));
                r.l[ct] += s[ct][t][i];
            }
    }
}

// Weights times values, the weights in NP parts.
template <int DC, int CT, int NP>
__device__ __forceinline__ void add_values(Running<DC, CT> &r, u32x4 (&v)[DC], float scale, const f32x4 (&w)[CT][2], bool edge, int first,
                                           const Sight<CT> &sight)
{
    bf16x8 f[CT][NP];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const float x[8] = {w[ct][0][0], w[ct][0][1], w[ct][0][2], w[ct][0][3], w[ct][1][0], w[ct][1][1], w[ct][1][2], w[ct][1][3]};
        parts_of<NP>(x, f[ct]);
    }
    if (edge) take_out_strange<DC, CT>(r.o, v, first, sight);
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bf16x8 x = values_of(v[c][2 * u], v[c][2 * u + 1], scale);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int n = 0; n < NP; ++n) r.o[ct][2 * c + u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, f[ct][n], r.o[ct][2 * c + u], 0, 0, 0);
        }
}

// Four elements of a column's output, from element d on.
__device__ __forceinline__ void store_out(const AttendArgs &p, int64_t first, int head, int col, int d, f32x4 x)
{
    if (d >= p.v.head_dim) return;
    const int token = col / p.group;
    const int64_t at = (first + token) * p.out_token + (head * p.group + col - token * p.group) * p.out_head + d;
    if (p.out_bf16) {
        uint16_t *to = static_cast<uint16_t *>(p.out) + at;
        if (p.out_vec) {
            union {
                bf16x2 h[2];
                u32x2 w;
            } u;
            u.h[0] = bf16x2{(__bf16)x[0], (__bf16)x[1]};
            u.h[1] = bf16x2{(__bf16)x[2], (__bf16)x[3]};
            *reinterpret_cast<u32x2 *>(to) = u.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (d + i < p.v.head_dim) to[i] = bf16_rne(x[i]);
        }
    } else {
        float *to = static_cast<float *>(p.out) + at;
        if (p.out_vec) *reinterpret_cast<f32x4 *>(to) = x;
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (d + i < p.v.head_dim) to[i] = x[i];
        }
    }
}

}  // namespace fz
