// Attention over pages of keys and values in 8 bits (gfx950 / CDNA4).
//
// A block of 32 tokens of a head lies in memory as the matrix instructions want it: scores are (keys x queries), 16 tokens x 32 elements x 16 columns
// a time, whose results are, lane for lane, the right operand of (values^T x weights).  Nothing goes through LDS and no
// lane needs another's weights; e4m3 codes become bf16 exactly, two an instruction, the values' power of two with them.
#include "pages_attend.h"

namespace fz {

namespace {

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

constexpr int kWorkers = 512;         // workgroups that share the work
constexpr int64_t kLeastShare = 4;    // blocks of a workgroup: one a wave

__host__ __device__ inline int64_t share_of(int64_t blocks, int workers)
{
    const int64_t share = (blocks + workers - 1) / workers;
    return share < kLeastShare ? kLeastShare : share;
}

// Rows of a few columns each (a token or some of a row): all blocks of all (row, tile of columns, head) lie in one line, which is
// cut into equal shares, one a workgroup, wherever that falls; a tile that several workgroups meet in goes through `part` and pages_join_kernel.  A share's
// blocks go round the workgroup's four waves, whose results meet in LDS at the tile's end.
template <int DC, int CT, int NS>
__global__ __launch_bounds__(256) void pages_attend_kernel(AttendArgs p)
{
    constexpr int kCols = 16 * CT, kFrags = CT * 2 * DC;
    extern __shared__ float lds[];
    const PageView &v = p.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15;

    // where this workgroup's share begins
    int64_t *sums = reinterpret_cast<int64_t *>(lds);
    const int per = (v.rows + 255) / 256;
    const int r0 = min(v.rows, (int)threadIdx.x * per), r1 = min(v.rows, r0 + per);
    int64_t mine = 0, tiles = 0;
    for (int r = r0; r < r1; ++r) {
        const RowWork w = row_work(p, r, kCols);
        mine += (int64_t)w.blocks * w.tiles;
        tiles += w.tiles;
    }
    sums[threadIdx.x] = mine;
    sums[256 + threadIdx.x] = tiles;
    __syncthreads();
    int64_t before = 0, total = 0, tiles_before = 0;
    for (int t = 0; t < 256; ++t) {
        if (t < (int)threadIdx.x) {
            before += sums[t];
            tiles_before += sums[256 + t];
        }
        total += sums[t];
    }
    if (blockIdx.x == 0) {   // for pages_join_kernel
        int64_t b = before, n = tiles_before;
        for (int r = r0; r < r1; ++r) {
            p.blocks_before[r] = b;
            p.tiles_before[r] = (int32_t)n;
            const RowWork w = row_work(p, r, kCols);
            b += (int64_t)w.blocks * w.tiles;
            n += w.tiles;
            if (r + 1 == v.rows) {
                p.blocks_before[v.rows] = b;
                p.tiles_before[v.rows] = (int32_t)n;
            }
        }
    }
    const int64_t share = share_of(total * v.heads, p.workers);
    const int64_t begin = blockIdx.x * share, end = min(total * v.heads, begin + share);
    if (begin >= end) return;
    int *found = reinterpret_cast<int *>(sums + 512);
    int64_t *found_before = sums + 513;
    if (before * v.heads <= begin && begin < (before + mine) * v.heads) {
        int64_t b = before;
        int r = r0;
        for (; r < r1; ++r) {
            const RowWork w = row_work(p, r, kCols);
            const int64_t n = (int64_t)w.blocks * w.tiles;
            if (begin < (b + n) * v.heads) break;
            b += n;
        }
        *found = r;
        *found_before = b;
    }
    __syncthreads();
    int row = __builtin_amdgcn_readfirstlane(*found);
    int64_t base = *found_before * v.heads;
    __syncthreads();

    for (int64_t at = begin; at < end;) {
        const RowWork w = row_work(p, row, kCols);
        const int64_t row_blocks = (int64_t)w.blocks * w.tiles * v.heads;
        if (at >= base + row_blocks) {
            base += row_blocks;
            ++row;
            continue;
        }
        const int64_t item = (at - base) / w.blocks;
        const int b0 = (int)(at - base - item * w.blocks), tile = (int)(item / v.heads), head = (int)(item - (int64_t)tile * v.heads);
        const int count = (int)min((int64_t)w.blocks - b0, end - at);
        const int64_t col0 = (int64_t)tile * kCols;

        bf16x8 q[CT][NS][DC];
        int place[CT];
        int lowest = INT32_MAX, highest = -1;   // places of the tile's tokens
        const int64_t cols = (int64_t)w.n.count * p.group;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const int64_t c = col0 + 16 * ct + col;
            load_queries<DC, NS>(p, w, head, c, q[ct]);
            place[ct] = c < cols ? w.len - w.n.count + (int)(c / p.group) : -1;
        }
        lowest = w.len - w.n.count + (int)(col0 / p.group);
        highest = w.len - w.n.count + (int)((min(cols, col0 + kCols) - 1) / p.group);

        Running<DC, CT> run;
        run.clear();
        const int32_t *table = v.tables + row * v.max_pages;
        const int block0 = w.lo + b0;
        auto page_of = [&](int i) { return table[(block0 + i) >> (v.page_log2 - 5)]; };
        u32x4 k[DC], x[DC];
        uint32_t scales = 0;
        auto base_of = [&](int page, int i) { return v.codes + v.block_at(page, head, (block0 + i) & (v.per_page - 1)) + lane * 16; };
        auto load_keys = [&](int page, int i) {
            const uint8_t *from = base_of(page, i);
#pragma unroll
            for (int c = 0; c < DC; ++c) k[c] = *reinterpret_cast<const u32x4 *>(from + c * 1024);
        };
        auto load_values = [&](int page, int i) {
            const uint8_t *from = base_of(page, i) + 32 * v.width;
#pragma unroll
            for (int c = 0; c < DC; ++c) x[c] = *reinterpret_cast<const u32x4 *>(from + c * 1024);
        };
        auto load_scales = [&](int page, int i) { return (uint32_t)*reinterpret_cast<const uint16_t *>(v.scales + v.scale_at(page, head, (block0 + i) & (v.per_page - 1))); };
        auto there = [&](int page) { return page >= 0 && page < v.num_pages; };

        int i = wave;
        int page = i < count ? page_of(i) : -1, next = i + 4 < count ? page_of(i + 4) : -1;
        if (there(page)) {
            load_keys(page, i);
            scales = load_scales(page, i);
            load_values(page, i);
        }
        for (; i < count; i += 4) {
            const int after = i + 8 < count ? page_of(i + 8) : -1;
            f32x4 s[CT][2];
            const bool here = there(page), more = there(next);
            const int first = (block0 + i) * kPageBlock;
            const bool edge = first + kPageBlock - 1 > lowest || (p.window > 0 && (int64_t)first <= highest - p.window);
            const float ks = p.scale_log2 * __uint_as_float((scales & 0xffu) << 23), vs = __uint_as_float((scales >> 8) << 23);
            if (here) scores_of<DC, CT, NS>(k, q, s);
            if (more) {
                load_keys(next, i + 4);
                scales = load_scales(next, i + 4);
            }
            if (here) {
                weigh<DC, CT>(run, s, ks, edge, first, place, p.window);
                add_values<DC, CT, NS>(run, x, vs, s, edge, first, place, p.window);
            }
            if (more) load_values(next, i + 4);
            page = next;
            next = after;
        }

        // the four waves' results into the first one's
        float *ml = lds;   // [4][2][kCols]
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            float l = run.l[ct];
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            run.l[ct] = l;
            if (lane < 16) {
                ml[(wave * 2) * kCols + 16 * ct + lane] = run.m[ct];
                ml[(wave * 2 + 1) * kCols + 16 * ct + lane] = l;
            }
        }
        __syncthreads();
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u) m = fmaxf(m, ml[u * 2 * kCols + 16 * ct + col]);
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int u = 0; u < 4; ++u) l += ml[(u * 2 + 1) * kCols + 16 * ct + col] * __builtin_amdgcn_exp2f(ml[u * 2 * kCols + 16 * ct + col] - ref);
            const float a = __builtin_amdgcn_exp2f(run.m[ct] - ref);
            run.m[ct] = m;
            run.l[ct] = l;
#pragma unroll
            for (int f = 0; f < 2 * DC; ++f)
#pragma unroll
                for (int e = 0; e < 4; ++e) run.o[ct][f][e] *= a;
        }
        __syncthreads();
        f32x4 *frags = reinterpret_cast<f32x4 *>(lds);   // [2][kFrags][64]
#pragma unroll
        for (int half = 2; half > 0; half >>= 1) {
            if (wave >= half && wave < 2 * half)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int f = 0; f < 2 * DC; ++f) frags[((wave - half) * kFrags + ct * 2 * DC + f) * 64 + lane] = run.o[ct][f];
            __syncthreads();
            if (wave < half)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int f = 0; f < 2 * DC; ++f) {
                        const f32x4 o = frags[(wave * kFrags + ct * 2 * DC + f) * 64 + lane];
#pragma unroll
                        for (int e = 0; e < 4; ++e) run.o[ct][f][e] += o[e];
                    }
            __syncthreads();
        }
        if (wave == 0) {
            const bool whole = b0 == 0 && count == w.blocks;
            const int64_t slot = blockIdx.x * 2 + (at == begin ? 0 : 1);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const int64_t c = col0 + 16 * ct + col;
                if (c >= cols) continue;
                const float inv = run.l[ct] == 0.f ? 0.f : 1.f / run.l[ct];
                if (!whole && lane < 16) {
                    p.part_ml[(slot * 2) * kCols + 16 * ct + col] = run.m[ct];
                    p.part_ml[(slot * 2 + 1) * kCols + 16 * ct + col] = run.l[ct];
                }
#pragma unroll
                for (int f = 0; f < 2 * DC; ++f) {
                    f32x4 o = run.o[ct][f];
                    if (!whole) {
                        reinterpret_cast<f32x4 *>(p.part_o)[(slot * kFrags + ct * 2 * DC + f) * 64 + lane] = o;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] *= inv;
                        store_out(p, w.n.first, head, c, 16 * f + 4 * (lane >> 4), o);
                    }
                }
            }
        }
        at += count;
    }
}

// A tile that several workgroups had a piece of: their sums under one reference.  Tiles of nobody's blocks get their zeros.
template <int DC, int CT>
__global__ __launch_bounds__(256) void pages_join_kernel(AttendArgs p)
{
    constexpr int kCols = 16 * CT, kFrags = CT * 2 * DC;
    const PageView &v = p.v;
    const int tile = blockIdx.x / v.heads, head = blockIdx.x - tile * v.heads;
    if (tile >= p.tiles_before[v.rows]) return;
    int row = 0;
    for (int step = 1 << 14; step > 0; step >>= 1)
        if (row + step < v.rows && p.tiles_before[row + step] <= tile) row += step;
    const RowWork w = row_work(p, row, kCols);
    const int in_row = tile - p.tiles_before[row];
    const int64_t share = share_of(p.blocks_before[v.rows] * v.heads, p.workers);
    const int64_t begin = p.blocks_before[row] * v.heads + ((int64_t)in_row * v.heads + head) * w.blocks;
    const int64_t w0 = begin / share, w1 = (begin + w.blocks - 1) / share;
    const int e = blockIdx.y * 256 + threadIdx.x;   // a fragment of a lane
    const int lane = e & 63, frag = e >> 6;
    if (frag >= kFrags || (w.blocks > 0 && w0 == w1)) return;
    const int ct = frag / (2 * DC), in = 16 * ct + (lane & 15);
    const int64_t c = (int64_t)in_row * kCols + in;
    if (c >= (int64_t)w.n.count * p.group) return;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    if (w.blocks > 0) {
        auto slot_of = [&](int64_t u) { return u * 2 + (u == w0 && begin != u * share ? 1 : 0); };
        float m = -INFINITY, l = 0.f;
        for (int64_t u = w0; u <= w1; ++u) m = fmaxf(m, p.part_ml[slot_of(u) * 2 * kCols + in]);
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll 4
        for (int64_t u = w0; u <= w1; ++u) {
            const int64_t slot = slot_of(u);
            const float a = __builtin_amdgcn_exp2f(p.part_ml[slot * 2 * kCols + in] - ref);
            l += a * p.part_ml[(slot * 2 + 1) * kCols + in];
            const f32x4 x = reinterpret_cast<const f32x4 *>(p.part_o)[(slot * kFrags + frag) * 64 + lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] += a * x[i];
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= inv;
    }
    store_out(p, w.n.first, head, c, 16 * (frag - ct * 2 * DC) + 4 * (lane >> 4), o);
}

// ---- host -------------------------------------------------------------------------------------------

struct AttendPlan {
    int ct, parts;
    size_t o_bytes, ml_bytes, rows_bytes;
    size_t bytes() const { return o_bytes + ml_bytes + 2 * rows_bytes; }
};
AttendPlan attend_plan(const freeze_pages *p, int group, int64_t most, int parts)
{
    AttendPlan pl;
    const int dc = page_width(p->head_dim) / 32;
    const int64_t cols = (most > 0 ? most : 1) * group;
    pl.parts = parts;
    pl.ct = parts > 1 || cols <= 16 ? 1 : cols <= 32 || dc > 4 ? 2 : 4;
    const size_t slots = 2 * kWorkers, kCols = 16 * pl.ct;
    pl.o_bytes = slots * kCols * page_width(p->head_dim) * 4;
    pl.ml_bytes = slots * 2 * kCols * 4;
    pl.rows_bytes = up256(((size_t)p->rows + 1) * 8);
    return pl;
}

template <int DC, int CT, int NS>
hipError_t launch_attend(const AttendArgs &a, int64_t tiles, hipStream_t s)
{
    constexpr int kFrags = CT * 2 * DC;
    constexpr size_t lds = std::max<size_t>({2 * (size_t)kFrags * 1024, 8 * 16 * CT * 4, 515 * 8});
    hipLaunchKernelGGL((pages_attend_kernel<DC, CT, NS>), dim3(a.workers), dim3(256), lds, s, a);
    if (hipGetLastError() != hipSuccess) return hipErrorLaunchFailure;
    hipLaunchKernelGGL((pages_join_kernel<DC, CT>), dim3((unsigned)(tiles * a.v.heads), (kFrags * 64 + 255) / 256), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <int DC>
hipError_t launch_width(const AttendArgs &a, const AttendPlan &pl, int64_t tiles, hipStream_t s)
{
    if (pl.parts > 1) return launch_attend<DC, 1, 3>(a, tiles, s);
    if (pl.ct == 1) return launch_attend<DC, 1, 1>(a, tiles, s);
    if (pl.ct == 2) return launch_attend<DC, 2, 1>(a, tiles, s);
    if constexpr (DC <= 4) return launch_attend<DC, 4, 1>(a, tiles, s);
    return hipErrorInvalidValue;
}

bool attend_sizes(const freeze_pages *p, int group, int64_t tokens, int64_t most)
{
    return page_sizes(p) && group >= 1 && group <= 1024 && tokens >= 0 && tokens < (int64_t)1 << 31 && most >= 0 &&
           ((double)tokens * group + 16.0 * (double)p->rows) * p->heads < 268435456.0;   // a grid of 256 threads for each 16 columns
}
int64_t most_of(int64_t tokens, int64_t most, bool packed) { return !packed ? 1 : most > 0 && most < tokens ? most : tokens; }

}  // namespace
}  // namespace fz

using namespace fz;

extern "C" {

size_t freeze_pages_attend_workspace_bytes(const freeze_pages *pages, int group, int64_t tokens, int64_t most, int packed)
{
    if (!attend_sizes(pages, group, tokens, most)) return 0;
    const AttendPlan pl = attend_plan(pages, group, most_of(tokens, most, packed), 1);
    return pl.bytes();
}

int freeze_pages_attend(const freeze_pages *pages, int layer, const void *q, int q_dtype, int64_t q_token_stride, int64_t q_head_stride, int group,
                        int64_t tokens, const int32_t *starts, int64_t most, float scale, int64_t window, void *out, int out_dtype,
                        int64_t out_token_stride, int64_t out_head_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!attend_sizes(pages, group, tokens, most) || layer < 0 || layer >= pages->layers || (q_dtype != FREEZE_F32 && q_dtype != FREEZE_BF16) ||
        (out_dtype != FREEZE_F32 && out_dtype != FREEZE_BF16) || !(scale > 0.f && scale < 3.0e38f) || window < 0 || window >= (int64_t)1 << 31 ||
        (!starts && tokens != 0 && tokens != pages->rows))
        return FREEZE_EINVAL;
    if (tokens == 0) return FREEZE_OK;
    const uintptr_t qs = q_dtype == FREEZE_F32 ? 4 : 2, os = out_dtype == FREEZE_F32 ? 4 : 2;
    const uintptr_t qb = reinterpret_cast<uintptr_t>(q), ob = reinterpret_cast<uintptr_t>(out), wb = reinterpret_cast<uintptr_t>(workspace);
    const int64_t heads = (int64_t)pages->heads * group;
    int64_t q_span, out_span;
    if (!q || !out || !workspace || qb % qs != 0 || ob % os != 0 || reinterpret_cast<uintptr_t>(starts) % 4 != 0 ||
        !heads_span(tokens, heads, pages->head_dim, q_token_stride, q_head_stride, false, &q_span) ||
        !heads_span(tokens, heads, pages->head_dim, out_token_stride, out_head_stride, true, &out_span))
        return FREEZE_EINVAL;
    const int64_t each = most_of(tokens, most, starts != nullptr);
    const AttendPlan pl = attend_plan(pages, group, each, q_dtype == FREEZE_F32 ? 3 : 1);
    if (workspace_bytes < freeze_pages_attend_workspace_bytes(pages, group, tokens, most, starts != nullptr) || wb % 256 != 0) return FREEZE_EWORKSPACE;
    Extent e[10];
    int n = 0;
    if (!page_extents(pages, 0, e, &n)) return FREEZE_EINVAL;
    auto add_extent = [&](uintptr_t b, size_t bytes, bool dst) {
        if (b) e[n++] = Extent{b, b + bytes, dst};
    };
    add_extent(qb, (size_t)q_span * qs, false);
    add_extent(ob, (size_t)out_span * os, true);
    add_extent(wb, pl.bytes(), true);
    add_extent(reinterpret_cast<uintptr_t>(starts), ((size_t)pages->rows + 1) * 4, false);
    if (written_twice(e, n)) return FREEZE_EINVAL;
    AttendArgs a{};
    a.v = page_view(pages, layer);
    a.q = q;
    a.out = out;
    a.q_token = tokens > 1 ? q_token_stride : 0;
    a.q_head = heads > 1 ? q_head_stride : 0;
    a.out_token = tokens > 1 ? out_token_stride : 0;
    a.out_head = heads > 1 ? out_head_stride : 0;
    a.tokens = tokens;
    a.most = each;
    a.window = window;
    a.starts = starts;
    a.group = group;
    a.q_vec = q_dtype == FREEZE_BF16 && qb % 16 == 0 && pages->head_dim % 8 == 0 && a.q_token % 8 == 0 && a.q_head % 8 == 0;
    a.out_bf16 = out_dtype == FREEZE_BF16;
    a.out_vec = ob % (4 * os) == 0 && pages->head_dim % 4 == 0 && a.out_token % 4 == 0 && a.out_head % 4 == 0;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.workers = kWorkers;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    a.blocks_before = reinterpret_cast<int64_t *>(ws);
    ws += pl.rows_bytes;
    a.tiles_before = reinterpret_cast<int32_t *>(ws);
    ws += pl.rows_bytes;
    a.part_ml = reinterpret_cast<float *>(ws);
    ws += pl.ml_bytes;
    a.part_o = reinterpret_cast<float *>(ws);
    const int64_t cols = 16 * pl.ct;
    const int64_t tiles = std::min(tokens * group / cols + pages->rows, tokens * ((group + cols - 1) / cols));
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t err = hipErrorInvalidValue;
    switch (a.v.width / 32) {
        case 1: err = launch_width<1>(a, pl, tiles, s); break;
        case 2: err = launch_width<2>(a, pl, tiles, s); break;
        case 3: err = launch_width<3>(a, pl, tiles, s); break;
        case 4: err = launch_width<4>(a, pl, tiles, s); break;
        case 5: err = launch_width<5>(a, pl, tiles, s); break;
        case 6: err = launch_width<6>(a, pl, tiles, s); break;
        case 7: err = launch_width<7>(a, pl, tiles, s); break;
        case 8: err = launch_width<8>(a, pl, tiles, s); break;
    }
    return err == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

}  // extern "C"
