// Pages of keys and values (gfx950 / CDNA4): the bookkeeping of a pool whose pages several rows share, and the appending of new tokens.
#include "pages.h"

namespace fz {

namespace {

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

constexpr int kBookThreads = 1024;

// exclusive sum over a workgroup's threads in their order; *total: over all of them
__device__ __forceinline__ int64_t exclusive_sum(int64_t v, int64_t *total)
{
    __shared__ int64_t wave_sum[kBookThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t u = __shfl_up(s, o);
        if (lane >= o) s += u;
    }
    __syncthreads();   // (the last call's sums are read)
    if (lane == 63) wave_sum[wave] = s;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
        if (w < wave) before += wave_sum[w];
        all += wave_sum[w];
    }
    *total = all;
    return before + s - v;
}

struct PageCopy {
    int32_t src, dst, row, blocks;   // blocks: the filled ones
};
struct PageFill {
    int32_t row, place, from, count; // places of a row's table, entries of the list of free pages
};

struct ReserveArgs {
    PageView v;
    const int32_t *add;
    int32_t *granted;
    int32_t *need;       // [rows] scratch: pages wanted, the sign bit: one of them for a copy, kDenied: no place in the table
    int32_t *free;       // [num_pages] scratch
    PageCopy *copies;    // [rows] scratch
    PageFill *fills;     // [rows] scratch
    int32_t *num_copies; // scratch
};
constexpr int32_t kDenied = 0x7fffffff;

// One workgroup: which pages a row gets follows from all rows before it.  A sum over the rows' wants, then the free pages in order until there are as many, then a
// wave for each row that gets several.  Bound by the latency of its dependent steps: 32 rows, 330 pages
// 7.5 us; 24 rows of up to 4,096 tokens 7.8 (16 where each row's own thread filled its table); 64 rows of one token 6.3.
__global__ __launch_bounds__(kBookThreads) void pages_reserve_kernel(ReserveArgs p)
{
    const PageView &v = p.v;
    const int per = (v.rows + kBookThreads - 1) / kBookThreads;
    const int r0 = min(v.rows, (int)threadIdx.x * per), r1 = min(v.rows, r0 + per);
    const int64_t page_mask = ((int64_t)1 << v.page_log2) - 1;
    constexpr int kEach = 16;
    auto free_from = [&](int64_t first) {   // which of kEach pages are free
        uint32_t is_free = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (first + e < v.num_pages && v.refs[first + e] == 0) is_free |= 1u << e;
        return is_free;
    };
    uint32_t is_free = free_from((int64_t)threadIdx.x * kEach);   // (on its way while the rows are looked at)
    int64_t mine = 0;
    int32_t only = 0;   // of the one row of a thread
    for (int r = r0; r < r1; ++r) {
        const int64_t n = v.length_of(r), a = p.add ? max(p.add[r], 0) : 1;
        const int64_t had = (n + page_mask) >> v.page_log2, has = (n + a + page_mask) >> v.page_log2;
        int32_t need = kDenied;
        if (has <= v.max_pages) {
            need = (int32_t)(has - had);
            if (a > 0 && (n & page_mask) != 0) {
                const int last = v.tables[(int64_t)r * v.max_pages + had - 1];
                if (last >= 0 && last < v.num_pages && v.refs[last] > 1) need = (need + 1) | (int32_t)0x80000000;
            }
            mine += need & 0x7fffffff;
        }
        if (per > 1) p.need[r] = need;
        else only = need;
    }
    int64_t wanted;
    int64_t at = exclusive_sum(mine, &wanted);
    // the first `wanted` free pages
    __shared__ int copies, fills;
    if (threadIdx.x == 0) copies = fills = 0;
    int64_t found = 0;
    for (int64_t base = 0; base < v.num_pages && found < wanted; base += kBookThreads * kEach) {
        const int64_t first = base + (int64_t)threadIdx.x * kEach;
        if (base > 0) is_free = free_from(first);
        int64_t here;
        int64_t to = found + exclusive_sum(__popc(is_free), &here);
        for (; is_free != 0 && to < wanted; is_free &= is_free - 1) p.free[to++] = (int32_t)(first + __builtin_ctz(is_free));
        found += here;
    }
    __syncthreads();   // the list is written (by this workgroup), every count is read
    for (int r = r0; r < r1; ++r) {
        const int32_t want = per > 1 ? p.need[r] : only;
        const int need = want & 0x7fffffff;
        const bool denied = want == kDenied;
        const bool ok = !denied && (need == 0 || at + need <= found);
        const int a = ok ? (p.add ? max(p.add[r], 0) : 1) : 0;
        p.granted[r] = a;
        if (ok && a > 0) {
            const int64_t n = v.length_of(r);
            int64_t j = (n + page_mask) >> v.page_log2, from = at;
            int32_t *table = v.tables + (int64_t)r * v.max_pages;
            int left = need;
            if (want < 0) {
                const int src = table[j - 1], dst = p.free[from++];
                --left;
                table[j - 1] = dst;
                atomicSub(&v.refs[src], 1);
                v.refs[dst] = 1;
                p.copies[atomicAdd(&copies, 1)] = PageCopy{src, dst, r, (int)(((n & page_mask) + kPageBlock - 1) / kPageBlock)};
            }
            if (left > 1) p.fills[atomicAdd(&fills, 1)] = PageFill{r, (int32_t)j, (int32_t)from, left};
            if (left == 1) {
                const int dst = p.free[from];
                table[j] = dst;
                v.refs[dst] = 1;
            }
            v.lengths[r] = (int)(n + a);
        }
        if (!denied) at += need;
    }
    __syncthreads();
    if (threadIdx.x == 0) *p.num_copies = copies;
    for (int i = threadIdx.x >> 6; i < fills; i += kBookThreads / 64) {
        const PageFill f = p.fills[i];
        int32_t *table = v.tables + (int64_t)f.row * v.max_pages + f.place;
        for (int e = threadIdx.x & 63; e < f.count; e += 64) {
            const int dst = p.free[f.from + e];
            table[e] = dst;
            v.refs[dst] = 1;
        }
    }
}

// bytes (a multiple of 16) from src to dst by a workgroup
__device__ __forceinline__ void copy_run(uint8_t *dst, const uint8_t *src, int64_t bytes)
{
    const u32x4 *s = reinterpret_cast<const u32x4 *>(src);
    u32x4 *d = reinterpret_cast<u32x4 *>(dst);
    const int64_t n = bytes / 16;
    int64_t i = threadIdx.x;
    for (; i + 3 * 256 < n; i += 4 * 256) {
        u32x4 x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __builtin_nontemporal_load(s + i + e * 256);
#pragma unroll
        for (int e = 0; e < 4; ++e) __builtin_nontemporal_store(x[e], d + i + e * 256);
    }
    for (; i < n; i += 256) d[i] = s[i];
}

// The filled blocks of the copied pages: a workgroup copies those of a head in a layer (one run of memory) at a time.  32 rows' last pages in 32 layers 11 us.
__global__ __launch_bounds__(256) void pages_copy_kernel(PageView v, int layers, const PageCopy *copies, const int32_t *num_copies, int64_t code_layer, int64_t scale_layer)
{
    const int per = layers * v.heads;
    const int64_t units = (int64_t)*num_copies * per;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const PageCopy c = copies[u / per];
        const int rest = (int)(u % per), layer = rest / v.heads, head = rest % v.heads;
        uint8_t *codes = v.codes + layer * code_layer;
        copy_run(codes + v.block_at(c.dst, head, 0), codes + v.block_at(c.src, head, 0), c.blocks * (64 * (int64_t)v.width));
        uint16_t *scales = reinterpret_cast<uint16_t *>(v.scales + layer * scale_layer);
        if ((int)threadIdx.x < c.blocks) scales[v.scale_at(c.dst, head, threadIdx.x) / 2] = scales[v.scale_at(c.src, head, threadIdx.x) / 2];
    }
}

// Tables in place: a workgroup takes some columns of all rows, so that every entry is read before one is written.  32 rows of 34 places 3.2 us (8.7 with all
// columns in one workgroup).
__global__ __launch_bounds__(256) void pages_fork_kernel(PageView v, const int32_t *parents, int cols_log2)
{
    extern __shared__ int32_t was[];   // [rows, cols]
    const int cols = 1 << cols_log2, n = v.rows << cols_log2;
    const int64_t c0 = (int64_t)blockIdx.x << cols_log2;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int64_t c = c0 + (i & (cols - 1));
        was[i] = c < v.max_pages ? v.tables[(i >> cols_log2) * v.max_pages + c] : -1;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 256) {
        const int row = i >> cols_log2, parent = parents[row];
        const int64_t c = c0 + (i & (cols - 1));
        if (c >= v.max_pages || parent < 0 || parent >= v.rows) continue;
        const int old = was[i], now = was[(parent << cols_log2) + (i & (cols - 1))];
        if (old == now) continue;
        v.tables[row * v.max_pages + c] = now;
        if (old >= 0 && old < v.num_pages) atomicSub(&v.refs[old], 1);
        if (now >= 0 && now < v.num_pages) atomicAdd(&v.refs[now], 1);
    }
    if (blockIdx.x != 0) return;
    __syncthreads();
    for (int r = threadIdx.x; r < v.rows; r += 256) was[r] = v.lengths[r];
    __syncthreads();
    for (int r = threadIdx.x; r < v.rows; r += 256) {
        const int parent = parents[r];
        if (parent >= 0 && parent < v.rows && parent != r) v.lengths[r] = was[parent];
    }
}

__global__ __launch_bounds__(256) void pages_truncate_kernel(PageView v, const int32_t *keep)
{
    const int r = blockIdx.x, n = v.length_of(r), k = keep[r];
    if (k < 0 || k >= n) return;
    __syncthreads();   // the length is read
    const int64_t first = ((int64_t)k + (1 << v.page_log2) - 1) >> v.page_log2, last = ((int64_t)n + (1 << v.page_log2) - 1) >> v.page_log2;
    int32_t *table = v.tables + r * v.max_pages;
    for (int64_t j = first + threadIdx.x; j < last; j += 256) {
        const int page = table[j];
        if (page >= 0 && page < v.num_pages) atomicSub(&v.refs[page], 1);
        table[j] = -1;
    }
    if (threadIdx.x == 0) v.lengths[r] = k;
}

struct CompactArgs {
    PageView v;
    int32_t *to;         // [num_pages] scratch: a page's number from now on
    int32_t *src, *dst;  // [num_pages] scratch: the moves
    int32_t *moves;      // scratch: how many
    int32_t *used;
};

// One workgroup: how many pages are in use, then the used ones behind as many numbers and the free ones before, each in order.
__global__ __launch_bounds__(kBookThreads) void pages_compact_kernel(CompactArgs p)
{
    const PageView &v = p.v;
    const int per = (v.num_pages + kBookThreads - 1) / kBookThreads;
    const int p0 = min(v.num_pages, (int)threadIdx.x * per), p1 = min(v.num_pages, p0 + per);
    int64_t mine = 0, used, moves, free;
    for (int i = p0; i < p1; ++i) mine += v.refs[i] > 0 ? 1 : 0;
    exclusive_sum(mine, &used);
    int64_t behind = 0, before = 0;
    for (int i = p0; i < p1; ++i) {
        const bool in_use = v.refs[i] > 0;
        behind += in_use && i >= used ? 1 : 0;
        before += !in_use && i < used ? 1 : 0;
    }
    behind = exclusive_sum(behind, &moves);
    before = exclusive_sum(before, &free);
    for (int i = p0; i < p1; ++i) {
        const bool in_use = v.refs[i] > 0;
        if (in_use && i >= used) p.src[behind++] = i;
        else p.to[i] = i;
        if (!in_use && i < used) p.dst[before++] = i;
    }
    __syncthreads();
    for (int64_t m = threadIdx.x; m < moves; m += kBookThreads) {   // (as many free numbers as pages to move)
        const int src = p.src[m], dst = p.dst[m];
        p.to[src] = dst;
        v.refs[dst] = v.refs[src];
        v.refs[src] = 0;
    }
    if (threadIdx.x == 0) {
        *p.moves = (int32_t)moves;
        *p.used = (int32_t)used;
    }
}

// Tables and pages, a piece of a page to a workgroup at a time: 119 pages of 16 x 128 KB (499 MB read and written) 100 us, 5.0 TB/s; by 2,048 workgroups 105.
constexpr int64_t kMovePiece = 16 << 10;
__global__ __launch_bounds__(256) void pages_move_kernel(CompactArgs p, int layers, int64_t code_layer, int64_t scale_layer)
{
    const PageView &v = p.v;
    const int64_t entries = v.rows * v.max_pages;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < entries; i += (int64_t)gridDim.x * 256) {
        const int page = v.tables[i];
        if (page >= 0 && page < v.num_pages) {
            const int to = p.to[page];
            if (to != page) v.tables[i] = to;
        }
    }
    const int64_t bytes = v.block_at(1, 0, 0), pieces = (bytes + kMovePiece - 1) / kMovePiece;
    const int64_t per = layers * pieces, units = *p.moves * per;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t m = u / per, rest = u - m * per, layer = rest / pieces, at = (rest - layer * pieces) * kMovePiece;
        const int src = p.src[m], dst = p.dst[m];
        uint8_t *codes = v.codes + layer * code_layer;
        copy_run(codes + v.block_at(dst, 0, 0) + at, codes + v.block_at(src, 0, 0) + at, min(kMovePiece, bytes - at));
        if (at == 0) {
            uint16_t *scales = reinterpret_cast<uint16_t *>(v.scales + layer * scale_layer);
            for (int b = threadIdx.x; b < v.heads * v.per_page; b += 256) scales[v.scale_at(dst, 0, 0) / 2 + b] = scales[v.scale_at(src, 0, 0) / 2 + b];
        }
    }
}

// ---- appending ----------------------------------------------------------------------------------------

struct AppendArgs {
    PageView v;
    const void *x[2];              // keys, values
    int64_t token_stride[2], head_stride[2];
    int64_t tokens, most;
    const int32_t *starts, *granted;
    int vec;                       // eight elements from a multiple of eight on are 16-byte loads
};

// The new tokens of a row and the blocks that they lie in.
struct AppendRow {
    NewTokens n;
    int len, first, blocks;
};
__device__ __forceinline__ AppendRow append_row(const AppendArgs &p, int row, int *floor)
{
    AppendRow w;
    w.n = new_tokens(p.starts, row, p.tokens, p.most, floor);
    w.len = p.v.length_of(row);
    w.first = w.len - w.n.count;
    const bool as_it_should = w.n.count > 0 && w.first >= 0 && (!p.granted || p.granted[row] == w.n.count);
    w.blocks = as_it_should ? (w.len + kPageBlock - 1) / kPageBlock - w.first / kPageBlock : 0;
    return w;
}

// A value in units of its block's power of two, and no number for one that is not finite.
__device__ __forceinline__ float code_of(float x)
{
    return (__float_as_uint(x) & 0x7fffffffu) >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : x;
}
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d)
{
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// codes scaled down by a power of two
__device__ __forceinline__ uint32_t scaled_codes(uint32_t w, float down)
{
    return four_codes(__builtin_amdgcn_cvt_f32_fp8(w, 0) * down, __builtin_amdgcn_cvt_f32_fp8(w, 1) * down, __builtin_amdgcn_cvt_f32_fp8(w, 2) * down,
                      __builtin_amdgcn_cvt_f32_fp8(w, 3) * down);
}

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

// Byte b of lane i of each four lanes becomes byte i of lane b: rows of four tokens to columns.
__device__ __forceinline__ uint32_t across_four(uint32_t w)
{
    const uint32_t i = threadIdx.x & 3;
    // what lies one, two and three lanes on
    const uint32_t w1 = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, 0x39, 0xf, 0xf, true), w2 = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, 0x4e, 0xf, 0xf, true),
                   w3 = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, 0x93, 0xf, 0xf, true);
    // byte i of each, in the order of the lanes that they are from: i, i + 1, i + 2, i + 3
    const uint32_t lo = __builtin_amdgcn_perm(w1, w, i | (4 + i) << 8), hi = __builtin_amdgcn_perm(w3, w2, i | (4 + i) << 8);
    const uint32_t all = (lo & 0xffffu) | hi << 16;
    const uint32_t turn = 8 * i;                        // from lane i on: turned to begin with lane 0's
    return turn ? all << turn | all >> (32 - turn) : all;
}

// A wave quantises the new tokens of one block of a head's keys or values.  A lane reads eight elements of two tokens of each chunk of 32 elements
// (keys' own 16 bytes of the chunk), so that the block's largest magnitude is one reduction over the wave; values' codes change places among four lanes with four
// tokens each.  16.7 k tokens of 8 heads of 128 (103 MB read and written) 23.5 us, 4.4 TB/s (30 with a magnitude at a time); one token for each of
// 64 rows 7.0: lengths, tables, counts and codes wait for one another.  18.6 k tokens with bf16 and fp32: heads of 128 24 and 38 us (114 and 190 MB), of 96 20 and 30, of 64 17 and 22;
// by single loads, where a head is no multiple of 8 elements or lies off 16 bytes, of 100 83 and 83, of 68 61 and 56, of 37 34 and 34.
// In the packed form every workgroup looks through all rows for its own: 256 rows of one token 10 us (9 in the other form), 1,024 32 (20), 4,096 312 (79), 16,384 9,900 (335).
// DC: chunks.
template <typename T, int DC>
__global__ __launch_bounds__(256) void pages_append_kernel(AppendArgs p)
{
    const PageView &v = p.v;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, t = lane & 15;
    __shared__ uint32_t wave_sum[4];
    __shared__ int wave_falls[4], found[2];
    int floor = 0;
    // the row of this workgroup's block
    const int groups = (2 * v.heads + 3) / 4;
    const int which = (int)(blockIdx.x / groups), unit = (int)(blockIdx.x - (unsigned)which * groups) * 4 + wave;
    if (!p.starts) {   // one token a row: a block each
        if (append_row(p, which, &floor).blocks == 0) return;
    } else {
        const int per = (v.rows + 255) / 256;
        const int r0 = min(v.rows, (int)threadIdx.x * per), r1 = min(v.rows, r0 + per);
        uint32_t mine, before, total;   // (of rows that overlap, the first time, not what they say)
        auto sums = [&] {
            bool fall = false;
            int f = floor;
            mine = 0;
            for (int r = r0; r < r1; ++r) {
                mine += append_row(p, r, &f).blocks;
                fall |= falls(p.starts, r);
            }
            fall = __any(fall);
            before = mine;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t u = __shfl_up(before, o);
                if (lane >= o) before += u;
            }
            if (lane == 63) {
                wave_sum[wave] = before;
                wave_falls[wave] = fall;
            }
            __syncthreads();
            before -= mine;
            total = 0;
            fall = false;
            for (int w = 0; w < 4; ++w) {
                if (w < wave) before += wave_sum[w];
                total += wave_sum[w];
                fall |= wave_falls[w] != 0;
            }
            return fall;
        };
        if (sums()) {
            floor = floor_of<4>(p.starts, r0, r1, p.tokens, p.most, wave_falls);
            sums();
        }
        if ((uint32_t)which >= total) return;
        if (before <= (uint32_t)which && (uint32_t)which < before + mine)
            for (int r = r0, b = (int)before; r < r1; ++r) {
                const int n = append_row(p, r, &floor).blocks;
                if (which < b + n) {
                    found[0] = r;
                    found[1] = which - b;
                    break;
                }
                b += n;
            }
        __syncthreads();
    }
    if (unit >= 2 * v.heads) return;
    const int row = p.starts ? __builtin_amdgcn_readfirstlane(found[0]) : which;
    floor = 0;
    const AppendRow w = append_row(p, row, &floor);
    const int block = w.first / kPageBlock + (p.starts ? __builtin_amdgcn_readfirstlane(found[1]) : 0), start = block * kPageBlock;
    const int kv = unit & 1, head = unit >> 1;
    const int page = v.tables[row * v.max_pages + (start >> v.page_log2)];
    const int kept = w.first - start, end = w.len - start;   // tokens of the block: those below `kept` are there already, those below `end` are new

    const T *x = static_cast<const T *>(p.x[kv]) + head * p.head_stride[kv];
    // a lane's values as they came: bf16 in pairs, fp32
    constexpr int kWords = sizeof(T) == 2 ? 1 : 2;
    u32x4 y[DC][2][kWords];
    auto value = [&](int c, int h, int e) {   // (constants after unrolling)
        if constexpr (sizeof(T) == 2) return __uint_as_float(e & 1 ? y[c][h][0][e / 2] & 0xffff0000u : y[c][h][0][e / 2] << 16);
        else return __uint_as_float(y[c][h][e / 4][e & 3]);
    };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int token = 16 * h + t;
        const T *src = x + (w.n.first + token - kept) * p.token_stride[kv] + 8 * g;
        const bool there = token >= kept && token < end;
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            const int d = 32 * c + 8 * g;
#pragma unroll
            for (int u = 0; u < kWords; ++u) y[c][h][u] = u32x4{0, 0, 0, 0};
            if (p.vec) {
                if (there && d < v.head_dim)
#pragma unroll
                    for (int u = 0; u < kWords; ++u) y[c][h][u] = reinterpret_cast<const u32x4 *>(src + 32 * c)[u];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (there && d + e < v.head_dim) {
                        if constexpr (sizeof(T) == 2) y[c][h][0][e / 2] |= (uint32_t)src[32 * c + e] << (16 * (e & 1));
                        else y[c][h][e / 4][e & 3] = __float_as_uint(src[32 * c + e]);
                    }
            }
        }
    }
    // the largest magnitude, of the finite ones where some are not
    uint32_t amax = 0;
    if constexpr (sizeof(T) == 2) {
        u16x2 most{0, 0};   // two values at a time
#pragma unroll
        for (int c = 0; c < DC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, y[c][h][0][e] & 0x7fff7fffu));
        amax = (uint32_t)max(most[0], most[1]) << 16;
    } else {
#pragma unroll
        for (int c = 0; c < DC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(value(c, h, e)) & 0x7fffffffu);
    }
    const bool strange = __any(amax >= 0x7f800000u);
    if (strange) {
        amax = 0;
#pragma unroll
        for (int c = 0; c < DC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t bits = __float_as_uint(value(c, h, e)) & 0x7fffffffu;
                    if (bits < 0x7f800000u && bits > amax) amax = bits;
                }
    }
    if (page < 0 || page >= v.num_pages) return;
    const int in_page = block & (v.per_page - 1), holders = v.refs[page];
    uint8_t *to = v.codes + v.block_at(page, head, in_page) + kv * (32 * v.width);
    uint8_t *scale = v.scales + v.scale_at(page, head, in_page) + kv;
    int old = (int)*scale - 127;
    // where this lane's four words of a chunk go: two times eight bytes
    const int at0 = kv ? (t >> 2) * 256 + ((8 * g + (t & 3)) & 15) * 16 + (g >> 1) * 8 : lane * 16, at1 = at0 + (kv ? 64 : 8);
    u32x2 was[DC][2];
    if (kept > 0) {
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            was[c][0] = *reinterpret_cast<const u32x2 *>(to + c * 1024 + at0);
            was[c][1] = *reinterpret_cast<const u32x2 *>(to + c * 1024 + at1);
        }
    }
    asm volatile("" : "+v"(old));   // (all on their way before the first is waited for)
    if (holders > 1) return;
    if (kept <= 0) old = -126;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o));
    int ex = (int)(amax >> 23) - 135 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    ex = ex < -126 ? -126 : ex;
    const bool grows = ex > old;
    if (!grows) ex = old;
    const float inv = __uint_as_float((uint32_t)(127 - ex) << 23);
    const float down = old - ex < -126 ? 0.f : __uint_as_float((uint32_t)(127 + old - ex) << 23);   // (of a code: at least 2^-9, so nothing is left of it anyway)
    // bytes of this lane's words that stay: of word q of a piece
    uint32_t stay[2][2];
#pragma unroll
    for (int piece = 0; piece < 2; ++piece)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            stay[piece][q] = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int token = kv ? 16 * q + (t & 12) + b : 16 * piece + t;
                if (token < kept) stay[piece][q] |= 0xffu << (8 * b);
            }
        }
#pragma unroll
    for (int c = 0; c < DC; ++c) {
        uint32_t code[2][2];   // [token half][four elements]
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float f[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = value(c, h, 4 * q + e) * inv;
                if (strange) {   // (the product is no number either, or infinite)
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] = code_of(f[e]);
                }
                code[h][q] = four_codes(f[0], f[1], f[2], f[3]);
                if (kv) code[h][q] = across_four(code[h][q]);
            }
#pragma unroll
        for (int piece = 0; piece < 2; ++piece) {
            u32x2 out;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                out[q] = kv ? code[q][piece] : code[piece][q];
                if (kept > 0) {
                    const uint32_t before = grows ? scaled_codes(was[c][piece][q], down) : was[c][piece][q];
                    out[q] = (out[q] & ~stay[piece][q]) | (before & stay[piece][q]);
                }
            }
            *reinterpret_cast<u32x2 *>(to + c * 1024 + (piece ? at1 : at0)) = out;
        }
    }
    if (lane == 0) *scale = (uint8_t)(ex + 127);
}

template <typename T>
hipError_t launch_append(const AppendArgs &a, dim3 grid, hipStream_t s)
{
    switch (a.v.width / 32) {
        case 1: hipLaunchKernelGGL((pages_append_kernel<T, 1>), grid, dim3(256), 0, s, a); break;
        case 2: hipLaunchKernelGGL((pages_append_kernel<T, 2>), grid, dim3(256), 0, s, a); break;
        case 3: hipLaunchKernelGGL((pages_append_kernel<T, 3>), grid, dim3(256), 0, s, a); break;
        case 4: hipLaunchKernelGGL((pages_append_kernel<T, 4>), grid, dim3(256), 0, s, a); break;
        case 5: hipLaunchKernelGGL((pages_append_kernel<T, 5>), grid, dim3(256), 0, s, a); break;
        case 6: hipLaunchKernelGGL((pages_append_kernel<T, 6>), grid, dim3(256), 0, s, a); break;
        case 7: hipLaunchKernelGGL((pages_append_kernel<T, 7>), grid, dim3(256), 0, s, a); break;
        default: hipLaunchKernelGGL((pages_append_kernel<T, 8>), grid, dim3(256), 0, s, a); break;
    }
    return hipGetLastError();
}

int64_t layer_bytes(size_t all, const freeze_pages *p) { return (int64_t)(all / p->layers); }

}  // namespace
}  // namespace fz

using namespace fz;

extern "C" {

size_t freeze_pages_bytes(const freeze_pages *pages) { return page_sizes(pages) ? page_code_bytes(pages) : 0; }

size_t freeze_pages_workspace_bytes(const freeze_pages *pages)
{
    if (!page_sizes(pages)) return 0;
    return 3 * up256((size_t)pages->num_pages * 4) + up256((size_t)pages->rows * 4) + 2 * up256((size_t)pages->rows * sizeof(PageCopy)) + 256;
}

int freeze_pages_reserve(const freeze_pages *pages, const int32_t *add, int32_t *out_granted, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!page_sizes(pages) || !out_granted || !workspace || reinterpret_cast<uintptr_t>(add) % 4 != 0 || reinterpret_cast<uintptr_t>(out_granted) % 4 != 0)
        return FREEZE_EINVAL;
    const size_t bytes = freeze_pages_workspace_bytes(pages);
    if (workspace_bytes < bytes || reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return FREEZE_EWORKSPACE;
    const size_t rows = (size_t)pages->rows;
    Extent e[8];
    int n = 0;
    if (!page_extents(pages, 3, e, &n)) return FREEZE_EINVAL;
    auto add_extent = [&](const void *q, size_t size, bool dst) {
        const uintptr_t b = reinterpret_cast<uintptr_t>(q);
        if (q) e[n++] = Extent{b, b + size, dst};
    };
    add_extent(add, rows * 4, false);
    add_extent(out_granted, rows * 4, true);
    add_extent(workspace, bytes, true);
    if (written_twice(e, n)) return FREEZE_EINVAL;
    ReserveArgs a{};
    a.v = page_view(pages, 0);
    a.add = add;
    a.granted = out_granted;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    a.num_copies = reinterpret_cast<int32_t *>(ws);
    ws += 256;
    a.need = reinterpret_cast<int32_t *>(ws);
    ws += up256(rows * 4);
    a.copies = reinterpret_cast<PageCopy *>(ws);
    ws += up256(rows * sizeof(PageCopy));
    a.fills = reinterpret_cast<PageFill *>(ws);
    ws += up256(rows * sizeof(PageFill));
    a.free = reinterpret_cast<int32_t *>(ws);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(kBookThreads), 0, s, a);
    if (hipGetLastError() != hipSuccess) return FREEZE_EHIP;
    const int64_t units = pages->rows * pages->layers * pages->heads;
    hipLaunchKernelGGL(pages_copy_kernel, dim3((unsigned)std::min<int64_t>(units, 2048)), dim3(256), 0, s, a.v, pages->layers, a.copies, a.num_copies,
                       layer_bytes(page_code_bytes(pages), pages), layer_bytes(page_scale_bytes(pages), pages));
    return hipGetLastError() == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

int freeze_pages_fork(const freeze_pages *pages, const int32_t *parents, void *stream)
{
    if (!page_sizes(pages) || !parents || reinterpret_cast<uintptr_t>(parents) % 4 != 0) return FREEZE_EINVAL;
    Extent e[8];
    int n = 0;
    if (!page_extents(pages, 1, e, &n)) return FREEZE_EINVAL;
    const uintptr_t b = reinterpret_cast<uintptr_t>(parents);
    e[n++] = Extent{b, b + (size_t)pages->rows * 4, false};
    if (written_twice(e, n)) return FREEZE_EINVAL;
    int log2 = 6;   // of a workgroup's columns: an entry or some a thread, several columns as long as 64 KB hold them
    while (log2 > 0 && pages->rows << log2 > (log2 > 2 ? 512 : 16384)) --log2;
    const int64_t groups = (pages->max_pages + (1 << log2) - 1) >> log2;
    const size_t lds = (size_t)pages->rows << (log2 + 2);
    hipLaunchKernelGGL(pages_fork_kernel, dim3((unsigned)groups), dim3(256), lds, static_cast<hipStream_t>(stream), page_view(pages, 0), parents, log2);
    return hipGetLastError() == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

int freeze_pages_truncate(const freeze_pages *pages, const int32_t *keep, void *stream)
{
    if (!page_sizes(pages) || !keep || reinterpret_cast<uintptr_t>(keep) % 4 != 0) return FREEZE_EINVAL;
    Extent e[8];
    int n = 0;
    if (!page_extents(pages, 1, e, &n)) return FREEZE_EINVAL;
    const uintptr_t b = reinterpret_cast<uintptr_t>(keep);
    e[n++] = Extent{b, b + (size_t)pages->rows * 4, false};
    if (written_twice(e, n)) return FREEZE_EINVAL;
    hipLaunchKernelGGL(pages_truncate_kernel, dim3((unsigned)pages->rows), dim3(256), 0, static_cast<hipStream_t>(stream), page_view(pages, 0), keep);
    return hipGetLastError() == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

int freeze_pages_compact(const freeze_pages *pages, int32_t *out_used, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!page_sizes(pages) || !out_used || !workspace || reinterpret_cast<uintptr_t>(out_used) % 4 != 0) return FREEZE_EINVAL;
    const size_t bytes = freeze_pages_workspace_bytes(pages);
    if (workspace_bytes < bytes || reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return FREEZE_EWORKSPACE;
    Extent e[8];
    int n = 0;
    if (!page_extents(pages, 3, e, &n)) return FREEZE_EINVAL;
    const uintptr_t u = reinterpret_cast<uintptr_t>(out_used), w = reinterpret_cast<uintptr_t>(workspace);
    e[n++] = Extent{u, u + 4, true};
    e[n++] = Extent{w, w + bytes, true};
    if (written_twice(e, n)) return FREEZE_EINVAL;
    CompactArgs a{};
    a.v = page_view(pages, 0);
    a.used = out_used;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    a.moves = reinterpret_cast<int32_t *>(ws);
    ws += 256;
    int32_t **lists[3] = {&a.to, &a.src, &a.dst};
    for (int32_t **list : lists) {
        *list = reinterpret_cast<int32_t *>(ws);
        ws += up256((size_t)pages->num_pages * 4);
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(kBookThreads), 0, s, a);
    if (hipGetLastError() != hipSuccess) return FREEZE_EHIP;
    hipLaunchKernelGGL(pages_move_kernel, dim3(8192), dim3(256), 0, s, a, pages->layers, layer_bytes(page_code_bytes(pages), pages),
                       layer_bytes(page_scale_bytes(pages), pages));
    return hipGetLastError() == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

int freeze_pages_append(const freeze_pages *pages, int layer, const void *k, int64_t k_token_stride, int64_t k_head_stride, const void *v,
                        int64_t v_token_stride, int64_t v_head_stride, int dtype, int64_t tokens, const int32_t *starts, int64_t most,
                        const int32_t *granted, void *stream)
{
    if (!page_sizes(pages) || layer < 0 || layer >= pages->layers || (dtype != FREEZE_F32 && dtype != FREEZE_BF16) || tokens < 0 || tokens >= (int64_t)1 << 31 ||
        most < 0 || (!starts && tokens != 0 && tokens != pages->rows) || (double)(tokens + 64 * pages->rows) * (pages->heads + 2) >= 1073741824.0)
        return FREEZE_EINVAL;
    if (tokens == 0) return FREEZE_OK;
    const uintptr_t size = dtype == FREEZE_F32 ? 4 : 2;
    int64_t ks, vs;
    if (!k || !v || reinterpret_cast<uintptr_t>(k) % size != 0 || reinterpret_cast<uintptr_t>(v) % size != 0 || reinterpret_cast<uintptr_t>(starts) % 4 != 0 ||
        reinterpret_cast<uintptr_t>(granted) % 4 != 0 || !heads_span(tokens, pages->heads, pages->head_dim, k_token_stride, k_head_stride, false, &ks) ||
        !heads_span(tokens, pages->heads, pages->head_dim, v_token_stride, v_head_stride, false, &vs))
        return FREEZE_EINVAL;
    Extent e[9];
    int n = 0;
    if (!page_extents(pages, 2, e, &n)) return FREEZE_EINVAL;
    auto add_extent = [&](const void *q, size_t bytes) {
        const uintptr_t b = reinterpret_cast<uintptr_t>(q);
        if (q) e[n++] = Extent{b, b + bytes, false};
    };
    add_extent(k, (size_t)ks * size);
    add_extent(v, (size_t)vs * size);
    add_extent(starts, ((size_t)pages->rows + 1) * 4);
    add_extent(granted, (size_t)pages->rows * 4);
    if (written_twice(e, n)) return FREEZE_EINVAL;
    AppendArgs a{};
    a.v = page_view(pages, layer);
    a.x[0] = k;
    a.x[1] = v;
    a.token_stride[0] = k_token_stride;
    a.token_stride[1] = v_token_stride;
    a.head_stride[0] = k_head_stride;
    a.head_stride[1] = v_head_stride;
    a.tokens = tokens;
    a.most = starts ? (most > 0 && most < tokens ? most : tokens) : 1;
    a.starts = starts;
    a.granted = granted;
    a.vec = pages->head_dim % 8 == 0;
    const void *both[2] = {k, v};
    for (int i = 0; i < 2; ++i) {
        if (tokens == 1) a.token_stride[i] = 0;
        if (pages->heads == 1) a.head_stride[i] = 0;
        a.vec &= reinterpret_cast<uintptr_t>(both[i]) % 16 == 0 && a.token_stride[i] % 8 == 0 && a.head_stride[i] % 8 == 0;
    }
    // a row's tokens lie in one block more than they fill, or two
    const int64_t blocks = starts ? std::min(tokens / kPageBlock + 2 * pages->rows, tokens) : tokens;
    const dim3 grid((unsigned)(blocks * ((2 * pages->heads + 3) / 4)));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t err = dtype == FREEZE_F32 ? launch_append<float>(a, grid, s) : launch_append<uint16_t>(a, grid, s);
    return err == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

}  // extern "C"
