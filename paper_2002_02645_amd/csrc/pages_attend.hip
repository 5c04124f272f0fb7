// Attention over pages of keys and values in 8 bits (gfx950 / CDNA4).
//
// A block of 32 tokens of a head lies in memory as the matrix instructions want it: scores are (keys x queries), 16 tokens x 32 elements x 16 columns
// a time, whose results are, lane for lane, the right operand of (values^T x weights).  Nothing goes through LDS and no
// lane needs another's weights; e4m3 codes become bf16 exactly, two an instruction, the values' power of two with them.
#include "pages_attend.h"

namespace fz {

namespace {

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// 64 rows of 4,000 .. 16,000 tokens (1.21 GB) and one of 131,072: 512 workgroups 193 and 50 us, 640: 192 and 48, 768 (three a CU): 189 and 47, 1,024: 225 and 57.
// A tile costs about what eight blocks do: 32 rows of up to 2,000 tokens 16.6 us at 2, 14.1 at 4, 12.7 at 8, 15.6 at 12.
constexpr int kWorkers = 768;         // workgroups that share the work
constexpr int64_t kTileCost = 8;      // of a tile beside its blocks', in blocks: queries, joining the waves
constexpr int64_t kLeastShare = 8;    // of a workgroup
// From kEvenTiles to kMostEven tiles there are as many workgroups as divide them, at most kWorkers, so that none of equal ones is split. Rows of 8 heads and 3,900 tokens each (and of
// 975 .. 6,825): 64 rows 105 -> 83 us (88 -> 86), 80 112 -> 107 (108 -> 111), 97, where 388 workgroups are left, 134 -> 123 (124 -> 122), 112 154 -> 138 (161 -> 155), 128
// 188 -> 157 (173 -> 169). Beyond, ragged ones lose: 144 rows 190 -> 198 (191 -> 209), 160 215 -> 207 (217 -> 223), 193 257 -> 279 (267 -> 305), 256 334 -> 316 (329 -> 331),
// 300 387 -> 397 (381 -> 407).
constexpr int kEvenTiles = 512, kMostEven = 1024;
// Where no row can have more blocks (by its table or the window) and there are no more tiles than workgroups, no tile is split and nothing joined. One row of 250 tokens 10.0
// -> 7.3 us, of 500 11.1 -> 9.5, of 900 11.3 against 12.7; 64 rows of 500 20.3 -> 15.8, of 900 33 -> 26.
constexpr int64_t kWholeBlocks = 24;

// With bf16 queries, weights are taken in two parts of bf16 (2^-17 in all) by both kernels, so that an output does not depend on how many others the call has, and is as exact
// as fp32 sums rounded once. Reading the codes hides the second product in the first kernel (64 rows of 10,000 tokens 192 us either way; 32 columns a wave 2 % more);
// prompts pay for it: five rows of up to 4,096 new tokens 302 us instead of 227 with weights rounded once (2^-8).
constexpr int kWeightParts = 2;

// Codes are read once (or by rows that share pages, at about the same time) and leave the caches to others: 189 us instead of 215 (64 rows of 4,000 .. 16,000).
__device__ __forceinline__ u32x4 load_codes(const uint8_t *p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)); }

template <int DC, int CT, int NS>
constexpr int kAttendPerCu = NS == 1 && CT == 1 && DC <= 4 ? 3 : NS == 1 && ((CT == 2 && DC <= 4) || CT == 1) ? 2 : 1;

// Rows of a few columns each (a token or some of a row): all blocks of all (row, tile of columns, head) lie in one line, kTileCost places before each tile's, which
// is cut into equal shares, one a workgroup, wherever that falls; a tile that several workgroups meet in goes through `part` and pages_join_kernel.  A share's
// blocks go round the workgroup's four waves, whose results meet in LDS at the tile's end.  64 rows of 4,000 .. 16,000 tokens (1.37 GB with 8 heads of 128) 217 us, 6.3 TB/s, with
// fp32 queries, at one workgroup a CU, 220; heads of 100 and 98, whose queries (and outputs) come by elements, the same; heads of 37 120 and 131 (5.7 and 5.2 TB/s).
template <int DC, int CT, int NS>
__global__ __launch_bounds__(256, (kAttendPerCu<DC, CT, NS>)) void pages_attend_kernel(AttendArgs p)
{
    constexpr int kCols = 16 * CT, kFrags = CT * 2 * DC;
    extern __shared__ float lds[];
    const PageView &v = p.v;
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), col = lane & 15;

    // where this workgroup's share begins
    struct Found {
        int64_t sums[8], base;
        RowWork w;
        int row;
    };
    Found *found = reinterpret_cast<Found *>(lds);
    const int per = (v.rows + 255) / 256;
    const int r0 = min(v.rows, (int)threadIdx.x * per), r1 = min(v.rows, r0 + per);
    auto places_of = [&](const RowWork &w) { return p.whole ? 1 : w.blocks + (int)kTileCost; };
    auto cost_of = [&](const RowWork &w) { return (int64_t)places_of(w) * w.tiles * v.heads; };
    RowWork last;
    int64_t mine, tiles;
    int floor = 0;
    auto sums = [&] {
        int f = floor;
        mine = tiles = 0;
        for (int r = r0; r < r1; ++r) {
            last = row_work(p, r, kCols, &f);
            mine += cost_of(last);
            tiles += last.tiles + (falls(p.starts, r) ? kFalls : 0);
        }
        return two_sums<4>(mine, tiles, found->sums);
    };
    TwoSums<4> so_far = sums();
    if (so_far.all[1] >= kFalls) {
        floor = floor_of<4>(p.starts, r0, r1, p.tokens, p.most, reinterpret_cast<int *>(&found->base));
        so_far = sums();
    }
    const int64_t before = so_far.before[0], total = uniform(so_far.all[0]);
    int workers = p.workers;
    const int all = (int)uniform(so_far.all[1] & (kFalls - 1)) * v.heads;
    if (!p.whole && all >= kEvenTiles && all <= kMostEven) workers = (all + (all + kWorkers - 1) / kWorkers - 1) / ((all + kWorkers - 1) / kWorkers);
    int64_t share = (total + workers - 1) / workers;
    share = share < kLeastShare && !p.whole ? kLeastShare : share;
    const int64_t begin = blockIdx.x * share, end = min(total, begin + share);
    if (threadIdx.x == 0 && !p.whole) p.split[blockIdx.x].pieces = 0;
    if (begin >= end) return;
    if (before <= begin && begin < before + mine) {
        int64_t b = before;
        int r = r0;
        if (per > 1)
            for (;; ++r) {
                last = row_work(p, r, kCols, &floor);
                if (begin < b + cost_of(last)) break;
                b += cost_of(last);
            }
        found->row = r;
        found->base = b;
        found->w = last;
    }
    __syncthreads();
    int row = uniform(found->row);
    int64_t base = uniform(found->base);
    RowWork w = uniform(found->w);
    floor = (int)w.n.first + w.n.count;
    __syncthreads();

    for (int64_t at = begin; at < end;) {
        const int64_t row_cost = cost_of(w);
        if (at >= base + row_cost) {
            base += row_cost;
            ++row;
            w = uniform(row_work(p, row, kCols, &floor));
            continue;
        }
        const int tile_cost = places_of(w), item = (int)((at - base) / tile_cost);
        const int from = (int)(at - base - (int64_t)item * tile_cost), upto = (int)min((int64_t)tile_cost, from + end - at);   // places of the tile's
        const int tile = item / v.heads, head = item - tile * v.heads;
        const int col0 = tile * kCols, cols = w.n.count * p.group;
        const int b0 = p.whole ? 0 : max(0, from - (int)kTileCost), count = p.whole ? w.blocks : max(0, upto - (int)kTileCost) - b0;
        const int64_t slot = blockIdx.x * 2 + (at == begin ? 0 : 1);
        at += upto - from;
        if (count == 0 && (w.blocks > 0 || from > 0)) continue;   // (a tile with nothing to attend to: zeros, by whoever has its first place)

        const Blocks blocks(v, row, head);
        const int block0 = w.lo + b0;
        u32x4 k[DC], x[DC];
        uint32_t scales = 0;
        auto load_keys = [&](int page, int i) {
            const uint8_t *from = blocks.at(page, block0 + i);
#pragma unroll
            for (int c = 0; c < DC; ++c) k[c] = load_codes(from + c * 1024 + lane * 16);
            scales = blocks.scale_bytes(page, block0 + i);
        };
        auto load_values = [&](int page, int i) {
            const uint8_t *from = blocks.at(page, block0 + i) + blocks.block_bytes / 2;
#pragma unroll
            for (int c = 0; c < DC; ++c) x[c] = load_codes(from + c * 1024 + lane * 16);
        };
        int i = wave;
        int page = i < count ? uniform(blocks.page(block0 + i)) : -1, coming = i + 4 < count ? blocks.page(block0 + i + 4) : -1;
        if (blocks.there(page)) {
            load_keys(page, i);
            load_values(page, i);
        }

        uint16_t *staged = reinterpret_cast<uint16_t *>(lds);
        stage_queries<DC, NS, 256>(p, w, head, col0, kCols, staged);
        __syncthreads();
        bf16x8 q[CT][NS][DC];
        Sight<CT> sight;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            take_queries<DC, NS>(staged, kCols, 16 * ct, q[ct]);
            const int c = col0 + 16 * ct + col;
            sight.set(ct, c < cols ? w.len - w.n.count + c / p.group : -1, p.window);
        }
        // places of the tile's tokens
        const int lowest = w.len - w.n.count + col0 / p.group, highest = w.len - w.n.count + (min(cols, col0 + kCols) - 1) / p.group;

        Running<DC, CT> run;
        run.clear();
        const int unseen = p.window > 0 ? (int)(highest - p.window) : -1;   // the last place that some column does not see any more
        for (; i < count; i += 4) {
            const int next = uniform(coming);   // (asked for a block ago)
            coming = i + 8 < count ? blocks.page(block0 + i + 8) : -1;
            f32x4 s[CT][2];
            const bool here = blocks.there(page), more = blocks.there(next);
            const int first = (block0 + i) * kPageBlock;
            const bool edge = first + kPageBlock - 1 > lowest || first <= unseen;
            const float ks = score_factor(p.scale_log2, scales), vs = value_factor(scales);
            if (here) scores_of<DC, CT, NS>(k, q, s);
            if (more) load_keys(next, i + 4);
            if (here) {
                weigh<DC, CT>(run, s, ks, edge, first, sight);
                add_values<DC, CT, (NS > 1 ? NS : kWeightParts)>(run, x, vs, s, edge, first, sight);
            }
            if (more) load_values(next, i + 4);
            page = next;
        }

        // the four waves' results under one reference
        __syncthreads();   // (the queries are read)
        float *ml = lds;   // [4][2][kCols]
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            float l = run.l[ct];
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (lane < 16) {
                ml[(wave * 2) * kCols + 16 * ct + lane] = run.m[ct];
                ml[(wave * 2 + 1) * kCols + 16 * ct + lane] = l;
            }
        }
        __syncthreads();
        const bool whole = count == w.blocks;
        if (threadIdx.x == 0 && !whole && b0 == 0) {
            // the others: up to the share that the tile's last place lies in
            const int64_t last_place = at - upto + tile_cost - 1;
            p.split[blockIdx.x] = SplitTile{w.n.first, cols, col0, head, (int)(last_place / share - blockIdx.x) + 1, (int)slot};
        }
        f32x4 *frags = reinterpret_cast<f32x4 *>(lds + 8 * kCols);   // [4][2 DC][64]
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u) m = fmaxf(m, ml[u * 2 * kCols + 16 * ct + col]);
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int u = 0; u < 4; ++u) l += ml[(u * 2 + 1) * kCols + 16 * ct + col] * __builtin_amdgcn_exp2f(ml[u * 2 * kCols + 16 * ct + col] - ref);
            const float a = __builtin_amdgcn_exp2f(run.m[ct] - ref);
#pragma unroll
            for (int f = 0; f < 2 * DC; ++f) frags[(wave * 2 * DC + f) * 64 + lane] = run.o[ct][f] * a;
            if (!whole && threadIdx.x < 16) {
                p.part_ml[(slot * 2) * kCols + 16 * ct + lane] = m;
                p.part_ml[(slot * 2 + 1) * kCols + 16 * ct + lane] = l;
            }
            __syncthreads();
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const int c = col0 + 16 * ct + col;   // (of thread and of lane alike)
            if (c < cols)
                for (int f = wave; f < 2 * DC; f += 4) {
                    f32x4 o = frags[f * 64 + lane];
#pragma unroll
                    for (int u = 1; u < 4; ++u) o += frags[(u * 2 * DC + f) * 64 + lane];
                    if (whole) store_out(p, w.n.first, head, c, 16 * f + 4 * (lane >> 4), o * inv);
                    else reinterpret_cast<f32x4 *>(p.part_o)[(slot * kFrags + ct * 2 * DC + f) * 64 + lane] = o;
                }
            __syncthreads();
        }
    }
}

// A tile that several workgroups had a piece of: their sums under one reference, the pieces over a workgroup's waves.  blockIdx.x: the worker of the first
// piece, blockIdx.y: a fragment (16 columns x 16 elements).
template <int DC, int CT>
__global__ __launch_bounds__(256) void pages_join_kernel(AttendArgs p)
{
    constexpr int kCols = 16 * CT, kFrags = CT * 2 * DC;
    const SplitTile t = p.split[blockIdx.x];
    if (t.pieces == 0) return;
    __shared__ f32x4 os[4][64];
    __shared__ float ms[4][16], ls[4][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, frag = blockIdx.y, ct = frag / (2 * DC), in = 16 * ct + (lane & 15);
    const bool there = t.col0 + in < t.columns;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    if (there) {
        constexpr int kAhead = 4;
        for (int u = wave; u < t.pieces; u += 4 * kAhead) {
            f32x4 x[kAhead];
            float pm[kAhead], pl[kAhead];
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const int piece = u + 4 * e;
                pm[e] = -INFINITY;
                pl[e] = 0.f;
                x[e] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (piece < t.pieces) {
                    const int64_t slot = piece == 0 ? t.slot : 2 * ((int64_t)blockIdx.x + piece);
                    pm[e] = p.part_ml[slot * 2 * kCols + in];
                    pl[e] = p.part_ml[(slot * 2 + 1) * kCols + in];
                    x[e] = reinterpret_cast<const f32x4 *>(p.part_o)[(slot * kFrags + frag) * 64 + lane];
                }
            }
            float top = m;
#pragma unroll
            for (int e = 0; e < kAhead; ++e) top = fmaxf(top, pm[e]);
            const float ref = top == -INFINITY ? 0.f : top, a = __builtin_amdgcn_exp2f(m - ref);
            m = top;
            l *= a;
            o *= a;
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const float b = __builtin_amdgcn_exp2f(pm[e] - ref);
                l += b * pl[e];
                o += x[e] * b;
            }
        }
    }
    os[wave][lane] = o;
    if (lane < 16) {
        ms[wave][lane] = m;
        ls[wave][lane] = l;
    }
    __syncthreads();
    if (wave != 0 || !there) return;
    const int c = lane & 15;
    const float top = fmaxf(fmaxf(ms[0][c], ms[1][c]), fmaxf(ms[2][c], ms[3][c])), ref = top == -INFINITY ? 0.f : top;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
    l = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const float a = __builtin_amdgcn_exp2f(ms[u][c] - ref);
        l += a * ls[u][c];
        o += os[u][lane] * a;
    }
    store_out(p, t.first, t.head, t.col0 + in, 16 * (frag - ct * 2 * DC) + 4 * (lane >> 4), o * (l == 0.f ? 0.f : 1.f / l));
}

// Prompts: a workgroup's waves have 16 * CT columns each, one after another, and walk over the blocks that these see, each by itself: the codes of a
// block come from memory once and from the caches for the other waves.  Nothing is split: there are tiles enough.  Later tiles of a row see more and go first.
// Bound by what a SIMD issues: a block's 48 matrix instructions (16 for scores, 32 for values with the weights in two parts: 768 cycles of the matrix cores, two issue places
// each) come with 64 conversions, 16 exponentials and 160 other vector instructions, which together take 108 % of the SIMDs' cycles: five rows of up to 4,096 new tokens
// 302 us, 0.65 PFLOP/s of the products asked for, 1.0 of those done (a library product of 8,192^3 on the same card: 1.10).  Measured with weights in one part (243 us):
// four columns of 16 a wave need 512 registers and copy half of them (643 us where two needed 307), three spill (406); codes turned into bf16
// once for a workgroup of eight waves, in LDS, 283 us; codes shared by four waves through LDS 275; codes two blocks ahead 241 against 245, at registers that wide heads lack.
// Heads above 160 have one column of 16 a wave and two waves a SIMD; with two columns and one wave 16 rows of 256 behind 4,000 need 857 us against 694 (heads of 192) and 1,039
// against 869 (256); heads of 160, two waves either way, 450 against 556.
// NS = 3: queries of fp32 and the weights in three parts of bf16 each, three times the products: 4 rows of 2,048 new tokens behind 500 places 529 us, where the kernel
// above needs 1,565 (it knows the end of a row's blocks, not of a tile's). Heads above
// 192 then have a SIMD's registers to one wave: 16 rows of 256 behind 4,000, heads of 256, 1,650 us against 2,436.
template <int DC, int CT, int NS>
__global__ __launch_bounds__(256, CT == 1 && NS == 1 && DC <= 4 ? 3 : NS > 1 && DC > 6 ? 1 : 2) void pages_prompt_kernel(AttendArgs p)
{
    constexpr int kWave = 16 * CT, kCols = 4 * kWave;
    const PageView &v = p.v;
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), col = lane & 15;
    extern __shared__ float lds[];
    // the tile: row and number within it
    int64_t *sums = reinterpret_cast<int64_t *>(lds);
    int *found = reinterpret_cast<int *>(sums + 8);
    const int per = (v.rows + 255) / 256;
    const int r0 = min(v.rows, (int)threadIdx.x * per), r1 = min(v.rows, r0 + per);
    int64_t mine;
    int floor = 0;
    auto tiles_of = [&] {
        int f = floor;
        int64_t fall = 0;
        mine = 0;
        for (int r = r0; r < r1; ++r) {
            mine += row_work(p, r, kCols, &f).tiles;
            fall += falls(p.starts, r);
        }
        return two_sums<4>(mine, fall, sums);
    };
    TwoSums<4> so_far = tiles_of();
    if (so_far.all[1] > 0) {
        floor = floor_of<4>(p.starts, r0, r1, p.tokens, p.most, found);
        so_far = tiles_of();
    }
    const int before = (int)so_far.before[0], total = (int)so_far.all[0];
    const int head = blockIdx.x % v.heads, tile = total - 1 - (int)(blockIdx.x / v.heads);
    if (tile < 0) return;
    if (before <= tile && tile < before + mine)
        for (int r = r0, b = before; r < r1; ++r) {
            const int n = row_work(p, r, kCols, &floor).tiles;
            if (tile < b + n) {
                found[0] = r;
                found[1] = tile - b;
                break;
            }
            b += n;
        }
    __syncthreads();
    const int row = uniform((int)found[0]);
    floor = 0;   // (this row is in order)
    const RowWork w = row_work(p, row, kCols, &floor);
    const int cols = w.n.count * p.group, tile0 = uniform((int)found[1]) * kCols, col0 = tile0 + wave * kWave;
    __syncthreads();
    uint16_t *staged = reinterpret_cast<uint16_t *>(lds);
    stage_queries<DC, NS, 256>(p, w, head, tile0, kCols, staged);
    __syncthreads();
    bf16x8 q[CT][NS][DC];
    Sight<CT> sight;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        take_queries<DC, NS>(staged, kCols, wave * kWave + 16 * ct, q[ct]);
        const int c = col0 + 16 * ct + col;
        sight.set(ct, c < cols ? w.len - w.n.count + c / p.group : -1, p.window);
    }
    __syncthreads();   // (the queries are read)
    if (col0 >= cols) return;
    const int lowest = w.len - w.n.count + col0 / p.group, highest = w.len - w.n.count + (min(cols, col0 + kWave) - 1) / p.group;
    const int seen = p.window > 0 ? (int)max((int64_t)0, lowest - p.window + 1) : 0;
    const int lo = seen / kPageBlock, hi = highest < 0 ? 0 : highest / kPageBlock + 1;

    constexpr int kParts = NS > 1 ? NS : kWeightParts;
    f32x4 o[CT][2 * DC];
    float m[CT], sum[CT];   // sum: of the lane's own tokens
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = -INFINITY;
        sum[ct] = 0.f;
#pragma unroll
        for (int f = 0; f < 2 * DC; ++f) o[ct][f] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const Blocks blocks(v, row, head);
    const int unseen = p.window > 0 ? (int)(highest - p.window) : -1;   // the last place that some column does not see any more
    const float scale_log2 = p.scale_log2;
    u32x4 k[DC], x[DC];
    // a page that is not there: block b of page 0 in its place, none of whose tokens count
    auto load_keys = [&](int page, int b) {
        const uint8_t *from = blocks.at(blocks.there(page) ? page : 0, b);
#pragma unroll
        for (int c = 0; c < DC; ++c) k[c] = *reinterpret_cast<const u32x4 *>(from + c * 1024 + lane * 16);
    };
    auto load_values = [&](int page, int b) {
        const uint8_t *from = blocks.at(blocks.there(page) ? page : 0, b) + blocks.block_bytes / 2;
#pragma unroll
        for (int c = 0; c < DC; ++c) x[c] = *reinterpret_cast<const u32x4 *>(from + c * 1024 + lane * 16);
    };
    auto scale_of = [&](int page, int b) { return blocks.scale_bytes(blocks.there(page) ? page : 0, b); };
    // Block b's weights and its values' product, beside the scores of block b + 1 (`then`): matrix and vector instructions that do not wait for each other.
    int page = lo < hi ? uniform(blocks.page(lo)) : -1, next = lo + 1 < hi ? uniform(blocks.page(lo + 1)) : -1, coming = lo + 2 < hi ? blocks.page(lo + 2) : -1;
    uint32_t scales = scale_of(page, lo), scales_next = scale_of(next, lo + 1);
    f32x4 s0[CT][2], s1[CT][2];
    load_keys(page, lo);
    load_values(page, lo);
    scores_of<DC, CT, NS>(k, q, s0);
    load_keys(next, lo + 1);
    auto step = [&](int b, f32x4 (&s)[CT][2], f32x4 (&then)[CT][2]) {
        const int first = b * kPageBlock;
        float ks = score_factor(scale_log2, scales), vs = value_factor(scales);
        if (!blocks.there(page)) {
            ks = vs = 1.f;   // (page 0's bytes may be anything: an infinite factor would make its zeros no numbers)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[ct][0] = s[ct][1] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < DC; ++c) x[c] = u32x4{0, 0, 0, 0};
        }
        if (first + kPageBlock - 1 > lowest || first <= unseen) {
            hide(s, first, sight);
            take_out_strange<DC, CT>(o, x, first, sight);
        }
        page = next;
        next = uniform(coming);   // (asked for a block ago)
        coming = b + 3 < hi ? blocks.page(b + 3) : -1;
        bool follow = false;
        float top[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            top[ct] = largest_of(s, ct) * ks;
            follow |= top[ct] > m[ct] + kSlack;
        }
        if (__any(follow)) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float t = fmaxf(top[ct], __shfl_xor(top[ct], 16));
                t = fmaxf(m[ct], fmaxf(t, __shfl_xor(t, 32)));
                const float a = t == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[ct] - t);
                m[ct] = t;
                sum[ct] *= a;
#pragma unroll
                for (int f = 0; f < 2 * DC; ++f) o[ct][f] *= a;
            }
        }
        scores_of<DC, CT, NS>(k, q, then);
        bf16x8 f[CT][kParts];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const float ref = m[ct] == -INFINITY ? 0.f : m[ct];
            float e[8];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[4 * t + i] = __builtin_amdgcn_exp2f(fmaf(s[ct][t][i], ks, -ref));
                    sum[ct] += e[4 * t + i];
                }
            parts_of<kParts>(e, f[ct]);
        }
        load_keys(next, b + 2);
#pragma unroll
        for (int c = 0; c < DC; ++c)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8 y = values_of(x[c][2 * u], x[c][2 * u + 1], vs);
#pragma unroll
                for (int n = 0; n < kParts; ++n)
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) o[ct][2 * c + u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, f[ct][n], o[ct][2 * c + u], 0, 0, 0);
            }
        scales = scales_next;
        scales_next = scale_of(next, b + 2);
        load_values(page, b + 1);
    };
    for (int b = lo; b < hi; b += 2) {
        step(b, s0, s1);
        if (b + 1 < hi) step(b + 1, s1, s0);
    }
    // outputs go through LDS, 16 columns of a wave at a time, to leave as whole rows
    f32x4 *mine_out = reinterpret_cast<f32x4 *>(lds) + wave * (16 * (8 * DC + 1));   // [16][8 DC + 1]
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        float l = sum[ct];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int f = 0; f < 2 * DC; ++f) mine_out[col * (8 * DC + 1) + 4 * f + (lane >> 4)] = o[ct][f] * inv;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
        for (int e = lane; e < 16 * 8 * DC; e += 64) {
            const int in = e / (8 * DC), d = e % (8 * DC), c = col0 + 16 * ct + in;
            if (c < cols) store_out(p, w.n.first, head, c, 4 * d, mine_out[in * (8 * DC + 1) + d]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// ---- host -------------------------------------------------------------------------------------------

constexpr int64_t kFewColumns = 64;   // of a row: the prompts' kernel has as many a workgroup with 16 a wave

struct AttendPlan {
    int ct, parts;
    int prompt;   // 0: not the prompts' kernel; 1, 2: with 16, 32 columns a wave (16 where heads are wider than 160)
    bool both;    // rows of few columns beside prompts: those go to the kernel that splits them
    size_t o_bytes, ml_bytes, split_bytes;
    size_t bytes() const { return o_bytes + ml_bytes + split_bytes; }
};
// most_blocks: that a row can have
AttendPlan attend_plan(const freeze_pages *p, int group, int64_t tokens, int64_t most, int parts, int64_t most_blocks)
{
    AttendPlan pl;
    const int64_t cols = (most > 0 ? most : 1) * group;
    pl.parts = parts;
    // Eight heads, groups of four, dim 128; new tokens a row behind 500 / 4,000 / 16,000 places, us:
    //   16 columns a wave against 32: 16 rows of 5: 16 18 / 49 47 / 161 112; of 16: 24 32 / 98 70 / 337 192; 4 rows of 8: 15 16 / 21 27 / 50 45
    //   (twice as much is read, but smaller tiles come and go faster: 4,096 columns and heads are where it turns);
    //   the better of those, the prompts' kernel with 16 and with 32 columns a wave: 1 row of 256 (8,192): 40 19 29 / 56 73 114 / 151 307 416; of 512 (16,384): 27 23 35 /
    //   72 78 120 / 233 322 424; of 1,024 (32,768): 60 40 48 / 153 133 133 / 485 473 438; 4 rows of 64: 14 16 24 / 60 84 114 / 154 311 418; of 128: 19 18 26 / 70 86 115 /
    //   242 311 415; of 256: 39 28 30 / 138 128 118 / 474 472 417; 16 rows of 32: 17 16 24 / 75 86 116 / 260 425 512; of 64: 38 24 26 / 145 127 116 / 522 508 511;
    //   of 128 (65,536): 85 45 41 / 334 232 192 / 1189 962 771.
    //   (A prompt's tile walks its blocks one after another, about 0.5 us each: few tiles of long rows wait for that, so sizes between take it where no row can be long.)
    //   With fp32, that kernel and this: 1 row of 256: 12 15 without a past, 21 26 / - / -; of 512: 42 32 / - / -; of 1,024: 132 62 / 370 207 / 1166 697; 4 rows of 64: 17 22;
    //   of 128: 31 25; of 256: 80 42 / 318 190 / 1113 699; 16 rows of 64: 73 35 / 311 186 / 1151 772; heads of 192: 1 row of 512: 79 43; of 1,024: 241 85 / 667 287 / 2082 982.
    const int64_t all = tokens * group * p->heads;
    pl.ct = parts > 1 || cols <= 16 || all < 4096 ? 1 : 2;
    pl.prompt = cols <= kFewColumns ? 0 : all >= 32768 ? 2 : all >= (parts > 1 ? 16384 : 8192) && most_blocks <= 64 ? 1 : 0;
    const size_t slots = 2 * kWorkers, kCols = 16 * pl.ct;
    pl.o_bytes = slots * kCols * page_width(p->head_dim) * 4;
    pl.ml_bytes = slots * 2 * kCols * 4;
    pl.split_bytes = up256(kWorkers * sizeof(SplitTile));
    // Rows of few columns beside prompts would each walk their blocks with one wave of four.  So where there may be such (the shortest row, where the others have as many tokens
    // as they may), and rows may be long or are short on the average, both kernels are launched, each for its rows.  A prompt of 1,024 tokens beside a row of one token
    // behind 1,000 / 2,000 / 4,000 / 16,000 / 131,071 places: 36 / 56 / 103 / 418 / 3,761 us with the prompts' kernel alone, 49 / 49 / 50 / 56 / 103 with both; of 2,048 beside 32 rows
    // of one behind 1,000 / 2,000 / 4,000 / 16,000: 95 114 153 518 and 106 118 140 268, beside 64 rows of 8 behind 10,000: 362 and 286 (472 with 16 columns a wave);
    // prompts of 4,096, 300, 200, 180 and 7 tokens, none of them long: 208 and 219.  1,024 rows of one token behind 1,000 in the packed form, `most` not given: 452 and 358 (429
    // with 32 columns a wave).
    const bool ones = tokens * group <= 16 * p->rows;
    pl.both = pl.prompt && (tokens - (p->rows - 1) * most) * group <= kFewColumns && (most_blocks > 64 || ones);
    if (pl.both && ones) pl.ct = 1;   // (the workspace's size is the one for 32 columns a wave)
    return pl;
}

template <int DC, int CT, int NS>
hipError_t launch_attend(const AttendArgs &a, hipStream_t s)
{
    constexpr int kFrags = CT * 2 * DC;
    constexpr size_t lds = std::max((size_t)NS * 16 * CT * kQueryRow<DC> * 2, (size_t)8 * 16 * CT * 4 + 4 * 2 * DC * 1024);
    static_assert(lds <= 65536 + 2048, "LDS");
    hipLaunchKernelGGL((pages_attend_kernel<DC, CT, NS>), dim3(a.workers), dim3(256), lds, s, a);
    if (hipGetLastError() != hipSuccess) return hipErrorLaunchFailure;
    if (a.whole) return hipSuccess;
    hipLaunchKernelGGL((pages_join_kernel<DC, CT>), dim3(a.workers, kFrags), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <int DC, int CT, int NS>
hipError_t launch_prompt(const AttendArgs &a, hipStream_t s)
{
    constexpr int64_t cols = 64 * CT;
    constexpr size_t lds = std::max((size_t)NS * cols * kQueryRow<DC> * 2, (size_t)4 * 16 * (8 * DC + 1) * 16);
    const int64_t all = a.tokens * a.group, rows = std::min<int64_t>(a.v.rows, all / a.least_cols);   // (rows that it takes)
    const int64_t n = std::min(all / cols + rows, a.tokens * ((a.group + cols - 1) / cols));
    hipLaunchKernelGGL((pages_prompt_kernel<DC, CT, NS>), dim3((unsigned)(n * a.v.heads)), dim3(256), lds, s, a);
    return hipGetLastError();
}
template <int DC>
hipError_t launch_split(const AttendArgs &a, const AttendPlan &pl, hipStream_t s)
{
    if (pl.parts > 1) return launch_attend<DC, 1, 3>(a, s);
    if (pl.ct == 1) return launch_attend<DC, 1, 1>(a, s);
    return launch_attend<DC, 2, 1>(a, s);
}
template <int DC>
hipError_t launch_width(AttendArgs a, const AttendPlan &pl, hipStream_t s)
{
    if (pl.both) {
        a.most_cols = kFewColumns;
        const hipError_t err = launch_split<DC>(a, pl, s);
        if (err != hipSuccess) return err;
        a.least_cols = kFewColumns + 1;
        a.most_cols = (int64_t)1 << 31;
    }
    if (pl.prompt) {
        if (pl.parts > 1) return launch_prompt<DC, 1, 3>(a, s);
        if constexpr (DC <= 5)
            if (pl.prompt == 2) return launch_prompt<DC, 2, 1>(a, s);
        return launch_prompt<DC, 1, 1>(a, s);
    }
    return launch_split<DC>(a, pl, s);
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
    const AttendPlan pl = attend_plan(pages, group, tokens, most_of(tokens, most, packed), 1, 0);
    return pl.bytes();
}

int freeze_pages_attend(const freeze_pages *pages, int layer, const void *q, int q_dtype, int64_t q_token_stride, int64_t q_head_stride, int group,
                        int64_t tokens, const int32_t *starts, int64_t most, float scale, int64_t window, void *out, int out_dtype,
                        int64_t out_token_stride, int64_t out_head_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!attend_sizes(pages, group, tokens, most) || layer < 0 || layer >= pages->layers || (q_dtype != FREEZE_F32 && q_dtype != FREEZE_BF16) ||
        (out_dtype != FREEZE_F32 && out_dtype != FREEZE_BF16) || !(scale > 0.f && scale <= 2.0e38f) || window < 0 || window >= (int64_t)1 << 31 ||
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
    const int64_t most_blocks = std::min(pages->max_pages * (pages->page_tokens / kPageBlock), window > 0 ? (window + each) / kPageBlock + 2 : (int64_t)1 << 31);
    const AttendPlan pl = attend_plan(pages, group, tokens, each, q_dtype == FREEZE_F32 ? 3 : 1, most_blocks);
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
    a.least_cols = 1;
    a.most_cols = (int64_t)1 << 31;
    a.group = group;
    a.q_vec = qb % 16 == 0 && pages->head_dim % 8 == 0 && a.q_token % 8 == 0 && a.q_head % 8 == 0;
    a.out_bf16 = out_dtype == FREEZE_BF16;
    a.out_vec = ob % (4 * os) == 0 && pages->head_dim % 4 == 0 && a.out_token % 4 == 0 && a.out_head % 4 == 0;
    a.scale_log2 = scale * 1.4426950408889634f;
    const int64_t cols = 16 * pl.ct, tiles = std::min(tokens * group / cols + pages->rows, tokens * ((group + cols - 1) / cols)) * pages->heads;
    a.whole = most_blocks <= kWholeBlocks && tiles <= kWorkers;
    a.workers = a.whole ? (int)std::min<int64_t>(tiles, kWorkers) : kWorkers;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    a.split = reinterpret_cast<SplitTile *>(ws);
    ws += pl.split_bytes;
    a.part_ml = reinterpret_cast<float *>(ws);
    ws += pl.ml_bytes;
    a.part_o = reinterpret_cast<float *>(ws);
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t err = hipErrorInvalidValue;
    switch (a.v.width / 32) {
        case 1: err = launch_width<1>(a, pl, s); break;
        case 2: err = launch_width<2>(a, pl, s); break;
        case 3: err = launch_width<3>(a, pl, s); break;
        case 4: err = launch_width<4>(a, pl, s); break;
        case 5: err = launch_width<5>(a, pl, s); break;
        case 6: err = launch_width<6>(a, pl, s); break;
        case 7: err = launch_width<7>(a, pl, s); break;
        case 8: err = launch_width<8>(a, pl, s); break;
    }
    return err == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

}  // extern "C"
