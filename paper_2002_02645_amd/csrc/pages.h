// Keys and values in pages of 8 bits: what the bookkeeping, the appending and the attention share.  Not part of the C ABI.
#pragma once
#include "../../include/freeze.h"
#include "extents.h"
#include "freeze_internal.h"

namespace fz {

constexpr int kPageBlock = 32;        // tokens that share an exponent
constexpr int kMostRows = 16384;
constexpr int kMostHeadDim = 256;

inline int page_width(int head_dim) { return (head_dim + 31) / 32 * 32; }

// The pool as the kernels see it; `layer` has gone into codes and scales.
struct PageView {
    uint8_t *codes, *scales;
    int32_t *refs, *tables, *lengths;
    int64_t max_pages;
    int num_pages, rows, heads, head_dim, width;
    int page_log2, per_page;          // log2 of a page's tokens, blocks of a page
    // first byte of a block's keys (its values follow), number of its two scales
    __host__ __device__ int64_t block_at(int page, int head, int block) const
    {
        return (((int64_t)page * heads + head) * per_page + block) * (64 * (int64_t)width);
    }
    __host__ __device__ int64_t scale_at(int page, int head, int block) const { return (((int64_t)page * heads + head) * per_page + block) * 2; }
    // tokens of a row, within what its table can hold
    __device__ int length_of(int row) const
    {
        const int64_t most = max_pages << page_log2;
        const int n = lengths[row];
        return n < 0 ? 0 : n > most ? (int)most : n;
    }
};

// sizes within the limits of the C ABI
inline bool page_sizes(const freeze_pages *p)
{
    if (!p || p->layers < 1 || p->layers > 1024 || p->heads < 1 || p->heads > 1024 || p->head_dim < 1 || p->head_dim > kMostHeadDim) return false;
    if (p->page_tokens < kPageBlock || p->page_tokens > 1024 || (p->page_tokens & (p->page_tokens - 1)) != 0) return false;
    if (p->num_pages < 1 || p->num_pages > (1 << 24) || p->rows < 1 || p->rows > kMostRows || p->max_pages < 1 || p->max_pages > (1 << 20)) return false;
    if (p->max_pages * p->page_tokens >= (int64_t)1 << 31) return false;
    const double bytes = 2.0 * page_width(p->head_dim) * p->page_tokens * (double)p->heads * (double)p->num_pages * (double)p->layers;
    return bytes <= (double)((int64_t)1 << 46);
}
inline size_t page_code_bytes(const freeze_pages *p)
{
    return (size_t)2 * page_width(p->head_dim) * p->page_tokens * p->heads * p->num_pages * p->layers;
}
inline size_t page_scale_bytes(const freeze_pages *p) { return page_code_bytes(p) / (32 * (size_t)page_width(p->head_dim)); }

inline PageView page_view(const freeze_pages *p, int layer)
{
    PageView v{};
    v.width = page_width(p->head_dim);
    v.codes = p->codes + page_code_bytes(p) / p->layers * layer;
    v.scales = p->scales + page_scale_bytes(p) / p->layers * layer;
    v.refs = p->refs;
    v.tables = p->tables;
    v.lengths = p->lengths;
    v.max_pages = p->max_pages;
    v.num_pages = (int)p->num_pages;
    v.rows = (int)p->rows;
    v.heads = p->heads;
    v.head_dim = p->head_dim;
    v.page_log2 = __builtin_ctz((unsigned)p->page_tokens);
    v.per_page = p->page_tokens / kPageBlock;
    return v;
}

// The extents of a pool and whether its pointers are there and aligned.  written: 1 the bookkeeping, 2 codes and scales, 3 both
inline bool page_extents(const freeze_pages *p, int written, Extent *e, int *n)
{
    auto add = [&](const void *q, size_t bytes, size_t align, bool dst) {
        const uintptr_t b = reinterpret_cast<uintptr_t>(q);
        e[(*n)++] = Extent{b, b + bytes, dst};
        return q && b % align == 0;
    };
    const bool data = written & 2, book = written & 1;
    return add(p->codes, page_code_bytes(p), 16, data) && add(p->scales, page_scale_bytes(p), 2, data) && add(p->refs, (size_t)p->num_pages * 4, 4, book) &&
           add(p->tables, (size_t)(p->rows * p->max_pages) * 4, 4, book) && add(p->lengths, (size_t)p->rows * 4, 4, book);
}

// Elements from the first to behind the last of [tokens, heads, dim] with strides; false where they are out of range or two heads share one.
inline bool heads_span(int64_t tokens, int64_t heads, int64_t dim, int64_t token_stride, int64_t head_stride, bool written, int64_t *span)
{
    constexpr int64_t kMost = (int64_t)1 << 44;
    if (token_stride < 0 || head_stride < 0 || token_stride > kMost || head_stride > kMost) return false;
    const double size = (double)(tokens - 1) * (double)token_stride + (double)(heads - 1) * (double)head_stride + (double)dim;
    if (size > (double)kMost) return false;
    *span = (tokens - 1) * token_stride + (heads - 1) * head_stride + dim;
    if (!written) return true;
    int64_t n0 = heads, s0 = head_stride, n1 = tokens, s1 = token_stride;
    if (s1 < s0) {
        std::swap(n0, n1);
        std::swap(s0, s1);
    }
    if (n0 > 1 && s0 < dim) return false;
    return n1 <= 1 || s1 >= (n0 > 1 ? (n0 - 1) * s0 : 0) + dim;
}

// One row's new tokens: their number (0: none, or not as they should be) and the first of them.
struct NewTokens {
    int count;
    int64_t first;
};
// floor: no smaller than the ends of the rows before that are in order by themselves; the row's own becomes part of it.  A row that begins below it counts for nothing, so that
// no token is two rows' (the grids have room for `tokens` tokens, and outputs one writer).
__device__ __forceinline__ NewTokens new_tokens(const int32_t *starts, int row, int64_t tokens, int64_t most, int *floor)
{
    if (!starts) return NewTokens{row < tokens ? 1 : 0, row};
    const int64_t a = starts[row], b = starts[row + 1];
    if (a < 0 || b <= a || b > tokens || b - a > most) return NewTokens{0, 0};
    const bool apart = a >= *floor;
    *floor = max(*floor, (int)b);
    return apart ? NewTokens{(int)(b - a), a} : NewTokens{0, 0};
}
// Whether a row ends before it begins.  Where none does, no two rows overlap, and floors of 0 serve all.
__device__ __forceinline__ bool falls(const int32_t *starts, int row) { return starts && starts[row + 1] < starts[row]; }
// The floor of a thread's first row, r0, in a workgroup of WAVES waves whose threads have the rows one after another.
template <int WAVES>
__device__ __forceinline__ int floor_of(const int32_t *starts, int r0, int r1, int64_t tokens, int64_t most, int *lds /* [WAVES] */)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int end = 0;
    for (int r = r0; r < r1; ++r) new_tokens(starts, r, tokens, most, &end);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(end, o);
        if (lane >= o) end = max(end, u);
    }
    __syncthreads();   // (what is there is read)
    if (lane == 63) lds[wave] = end;
    int before = __shfl_up(end, 1);
    if (lane == 0) before = 0;
    __syncthreads();
    for (int w = 0; w < wave; ++w) before = max(before, lds[w]);
    __syncthreads();   // (it is the caller's again)
    return before;
}

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

}  // namespace fz
