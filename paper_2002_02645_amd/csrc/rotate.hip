// Rotary positions (gfx950 / CDNA4).
#include "../../include/freeze.h"
#include "pages.h"

namespace fz {

namespace {

constexpr int kMostTensors = 8;
struct RotateTensor {
    const void *src;
    void *dst;
    int64_t src_token, src_head, dst_token, dst_head;
    int heads, bf16;
    int per_head;        // items of a head: of a piece or two of them, or of a pair or an element that is copied
    int piece;           // bytes: 16, 8, 4; 0: by elements
};
struct RotateArgs {
    RotateTensor t[kMostTensors];
    int num, pairs, interleaved;
    int each;            // tokens of a workgroup
    int64_t tokens;
    const int32_t *positions;
    const double *frequencies;
    float factor, sign;
};

__device__ __forceinline__ float load_value(const void *p, int64_t i, int bf16)
{
    return bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[i] << 16) : static_cast<const float *>(p)[i];
}
__device__ __forceinline__ void store_value(void *p, int64_t i, int bf16, float x)
{
    if (bf16) static_cast<uint16_t *>(p)[i] = bf16_rne(x);
    else static_cast<float *>(p)[i] = x;
}

// Factor times sine and cosine of a token's angle.
__device__ __forceinline__ float2 turn(const RotateArgs &p, int64_t token, int i)
{
    constexpr double kTurn = 0.15915494309189533577;   // 1 / (2 pi)
    const double x = (double)p.positions[token] * p.frequencies[i] * kTurn;
    const float r = (float)(x - rint(x));              // whole turns taken off in fp64: what is left is as exact as the angle itself
    float s, c;
    sincospif(2.f * r, &s, &c);
    return float2{c * p.factor, s * p.factor * p.sign};
}

// a and b turned by w (cosine, sine): one rounding of a product and of a sum each, the same in every form of the kernel
__device__ __forceinline__ float turned_a(float a, float b, float2 w) { return fmaf(a, w.x, -(b * w.y)); }
__device__ __forceinline__ float turned_b(float a, float b, float2 w) { return fmaf(b, w.x, a * w.y); }

// A piece of W words as its V values and back
template <int W>
using Words = __attribute__((ext_vector_type(W))) uint32_t;
template <int V, int W>
__device__ __forceinline__ void open_up(Words<W> w, float (&x)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = __uint_as_float(V == W ? w[e] : e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
}
template <int V, int W>
__device__ __forceinline__ Words<W> close_up(const float (&x)[V])
{
    Words<W> w;
#pragma unroll
    for (int e = 0; e < W; ++e) {
        if constexpr (V == W) w[e] = __float_as_uint(x[e]);
        else w[e] = (uint32_t)bf16_rne(x[2 * e]) | (uint32_t)bf16_rne(x[2 * e + 1]) << 16;
    }
    return w;
}

// An item of a head in pieces of V values, W words: V / 2 pairs side by side; V pairs, half a turned part apart; or a piece that is copied.
template <int V, int W>
__device__ __forceinline__ void rotate_pieces(const RotateArgs &p, const void *from, int64_t src_at, void *to, int64_t dst_at, const float2 *table, int i)
{
    const Words<W> *src = reinterpret_cast<const Words<W> *>(static_cast<const uint8_t *>(from) + src_at * (4 * W / V));
    Words<W> *dst = reinterpret_cast<Words<W> *>(static_cast<uint8_t *>(to) + dst_at * (4 * W / V));
    const int pieces = p.pairs / V;   // of one half of the turned part
    if (p.interleaved) {
        Words<W> w = src[i];
        if (i * V < 2 * p.pairs) {
            float x[V], y[V];
            open_up<V, W>(w, x);
#pragma unroll
            for (int e = 0; e < V / 2; ++e) {
                const float2 a = table[i * (V / 2) + e];
                y[2 * e] = turned_a(x[2 * e], x[2 * e + 1], a);
                y[2 * e + 1] = turned_b(x[2 * e], x[2 * e + 1], a);
            }
            w = close_up<V, W>(y);
        }
        dst[i] = w;
        return;
    }
    if (i >= pieces) {
        dst[i + pieces] = src[i + pieces];
        return;
    }
    float a[V], b[V], x[V], y[V];
    open_up<V, W>(src[i], a);
    open_up<V, W>(src[i + pieces], b);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float2 w = table[i * V + e];
        x[e] = turned_a(a[e], b[e], w);
        y[e] = turned_b(a[e], b[e], w);
    }
    dst[i] = close_up<V, W>(x);
    dst[i + pieces] = close_up<V, W>(y);
}

// A workgroup takes some tokens (and, of few tokens, a part of their heads: blockIdx.y): their sines and cosines once, for the heads of every tensor.
// Bound by memory: 32,768 tokens of 40 heads of 128 bf16 (671 MB read and written) 128 us, 5.2 TB/s (400 by pairs); 16 tokens 5.0 us.
// fp32: 265 us for twice the bytes, 5.1 TB/s.
// Heads that are no whole pieces of 16 bytes go by the widest that fit: 40 M elements of bf16 (160 MB), halves apart, 28 us in pieces of 16 (heads of 128), 32 in 8 (of 72;
// 79 by elements), 47 in 4 (of 100; 77), 81 by elements (of 66, whose halves are odd), which what an item costs to find bounds.
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs p)
{
    extern __shared__ float2 table[];   // [each][pairs]
    for (int64_t first = (int64_t)blockIdx.x * p.each; first < p.tokens; first += (int64_t)gridDim.x * p.each) {
        const int here = (int)min((int64_t)p.each, p.tokens - first);
        __syncthreads();
        for (int j = threadIdx.x; j < here * p.pairs; j += 256) {
            const int token = j / p.pairs;
            table[j] = turn(p, first + token, j - token * p.pairs);
        }
        __syncthreads();
        for (int k = 0; k < p.num; ++k) {
            const RotateTensor &t = p.t[k];
            const int per_token = t.heads * t.per_head;
            for (int j = blockIdx.y * 256 + threadIdx.x; j < here * per_token; j += 256 * gridDim.y) {
                const int token = j / per_token, rest = j - token * per_token, head = rest / t.per_head, i = rest - head * t.per_head;
                const int64_t src = (first + token) * t.src_token + head * t.src_head, dst = (first + token) * t.dst_token + head * t.dst_head;
                const float2 *w = table + token * p.pairs;
                if (t.piece == 16) {
                    if (t.bf16) rotate_pieces<8, 4>(p, t.src, src, t.dst, dst, w, i);
                    else rotate_pieces<4, 4>(p, t.src, src, t.dst, dst, w, i);
                } else if (t.piece == 8) {
                    if (t.bf16) rotate_pieces<4, 2>(p, t.src, src, t.dst, dst, w, i);
                    else rotate_pieces<2, 2>(p, t.src, src, t.dst, dst, w, i);
                } else if (t.piece == 4) {
                    rotate_pieces<2, 1>(p, t.src, src, t.dst, dst, w, i);
                } else if (i < p.pairs) {
                    const int a = p.interleaved ? 2 * i : i, b = p.interleaved ? a + 1 : i + p.pairs;
                    const float x = load_value(t.src, src + a, t.bf16), y = load_value(t.src, src + b, t.bf16);
                    store_value(t.dst, dst + a, t.bf16, turned_a(x, y, w[i]));
                    store_value(t.dst, dst + b, t.bf16, turned_b(x, y, w[i]));
                } else {
                    const int e = i + p.pairs;
                    if (t.bf16) static_cast<uint16_t *>(t.dst)[dst + e] = static_cast<const uint16_t *>(t.src)[src + e];
                    else static_cast<uint32_t *>(t.dst)[dst + e] = static_cast<const uint32_t *>(t.src)[src + e];
                }
            }
        }
    }
}

// Bytes that a tensor takes up: pieces of `row` bytes, `stride` bytes from one to the next (0: one piece).
struct Region {
    uintptr_t begin, end, row, stride;
    bool dst;
};
// Whether two share a byte, as far as their extents say; of two that lie side by side in the rows of one buffer, whether their pieces do.
bool share_a_byte(const Region &a, const Region &b)
{
    if (a.end <= b.begin || b.end <= a.begin) return false;
    if (a.stride == 0 || a.stride != b.stride || a.row > a.stride || b.row > b.stride) return true;
    const uintptr_t from = a.begin <= b.begin ? (b.begin - a.begin) % a.stride : (a.stride - (a.begin - b.begin) % a.stride) % a.stride;   // of b in a's rows
    return from < a.row || a.stride - from < b.row;
}

}  // namespace
}  // namespace fz

using namespace fz;

extern "C" {

int freeze_rotate_positions(const freeze_heads *heads, int num, int64_t tokens, int64_t head_dim, const int32_t *positions,
                            const double *frequencies, int64_t pairs, int interleaved, float factor, int inverse, void *stream)
{
    if (num < 0 || num > kMostTensors || tokens < 0 || tokens >= (int64_t)1 << 31 || head_dim < 1 || head_dim > 4096 || pairs < 0 || 2 * pairs > head_dim ||
        (num > 0 && !heads) || !(factor >= -3.0e38f && factor <= 3.0e38f))
        return FREEZE_EINVAL;
    RotateArgs a{};
    Region e[2 * kMostTensors + 2];
    int n = 0;
    double items = 0;
    for (int i = 0; i < num; ++i) {
        const freeze_heads &h = heads[i];
        if ((h.dtype != FREEZE_F32 && h.dtype != FREEZE_BF16) || h.heads < 0 || h.heads > 8192) return FREEZE_EINVAL;
        if (tokens == 0 || h.heads == 0) continue;
        const uintptr_t size = h.dtype == FREEZE_F32 ? 4 : 2, src = reinterpret_cast<uintptr_t>(h.src), dst = reinterpret_cast<uintptr_t>(h.dst);
        int64_t ss, ds;
        if (!h.src || !h.dst || src % size != 0 || dst % size != 0 || !heads_span(tokens, h.heads, head_dim, h.src_token_stride, h.src_head_stride, false, &ss) ||
            !heads_span(tokens, h.heads, head_dim, h.dst_token_stride, h.dst_head_stride, true, &ds))
            return FREEZE_EINVAL;
        const bool in_place = src == dst && (tokens == 1 || h.src_token_stride == h.dst_token_stride) && (h.heads == 1 || h.src_head_stride == h.dst_head_stride);
        auto add = [&](uintptr_t at, int64_t span, int64_t token_stride, int64_t head_stride, bool written) {
            e[n++] = Region{at, at + (uintptr_t)span * size, (uintptr_t)((h.heads - 1) * head_stride + head_dim) * size,
                            tokens > 1 ? (uintptr_t)token_stride * size : 0, written};
        };
        if (!in_place) add(src, ss, h.src_token_stride, h.src_head_stride, false);
        add(dst, ds, h.dst_token_stride, h.dst_head_stride, true);
        RotateTensor &t = a.t[a.num++];
        t = RotateTensor{h.src, h.dst, tokens > 1 ? h.src_token_stride : 0, h.heads > 1 ? h.src_head_stride : 0, tokens > 1 ? h.dst_token_stride : 0,
                         h.heads > 1 ? h.dst_head_stride : 0, h.heads, h.dtype == FREEZE_BF16, 0, 0};
        // the widest pieces that are whole: of the turned part (of either half), of what is copied, from head to head and token to token
        const int64_t turned = interleaved ? 2 * pairs : pairs;
        for (int bytes = 16; bytes > (int)size && t.piece == 0; bytes /= 2)
            if (src % bytes == 0 && dst % bytes == 0 && (t.src_token | t.src_head | t.dst_token | t.dst_head | turned | head_dim) % (bytes / (int64_t)size) == 0) t.piece = bytes;
        t.per_head = (int)(t.piece ? (head_dim - (interleaved ? 0 : pairs)) * (int64_t)size / t.piece : head_dim - pairs);
        items += (double)tokens * t.heads * t.per_head;
    }
    if (a.num == 0) return FREEZE_OK;
    const uintptr_t pb = reinterpret_cast<uintptr_t>(positions), fb = reinterpret_cast<uintptr_t>(frequencies);
    if ((pairs > 0 && (!positions || !frequencies)) || pb % 4 != 0 || fb % 8 != 0) return FREEZE_EINVAL;
    if (positions) e[n++] = Region{pb, pb + (size_t)tokens * 4, 0, 0, false};
    if (frequencies) e[n++] = Region{fb, fb + (size_t)pairs * 8, 0, 0, false};
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if ((e[i].dst || e[j].dst) && share_a_byte(e[i], e[j])) return FREEZE_EINVAL;
    a.pairs = (int)pairs;
    a.interleaved = interleaved != 0;
    a.tokens = tokens;
    a.positions = positions;
    a.frequencies = frequencies;
    a.factor = factor;
    a.sign = inverse ? -1.f : 1.f;
    // Eight tokens a workgroup where that leaves 2,048 of them, and their sines fit; few tokens' heads over several.
    a.each = (int)std::max<int64_t>(1, std::min<int64_t>({8, tokens / 2048, pairs > 0 ? 4096 / pairs : 8}));
    const int64_t groups = (tokens + a.each - 1) / a.each;
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>({512 / groups, (int64_t)(items / (double)groups / 256), 64}));
    hipLaunchKernelGGL(rotate_kernel, dim3((unsigned)std::min<int64_t>(groups, 1 << 16), (unsigned)parts), dim3(256), (size_t)pairs * a.each * 8,
                       static_cast<hipStream_t>(stream), a);
    return hipGetLastError() == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

}  // extern "C"
