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
};
struct RotateArgs {
    RotateTensor t[kMostTensors];
    int num, pairs, dim, interleaved;
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

// Sine and cosine of 2 pi x for |x| <= 1/2 turns, sign and factor applied by the caller.
__device__ __forceinline__ void turn(const RotateArgs &p, int64_t token, int i, float *c, float *s)
{
    constexpr double kTurn = 0.15915494309189533577;   // 1 / (2 pi)
    const double x = (double)p.positions[token] * p.frequencies[i] * kTurn;
    const float r = (float)(x - rint(x));              // whole turns taken off in fp64: what is left is as exact as the angle itself
    sincospif(2.f * r, s, c);
    *c *= p.factor;
    *s *= p.factor * p.sign;
}

// A workgroup takes a token: its sines and cosines once, for the heads of every tensor.
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs p)
{
    extern __shared__ float table[];   // [pairs] cosines, [pairs] sines
    for (int64_t token = blockIdx.x; token < p.tokens; token += gridDim.x) {
        __syncthreads();
        for (int i = threadIdx.x; i < p.pairs; i += 256) turn(p, token, i, &table[i], &table[p.pairs + i]);
        __syncthreads();
        for (int k = 0; k < p.num; ++k) {
            const RotateTensor &t = p.t[k];
            const int items = p.dim - p.pairs;   // of a head: pairs, then elements that are copied
            for (int j = threadIdx.x; j < t.heads * items; j += 256) {
                const int head = j / items, i = j - head * items;
                const int64_t src = token * t.src_token + head * t.src_head, dst = token * t.dst_token + head * t.dst_head;
                if (i < p.pairs) {
                    const int a = p.interleaved ? 2 * i : i, b = p.interleaved ? a + 1 : i + p.pairs;
                    const float x = load_value(t.src, src + a, t.bf16), y = load_value(t.src, src + b, t.bf16), c = table[i], s = table[p.pairs + i];
                    store_value(t.dst, dst + a, t.bf16, x * c - y * s);
                    store_value(t.dst, dst + b, t.bf16, x * s + y * c);
                } else if (t.src != t.dst) {
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
        (num > 0 && !heads) || !(factor > -3.0e38f && factor < 3.0e38f))
        return FREEZE_EINVAL;
    RotateArgs a{};
    Region e[2 * kMostTensors + 2];
    int n = 0;
    for (int i = 0; i < num; ++i) {
        const freeze_heads &h = heads[i];
        if ((h.dtype != FREEZE_F32 && h.dtype != FREEZE_BF16) || h.heads < 0 || h.heads > 65536) return FREEZE_EINVAL;
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
                         h.heads > 1 ? h.dst_head_stride : 0, h.heads, h.dtype == FREEZE_BF16};
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
    a.dim = (int)head_dim;
    a.interleaved = interleaved != 0;
    a.tokens = tokens;
    a.positions = positions;
    a.frequencies = frequencies;
    a.factor = factor;
    a.sign = inverse ? -1.f : 1.f;
    const unsigned grid = (unsigned)std::min<int64_t>(tokens, 1 << 16);
    hipLaunchKernelGGL(rotate_kernel, dim3(grid), dim3(256), (size_t)pairs * 8, static_cast<hipStream_t>(stream), a);
    return hipGetLastError() == hipSuccess ? FREEZE_OK : FREEZE_EHIP;
}

}  // extern "C"
