// Rows held in 8 bits (gfx950 / CDNA4): e4m3 codes and a power of two for each block of 128 values.
#include "../../include/freeze.h"
#include "quantised.h"

namespace fz {

namespace {

// Sixteen values a thread (four loads of 16 bytes in fp32, two in bf16, one store), eight threads a block of 128.  Bound by memory:
// 10,000 x 8,192 fp32 71 - 74 us, 5.5 - 5.8 TB/s read and written.  (A run of memory to each load, a block to 32 lanes: 74, 71 past the
// caches; in bf16, 16 lanes, 20.4 us against 19.2 for 4,096 x 8,192.)  VEC: rows start on 16-byte boundaries (bases and strides).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quantise_rows_kernel(const T *x, int64_t rows, int64_t d, int64_t row_stride, QuantRows out)
{
    constexpr int V = 16 / (int)sizeof(T);
    const int64_t per_row = out.d_pad / 16, total = rows * per_row;   // a multiple of 8: a block's threads go on together
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t r = t / per_row, c = (t - r * per_row) * 16;
        const T *src = x + r * row_stride + c;
        float v[16];
        if (VEC && c + 16 <= d) {
            sixteen_of(src, v);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                v[e] = 0.f;
                if (c + e < d) {
                    if constexpr (V == 4) v[e] = src[e];
                    else v[e] = __uint_as_float((uint32_t)src[e] << 16);
                }
            }
        }
        int ex;
        const u32x4 codes = codes_of(v, &ex);
        *reinterpret_cast<u32x4 *>(out.codes + out.code_at(r, c >> 4)) = codes;
        if ((c & 127) == 0) {
            const int64_t b = c >> 7;
            out.scales[out.scale_at(r, b)] = (uint8_t)(ex + 127);
            if (c + 128 == out.d_pad)
                for (int64_t q = b + 1; q < out.sd; ++q) out.scales[out.scale_at(r, q)] = 1;
        }
    }
}

__global__ __launch_bounds__(256) void tile_codes_kernel(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, QuantRows out)
{
    const int64_t per_row = out.d_pad / 16, total = rows * per_row;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t r = t / per_row, chunk = t - r * per_row, c = chunk * 16;
        u32x4 v = *reinterpret_cast<const u32x4 *>(codes + r * out.d_pad + c);
        if (c + 16 > d) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t left = d - (c + 4 * e);   // codes of this word
                v[e] = left >= 4 ? v[e] : (left <= 0 ? 0u : v[e] & ((1u << (8 * (int)left)) - 1u));
            }
        }
        *reinterpret_cast<u32x4 *>(out.codes + out.code_at(r, chunk)) = v;
        if ((c & 127) == 0) {
            const int64_t b = c >> 7;
            out.scales[out.scale_at(r, b)] = scales[r * out.sd + b];
            if (c + 128 == out.d_pad)
                for (int64_t q = b + 1; q < out.sd; ++q) out.scales[out.scale_at(r, q)] = 1;
        }
    }
}

unsigned blocks_for(int64_t threads)
{
    const int64_t n = (threads + 255) / 256;
    return (unsigned)(n < 65536 ? n : 65536);
}

}  // namespace

hipError_t launch_quantise_rows(const void *x, int dtype, int64_t rows, int64_t d, int64_t row_stride, const QuantRows &out, hipStream_t s)
{
    if (rows <= 0) return hipSuccess;
    const dim3 grid(blocks_for(rows * (out.d_pad / 16))), block(256);
    const int64_t size = dtype == FREEZE_F32 ? 4 : 2;
    const bool vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && row_stride * size % 16 == 0;
    if (dtype == FREEZE_F32) {
        auto k = vec ? quantise_rows_kernel<float, true> : quantise_rows_kernel<float, false>;
        hipLaunchKernelGGL(k, grid, block, 0, s, static_cast<const float *>(x), rows, d, row_stride, out);
    } else {
        auto k = vec ? quantise_rows_kernel<uint16_t, true> : quantise_rows_kernel<uint16_t, false>;
        hipLaunchKernelGGL(k, grid, block, 0, s, static_cast<const uint16_t *>(x), rows, d, row_stride, out);
    }
    return hipGetLastError();
}

hipError_t launch_tile_codes(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, const QuantRows &out, hipStream_t s)
{
    hipLaunchKernelGGL(tile_codes_kernel, dim3(blocks_for(rows * (out.d_pad / 16))), dim3(256), 0, s, codes, scales, rows, d, out);
    return hipGetLastError();
}

}  // namespace fz
