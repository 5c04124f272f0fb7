// Rows held in 8 bits (e4m3 codes, a power of two for each block of 128 values) and the dense layer on them
// (gfx950 / CDNA4).
//
//     y[r, c] = act(bias[c] + sum_B 2^(Ex[r, B] + Ew[c, B]) sum_{i in B} x8[r, i] w8[c, i])
#include "../../include/freeze.h"
#include "quantised.h"

namespace fz {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

namespace {

// The exponent of a block from the bits of its largest magnitude 1.f * 2^(E - 127): 448 = 1.75 * 2^8, so 2^(E - 135),
// or twice that where 1.f is above 1.75; not below 2^-126, so that both the factor and its inverse are normal numbers.
__device__ __forceinline__ int block_exponent(uint32_t amax_bits)
{
    const int e = (int)(amax_bits >> 23) - 135 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -126 ? -126 : e;
}

// Eight values a thread, sixteen threads a block of 128.  VEC: rows start on 16-byte boundaries (bases and strides).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quantise_rows_kernel(const T *x, int64_t rows, int64_t d, int64_t row_stride, int64_t d_pad,
                                                            int64_t sd, uint8_t *codes, uint8_t *scales)
{
    const int64_t per_row = d_pad / 8, total = rows * per_row;   // a multiple of 16: a block's threads go on together
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t r = t / per_row, c = (t - r * per_row) * 8;
        const T *src = x + r * row_stride + c;
        float v[8];
        if (VEC && c + 8 <= d) {
            if constexpr (sizeof(T) == 4) {
                const f32x4 a = reinterpret_cast<const f32x4 *>(src)[0], b = reinterpret_cast<const f32x4 *>(src)[1];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = a[e];
                    v[4 + e] = b[e];
                }
            } else {
                const u32x4 a = *reinterpret_cast<const u32x4 *>(src);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[2 * e] = __uint_as_float(a[e] << 16);
                    v[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = 0.f;
                if (c + e < d) {
                    if constexpr (sizeof(T) == 4) v[e] = src[e];
                    else v[e] = __uint_as_float((uint32_t)src[e] << 16);
                }
            }
        }
        uint32_t amax = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = __float_as_uint(v[e]) & 0x7fffffffu;
            amax = u > amax ? u : amax;
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
            const uint32_t u = (uint32_t)__shfl_xor((int)amax, o, 16);
            amax = u > amax ? u : amax;
        }
        const int ex = block_exponent(amax);
        const float inv = __uint_as_float((uint32_t)(127 - ex) << 23);
        int w0 = 0, w1 = 0;
        w0 = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, w0, false);
        w0 = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, w0, true);
        w1 = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, w1, false);
        w1 = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, w1, true);
        *reinterpret_cast<u32x2 *>(codes + r * d_pad + c) = u32x2{(uint32_t)w0, (uint32_t)w1};
        if ((c & 127) == 0) {
            const int64_t b = c >> 7;
            scales[r * sd + b] = (uint8_t)(ex + 127);
            if (c + 128 == d_pad)
                for (int64_t q = b + 1; q < sd; ++q) scales[r * sd + q] = 1;
        }
    }
}

__global__ __launch_bounds__(256) void copy_codes_kernel(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, int64_t d_pad,
                                                         int64_t sd, uint8_t *out_codes, uint8_t *out_scales)
{
    const int64_t per_row = d_pad / 16, total = rows * per_row;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t r = t / per_row, c = (t - r * per_row) * 16;
        u32x4 v = *reinterpret_cast<const u32x4 *>(codes + r * d_pad + c);
        if (c + 16 > d) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t left = d - (c + 4 * e);   // codes of this word
                v[e] = left >= 4 ? v[e] : (left <= 0 ? 0u : v[e] & ((1u << (8 * (int)left)) - 1u));
            }
        }
        *reinterpret_cast<u32x4 *>(out_codes + r * d_pad + c) = v;
        if ((c & 127) == 0) {
            const int64_t b = c >> 7;
            out_scales[r * sd + b] = scales[r * sd + b];
            if (c + 128 == d_pad)
                for (int64_t q = b + 1; q < sd; ++q) out_scales[r * sd + q] = 1;
        }
    }
}

// the four code bytes of a word, times 2^(exponent of s): two words of bf16 pairs (exact)
__device__ __forceinline__ void widen(uint32_t codes, float s, uint32_t &lo, uint32_t &hi)
{
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes, s, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes, s, true));
}

// A wave forms 16 x 16 outputs straight from memory.
__global__ __launch_bounds__(256) void quant_product_kernel(QuantProduct p)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c0 = ((int64_t)blockIdx.x * 4 + wave) * 16, r0 = (int64_t)blockIdx.y * 16;
    if (c0 >= p.m) return;
    const int64_t wr = c0 + (lane & 15) < p.m ? c0 + (lane & 15) : p.m - 1, xr = r0 + (lane & 15) < p.b ? r0 + (lane & 15) : p.b - 1;
    const uint8_t *w = p.w + wr * p.d_pad + (lane >> 4) * 32, *x = p.x + xr * p.d_pad + (lane >> 4) * 32;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int64_t k = 0; k < p.d_pad; k += kQuantBlock) {
        const float sw = __uint_as_float((uint32_t)p.ws[wr * p.sd + k / kQuantBlock] << 23);
        const float sx = __uint_as_float((uint32_t)p.xs[xr * p.sd + k / kQuantBlock] << 23);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x4 a = *reinterpret_cast<const u32x4 *>(w + k + h * 16), b = *reinterpret_cast<const u32x4 *>(x + k + h * 16);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                uint32_t aw[4], bw[4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    widen(a[2 * q + e], sw, aw[2 * e], aw[2 * e + 1]);
                    widen(b[2 * q + e], sx, bw[2 * e], bw[2 * e + 1]);
                }
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{aw[0], aw[1], aw[2], aw[3]}),
                                                              __builtin_bit_cast(bf16x8, u32x4{bw[0], bw[1], bw[2], bw[3]}), acc, 0, 0, 0);
            }
        }
    }
    const int64_t row = r0 + (lane & 15), col = c0 + (lane >> 4) * 4;
    if (row >= p.b) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (col + e >= p.m) break;
        float v = acc[e] + (p.bias ? p.bias[col + e] : 0.f);
        if (p.relu) v = __builtin_fmaxf(v, 0.f);
        if (p.out_bf16) static_cast<uint16_t *>(p.out)[row * p.out_stride + col + e] = bf16_rne(v);
        else static_cast<float *>(p.out)[row * p.out_stride + col + e] = v;
    }
}

unsigned blocks_for(int64_t threads)
{
    const int64_t n = (threads + 255) / 256;
    return (unsigned)(n < 65536 ? n : 65536);
}

}  // namespace

hipError_t launch_quantise_rows(const void *x, int dtype, int64_t rows, int64_t d, int64_t row_stride, uint8_t *codes,
                                uint8_t *scales, hipStream_t s)
{
    if (rows <= 0) return hipSuccess;
    const int64_t d_pad = quant_code_stride(d), sd = quant_scale_stride(d);
    const dim3 grid(blocks_for(rows * (d_pad / 8))), block(256);
    const int64_t size = dtype == FREEZE_F32 ? 4 : 2;
    const bool vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && row_stride * size % 16 == 0;
    if (dtype == FREEZE_F32) {
        auto k = vec ? quantise_rows_kernel<float, true> : quantise_rows_kernel<float, false>;
        hipLaunchKernelGGL(k, grid, block, 0, s, static_cast<const float *>(x), rows, d, row_stride, d_pad, sd, codes, scales);
    } else {
        auto k = vec ? quantise_rows_kernel<uint16_t, true> : quantise_rows_kernel<uint16_t, false>;
        hipLaunchKernelGGL(k, grid, block, 0, s, static_cast<const uint16_t *>(x), rows, d, row_stride, d_pad, sd, codes, scales);
    }
    return hipGetLastError();
}

hipError_t launch_copy_codes(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, uint8_t *out_codes, uint8_t *out_scales,
                             hipStream_t s)
{
    const int64_t d_pad = quant_code_stride(d), sd = quant_scale_stride(d);
    hipLaunchKernelGGL(copy_codes_kernel, dim3(blocks_for(rows * (d_pad / 16))), dim3(256), 0, s, codes, scales, rows, d, d_pad, sd,
                       out_codes, out_scales);
    return hipGetLastError();
}

hipError_t launch_quant_product(const QuantProduct &p, hipStream_t s)
{
    // rows in slices that a grid's second axis holds
    constexpr int64_t kSlice = 65535 * 16;
    for (int64_t r = 0; r < p.b; r += kSlice) {
        QuantProduct q = p;
        q.b = p.b - r < kSlice ? p.b - r : kSlice;
        q.x = p.x + r * p.d_pad;
        q.xs = p.xs + r * p.sd;
        q.out = static_cast<uint8_t *>(p.out) + r * p.out_stride * (p.out_bf16 ? 2 : 4);
        hipLaunchKernelGGL(quant_product_kernel, dim3((unsigned)((p.m + 63) / 64), (unsigned)((q.b + 15) / 16)), dim3(256), 0, s, q);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace fz
