// Rows held in 8 bits and the dense layer on them: what the host dispatcher and the kernels share.  Not part of the C ABI.
#pragma once
#include "freeze_internal.h"
#include "quant_plan.h"

namespace fz {

constexpr int64_t kL2Bytes = 32 << 20;       // of the eight XCDs together
constexpr int64_t kQuantMaxD = 1 << 22;      // 2^31 rows of it stay within 64 bits of bytes

inline int64_t quant_code_stride(int64_t d) { return (d + kQuantBlock - 1) / kQuantBlock * kQuantBlock; }
inline int64_t quant_scale_stride(int64_t d) { return ((d + kQuantBlock - 1) / kQuantBlock + 3) / 4 * 4; }

// Quantised rows as the product reads them: tiles of `tile` rows (kQuantTile, or fewer for a small batch), in a tile k-step by k-step
// (128 codes), so that a stage of the product is one run of memory; of a row's 128 bytes, chunk c (16 bytes) lies at
// c ^ row128_swizzle(row), as in LDS.  The scale bytes of four k-steps lie together, 4 bytes a row.  Rows behind the last one are
// whatever they were: they meet outputs that are not stored.
struct QuantRows {
    uint8_t *codes, *scales;
    int64_t d_pad, sd;      // bytes of a row
    int tile;               // rows of a tile; 0: row after row (the layout of freeze_quantise_rows)
    __host__ __device__ int64_t code_at(int64_t r, int64_t chunk) const   // chunk: 16 codes
    {
        if (tile == 0) return r * d_pad + chunk * 16;
        const int64_t t = (uint32_t)r / (uint32_t)tile;   // (at most 2^31 rows)
        const int in = (int)(r - t * tile);
        return t * tile * d_pad + ((chunk >> 3) * tile + in) * 128 + (((int)chunk & 7) ^ row128_swizzle(in)) * 16;
    }
    __host__ __device__ int64_t scale_at(int64_t r, int64_t block) const
    {
        if (tile == 0) return r * sd + block;
        const int64_t t = (uint32_t)r / (uint32_t)tile;
        const int in = (int)(r - t * tile);
        return t * tile * sd + ((block >> 2) * tile + in) * 4 + (block & 3);
    }
};

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// The exponent of a block from the bits of its largest magnitude 1.f * 2^(E - 127): 448 = 1.75 * 2^8, so 2^(E - 135),
// or twice that where 1.f is above 1.75; not below 2^-126, so that both the factor and its inverse are normal numbers.
__device__ __forceinline__ int block_exponent(uint32_t amax_bits)
{
    const int e = (int)(amax_bits >> 23) - 135 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -126 ? -126 : e;
}

// sixteen values from a 16-byte boundary on
__device__ __forceinline__ void sixteen_of(const float *src, float (&v)[16])
{
    u32x4 w[4];
#pragma unroll
    for (int l = 0; l < 4; ++l) w[l] = reinterpret_cast<const u32x4 *>(src)[l];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(w[e / 4][e % 4]);
}
__device__ __forceinline__ void sixteen_of(const uint16_t *src, float (&v)[16])
{
    u32x4 w[2];
#pragma unroll
    for (int l = 0; l < 2; ++l) w[l] = reinterpret_cast<const u32x4 *>(src)[l];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(e % 2 ? w[e / 8][e % 8 / 2] & 0xffff0000u : w[e / 8][e % 8 / 2] << 16);
}

// codes of sixteen values; eight neighbouring lanes hold a block
__device__ __forceinline__ u32x4 codes_of(const float (&v)[16], int *exponent)
{
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint32_t u = __float_as_uint(v[e]) & 0x7fffffffu;
        amax = u > amax ? u : amax;
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
        const uint32_t u = (uint32_t)__shfl_xor((int)amax, o, 8);
        amax = u > amax ? u : amax;
    }
    const int ex = block_exponent(amax);
    *exponent = ex;
    const float inv = __uint_as_float((uint32_t)(127 - ex) << 23);
    u32x4 codes;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        int q = 0;
        q = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * w] * inv, v[4 * w + 1] * inv, q, false);
        q = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * w + 2] * inv, v[4 * w + 3] * inv, q, true);
        codes[w] = (uint32_t)q;
    }
    return codes;
}

// x [rows, d] (dtype: FREEZE_F32 or FREEZE_BF16) -> codes, scales
hipError_t launch_quantise_rows(const void *x, int dtype, int64_t rows, int64_t d, int64_t row_stride, const QuantRows &out, hipStream_t s);
// codes and scales row after row -> out, zeros behind d
hipError_t launch_tile_codes(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, const QuantRows &out, hipStream_t s);

struct QuantProduct {
    const uint8_t *x, *xs;   // b rows in tiles of the plan's bm
    const uint8_t *w, *ws;   // m rows in tiles of kQuantTile
    const float *bias;       // [m] or null
    void *out;               // [b, m], rows out_stride elements apart
    int64_t out_stride;
    int64_t b, m, d_pad, sd;
    int out_bf16, relu;
    int vec;                 // 1: four outputs of a row from a multiple of four on are one aligned store; 2: and eight bf16 are
    int w_once;              // the weights are read by one workgroup each, and more than L2 holds
    const void *raw;         // few rows straight from the caller's values (x, xs: not used); null: none
    int raw_bf16;
    int64_t raw_stride, d;
    float *part;             // plan's floats of scratch (none: null)
    int nk, x_tiles, w_tiles, splits;   // the plan's
};
// whether the product quantises its b rows itself
bool quant_takes_values(const QuantPlan &pl, const void *x, int dtype, int64_t b, int64_t d, int64_t row_stride);
hipError_t launch_quant_product(const QuantPlan &pl, QuantProduct p, hipStream_t s);

}  // namespace fz
