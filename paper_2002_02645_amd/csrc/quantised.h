// Rows held in 8 bits and the dense layer on them: what the host dispatcher and the kernels share.  Not part of the C ABI.
#pragma once
#include "freeze_internal.h"

namespace fz {

constexpr int kQuantBlock = 128;             // values that share an exponent: one k-step of the product
constexpr int64_t kQuantMaxD = 1 << 22;      // a tile of 256 rows spans 32-bit offsets

inline int64_t quant_code_stride(int64_t d) { return (d + kQuantBlock - 1) / kQuantBlock * kQuantBlock; }
inline int64_t quant_scale_stride(int64_t d) { return ((d + kQuantBlock - 1) / kQuantBlock + 3) / 4 * 4; }

// x [rows, d] (dtype: FREEZE_F32 or FREEZE_BF16) -> codes, scales
hipError_t launch_quantise_rows(const void *x, int dtype, int64_t rows, int64_t d, int64_t row_stride, uint8_t *codes,
                                uint8_t *scales, hipStream_t s);
// codes and scales as given -> the same with zeros behind d
hipError_t launch_copy_codes(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, uint8_t *out_codes, uint8_t *out_scales,
                             hipStream_t s);

struct QuantProduct {
    const uint8_t *x, *xs;   // [b, d_pad], [b, sd]
    const uint8_t *w, *ws;   // [m, d_pad], [m, sd]
    const float *bias;       // [m] or null
    void *out;               // [b, m], rows out_stride elements apart
    int64_t out_stride;
    int64_t b, m, d_pad, sd;
    int out_bf16, relu;
    int vec;                 // four outputs of a row from a multiple of four on are one aligned store
    float *part;             // plan's floats of scratch (none: null)
    // the plan's
    int64_t len;             // k-steps of a workgroup's range of the flattened (tile, k-step) space
    int nk, x_tiles, w_tiles, slots, xcd_share;
};
// How a product is cut.
struct QuantPlan {
    int variant;        // of quant_gemm_kernel
    int bm, bn;         // rows of x, rows of w of a tile
    int x_tiles, w_tiles, nk, slots, wgs;
    int64_t len;
    size_t part;        // floats of the sums of cut tiles
};
QuantPlan plan_quant_product(int64_t b, int64_t m, int64_t d_pad, bool out_bf16, int num_cus);
hipError_t launch_quant_product(const QuantPlan &pl, QuantProduct p, hipStream_t s);

}  // namespace fz
