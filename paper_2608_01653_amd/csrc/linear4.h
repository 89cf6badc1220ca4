// Internal launchers of the linear layers of 4-bit weights (host side, gfx950).
#pragma once

#include "linear.h"

namespace hatq {

// Weights into the kernels' order: from floats (codes == nullptr) or from codes.
struct Linear4PrepArgs {
    const void *w;              // [held][cin] of w_type
    const int8_t *codes;        // [held][cin]
    const uint16_t *scale_in;   // with codes: bf16 [held][groups]
    const float *bias_in;       // [held] or nullptr
    uint8_t *wpack;
    uint16_t *w_scale;
    float *bias;
    int32_t w_type;
    int32_t cin, cout, gated, hblock, group, k_stride, cout_pad;
};
hipError_t launch_linear4_prepare(const Linear4PrepArgs &a, hipStream_t st);

struct Linear4Args {
    const int8_t *xq;           // [rows][k_stride]
    const float *sx;
    const uint8_t *wp;
    const uint16_t *w_scale;
    const float *bias;
    void *y;
    int64_t y_stride;
    int32_t y_type;
    int32_t rows, cout, k_stride;
    int32_t gated, group;
    float inv_b;
};
// Tokens that the product's blocks quantize themselves, with no workspace (xq and sx unused).
bool linear4_takes_tokens(int32_t rows, int32_t cout, int32_t gated, int32_t k_stride);
hipError_t launch_linear4_tokens(const Linear4Args &a, const TokenArgs &x, hipStream_t st);
// Codes and scales from memory.
hipError_t launch_linear4(const Linear4Args &a, hipStream_t st);

}  // namespace hatq
