// Internal launchers of the linear layers over tokens (host side, gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hatq {

constexpr int kMaxExperts = 1024;
constexpr int kMaxRows = 1 << 24;   // of one call: every block and tile index fits 31 bits

// n blocks over two grid dimensions (index y * gridDim.x + x): a dimension holds
// less than 2^32 threads.
inline dim3 grid_of(int64_t n) {
    const int64_t x = n < (1 << 20) ? n : 1 << 20;
    return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

// Tokens to codes: rows of cin elements of x_type (hatq_dtype), stride x_stride.
struct TokenArgs {
    const void *x;
    int8_t *xq;
    float *sx;
    int64_t x_stride;
    int32_t x_type;
    int32_t rows, cin, k_stride;
    int32_t log_b;      // transform block 2^log_b
    int32_t by16;       // codes: 0 by rows, 1 as 16 rows' matrix operands, [rows / 16][k_stride / 16][16][16]
};
hipError_t launch_token_quant(const TokenArgs &a, hipStream_t st);

// Weights into the kernels' order: from floats (codes == nullptr) or from codes.
struct LinearPrepArgs {
    const void *w;          // [experts][held][cin] of w_type
    const int8_t *codes;    // [experts][held][cin]
    const float *scale_in;  // with codes: [experts][held]
    const float *bias_in;   // [experts][held] or nullptr
    int8_t *wpack;
    float *w_scale, *bias;
    int32_t w_type;
    int32_t experts, cin, cout, gated, hblock, k_stride, cout_pad;
};
hipError_t launch_linear_prepare(const LinearPrepArgs &a, hipStream_t st);

// One product: rows of codes by the held channels.  Grouped: ends != nullptr.
struct LinearArgs {
    const int8_t *xq;
    const float *sx;
    const int8_t *wp;
    const float *w_scale, *bias;
    const int32_t *ends, *src;
    void *y;
    int64_t y_stride;
    int32_t y_type;
    int32_t rows, x_rows, experts;
    int32_t cout, cout_pad, k_stride;
    int32_t gated;
    float inv_b;
};
hipError_t launch_linear(const LinearArgs &a, hipStream_t st);

// The kernel that launch_linear takes: tiles of rows x packed columns, or the weights streamed
// past 16 or 32 rows by `waves` waves a group of channels.
enum { kTile32x64, kTile64x64, kTile64x128, kTile128x128, kTile128x256, kTile256x256, kStream16, kStream32 };
struct LinearChoice {
    int kernel, waves;
};
LinearChoice choose_linear(const LinearArgs &a);

// One layer's product of tokens that its own blocks quantize (xq and sx unused, no ends):
// for a few tokens (HATQ_TOKEN_ROWS, HATQ_TOKEN_CODES) and for small layers.
bool linear_takes_tokens(const LinearArgs &a);
struct TokenChoice {
    bool small;   // linear_small_kernel, else linear_token_kernel
    int ch;       // chunks of 8 elements a lane
};
TokenChoice choose_tokens(const LinearArgs &a);
hipError_t launch_linear_tokens(const LinearArgs &a, const TokenArgs &x, hipStream_t st);

struct OrderArgs {
    const int32_t *ids;
    int32_t *ends, *src, *pos, *ws;
    int32_t tokens, topk, experts;
};
size_t expert_order_ws_ints(int64_t pairs, int32_t experts);
hipError_t launch_expert_order(const OrderArgs &a, hipStream_t st);

// Both of an expert block's first steps, in one launch where they are small enough.
hipError_t launch_order_quant(const OrderArgs &o, const TokenArgs &a, hipStream_t st);

struct CombineArgs {
    const float *h;
    const int32_t *pos;
    const float *weights;
    void *y;
    int64_t h_stride, y_stride;
    int32_t y_type;
    int32_t h_rows, cols, tokens, topk;
};
hipError_t launch_expert_combine(const CombineArgs &a, hipStream_t st);

}  // namespace hatq
