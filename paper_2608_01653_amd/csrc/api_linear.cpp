// C-ABI entry points of the linear layers over tokens: host-side validation and
// launch order.  Every argument check runs before the first HIP call, so invalid
// calls launch nothing, touch no output and need no GPU.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/hatq.h"
#include "linear.h"

namespace {

constexpr int32_t kMaxWidth = 1 << 16;           // cin, held channels: 65536 * 127^2 < 2^31
constexpr int64_t kMaxBytes = (int64_t)1 << 46;  // of one tensor
constexpr int32_t kMaxCols = 1 << 30;            // of a weighted sum: column indices by fours fit 31 bits

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t align256(size_t v) { return (v + 255) & ~size_t(255); }
int32_t hip_status(hipError_t e) { return e == hipSuccess ? HATQ_OK : HATQ_EHIP; }
bool known_type(int32_t t) { return t == HATQ_F32 || t == HATQ_BF16 || t == HATQ_F16; }
int32_t type_size(int32_t t) { return t == HATQ_F32 ? 4 : 2; }

// log2 of a transform block the token kernels take, or -1.
int32_t log_block(int32_t b) {
    for (int32_t l = 0; l <= 7; ++l)
        if (b == 1 << l) return l;
    return -1;
}

// HATQ_OK, HATQ_EINVAL, or HATQ_EUNSUPPORTED for an order of the convolutions
// that the token kernels lack.
int32_t check_block(int32_t b, int32_t cin) {
    if (b == 192 || b == 320) return HATQ_EUNSUPPORTED;
    if (log_block(b) < 0) return HATQ_EINVAL;
    return cin % b == 0 ? HATQ_OK : HATQ_EUNSUPPORTED;
}

int32_t k_stride_of(int32_t cin) { return (cin + 63) / 64 * 64; }
int32_t cout_pad_of(int32_t cout, int32_t gated) { return (cout + 31) / 32 * 32 * (gated ? 2 : 1); }

int32_t check_shape(int32_t experts, int32_t cin, int32_t cout, int32_t gated, int32_t hblock) {
    if (experts <= 0 || cin <= 0 || cout <= 0 || (gated != 0 && gated != 1)) return HATQ_EINVAL;
    if (log_block(hblock) < 0 && hblock != 192 && hblock != 320) return HATQ_EINVAL;
    if (experts > hatq::kMaxExperts || cin > kMaxWidth || cout > kMaxWidth / (gated ? 2 : 1)) return HATQ_EUNSUPPORTED;
    return check_block(hblock, cin);
}

struct Places {
    size_t scale, bias, bytes;   // offsets into the buffer (codes first), its size
};
Places places(int32_t experts, int32_t cin, int32_t cout, int32_t gated) {
    const size_t cols = (size_t)experts * cout_pad_of(cout, gated);
    Places p;
    p.scale = align256(cols * k_stride_of(cin));
    p.bias = p.scale + align256(cols * 4);
    p.bytes = p.bias + align256(cols * 4);
    return p;
}

int32_t check_weights(const hatq_linear_weights *W) {
    if (!W) return HATQ_EINVAL;
    const int32_t s = check_shape(W->experts, W->cin, W->cout, W->gated, W->hblock);
    if (s != HATQ_OK) return s;
    if (W->k_stride != k_stride_of(W->cin) || W->cout_pad != cout_pad_of(W->cout, W->gated)) return HATQ_EINVAL;
    if (!W->wpack || !W->w_scale || !W->bias) return HATQ_EINVAL;
    if (!aligned(W->wpack, 16) || !aligned(W->w_scale, 16) || !aligned(W->bias, 16)) return HATQ_EINVAL;
    return HATQ_OK;
}

// A tensor of `rows` rows of `cols` elements of `type` at `stride`.
int32_t check_rows(const void *p, int32_t type, int32_t rows, int32_t cols, int64_t stride) {
    if (!p || !known_type(type) || stride < cols) return HATQ_EINVAL;
    if (!aligned(p, type_size(type))) return HATQ_EINVAL;
    if (stride > kMaxBytes / type_size(type) / rows) return HATQ_EINVAL;
    return HATQ_OK;
}

int32_t prepare(int32_t experts, int32_t cin, int32_t cout, int32_t gated, int32_t hblock, const void *w,
                int32_t w_type, const int8_t *codes, const float *scale, const float *bias, void *dst,
                size_t dst_bytes, hatq_linear_weights *out, void *stream) {
    const int32_t s = check_shape(experts, cin, cout, gated, hblock);
    if (s != HATQ_OK) return s;
    if (!dst || !out || !aligned(dst, 256)) return HATQ_EINVAL;
    if (codes ? (!scale || !aligned(scale, 4)) : (!w || !known_type(w_type) || !aligned(w, type_size(w_type))))
        return HATQ_EINVAL;
    if (bias && !aligned(bias, 4)) return HATQ_EINVAL;
    const Places p = places(experts, cin, cout, gated);
    if (dst_bytes < p.bytes) return HATQ_EWORKSPACE;
    int8_t *base = static_cast<int8_t *>(dst);
    hatq::LinearPrepArgs a{};
    a.w = w;
    a.codes = codes;
    a.scale_in = scale;
    a.bias_in = bias;
    a.wpack = base;
    a.w_scale = reinterpret_cast<float *>(base + p.scale);
    a.bias = reinterpret_cast<float *>(base + p.bias);
    a.w_type = w_type;
    a.experts = experts;
    a.cin = cin;
    a.cout = cout;
    a.gated = gated;
    a.hblock = hblock;
    a.k_stride = k_stride_of(cin);
    a.cout_pad = cout_pad_of(cout, gated);
    if (hatq::launch_linear_prepare(a, static_cast<hipStream_t>(stream)) != hipSuccess) return HATQ_EHIP;
    *out = {experts, cin, cout, gated, hblock, a.k_stride, a.cout_pad, a.wpack, a.w_scale, a.bias};
    return HATQ_OK;
}

// The checks of one product but for those of its rows' codes.
int32_t check_product(const hatq_linear_weights *W, bool grouped, const int32_t *ends, const int32_t *src,
                      int32_t rows, int32_t x_rows, const void *y, int32_t y_type, int64_t y_stride) {
    const int32_t s = check_weights(W);
    if (s != HATQ_OK) return s;
    if (rows < 0 || x_rows < 0) return HATQ_EINVAL;
    if (!grouped && W->experts != 1) return HATQ_EINVAL;
    if (rows > hatq::kMaxRows || x_rows > hatq::kMaxRows) return HATQ_EUNSUPPORTED;
    if (rows == 0) return HATQ_OK;
    if (grouped) {
        if (!ends || !aligned(ends, 4) || (src && !aligned(src, 4))) return HATQ_EINVAL;
        if (x_rows < 1 || (!src && x_rows < rows)) return HATQ_EINVAL;
    }
    return check_rows(y, y_type, rows, W->cout, y_stride);
}

hatq::LinearArgs product_args(const hatq_linear_weights *W, const int8_t *xq, const float *sx, int32_t x_rows,
                              const int32_t *ends, const int32_t *src, int32_t rows, void *y, int32_t y_type,
                              int64_t y_stride) {
    hatq::LinearArgs a{};
    a.xq = xq;
    a.sx = sx;
    a.wp = W->wpack;
    a.w_scale = W->w_scale;
    a.bias = W->bias;
    a.ends = ends;
    a.src = src;
    a.y = y;
    a.y_stride = y_stride;
    a.y_type = y_type;
    a.rows = rows;
    a.x_rows = x_rows;
    a.experts = W->experts;
    a.cout = W->cout;
    a.cout_pad = W->cout_pad;
    a.k_stride = W->k_stride;
    a.gated = W->gated;
    a.inv_b = 1.0f / (float)W->hblock;
    return a;
}

int32_t product(const hatq_linear_weights *W, const int8_t *xq, const float *sx, int32_t x_rows, const int32_t *ends,
                const int32_t *src, int32_t rows, void *y, int32_t y_type, int64_t y_stride, hipStream_t st) {
    return hip_status(hatq::launch_linear(
        product_args(W, xq, sx, x_rows, ends, src, rows, y, y_type, y_stride), st));
}

hatq::TokenArgs token_args(const hatq_linear_weights *W, const void *x, int32_t x_type, int32_t rows,
                           int64_t x_stride, int8_t *xq, float *sx) {
    hatq::TokenArgs a{};
    a.x = x;
    a.xq = xq;
    a.sx = sx;
    a.x_stride = x_stride;
    a.x_type = x_type;
    a.rows = rows;
    a.cin = W->cin;
    a.k_stride = W->k_stride;
    a.log_b = log_block(W->hblock);
    return a;
}

// One layer's calls that need no workspace: linear_takes_tokens takes all of them.
bool few_tokens(const hatq_linear_weights *W, int32_t rows) {
    return rows <= HATQ_TOKEN_ROWS && (int64_t)rows * W->k_stride <= HATQ_TOKEN_CODES;
}

// Floats in, after the checks.  ws: hatq_linear_ws_bytes(W, x_rows), not used for a few
// tokens of one layer.
int32_t enqueue(const hatq_linear_weights *W, const void *x, int32_t x_type, int32_t x_rows, int64_t x_stride,
                const int32_t *ends, const int32_t *src, int32_t rows, void *y, int32_t y_type, int64_t y_stride,
                void *ws, hipStream_t st) {
    int8_t *xq = static_cast<int8_t *>(ws);
    float *sx = reinterpret_cast<float *>(xq + align256((size_t)x_rows * W->k_stride));
    const hatq::TokenArgs t = token_args(W, x, x_type, x_rows, x_stride, xq, sx);
    const hatq::LinearArgs a = product_args(W, xq, sx, x_rows, ends, src, rows, y, y_type, y_stride);
    if (hatq::linear_takes_tokens(a)) return hip_status(hatq::launch_linear_tokens(a, t, st));
    if (!ws) return HATQ_EINVAL;
    if (hatq::launch_token_quant(t, st) != hipSuccess) return HATQ_EHIP;
    return hip_status(hatq::launch_linear(a, st));
}

int32_t forward(const hatq_linear_weights *W, bool grouped, const void *x, int32_t x_type, int32_t x_rows,
                int64_t x_stride, const int32_t *ends, const int32_t *src, int32_t rows, void *y, int32_t y_type,
                int64_t y_stride, void *ws, size_t ws_bytes, void *stream) {
    int32_t s = check_product(W, grouped, ends, src, rows, x_rows, y, y_type, y_stride);
    if (s != HATQ_OK || rows == 0) return s;
    if ((s = check_rows(x, x_type, x_rows, W->cin, x_stride)) != HATQ_OK) return s;
    if (grouped || !few_tokens(W, rows)) {
        if (!ws || !aligned(ws, 256)) return HATQ_EINVAL;
        if (ws_bytes < hatq_linear_ws_bytes(W, x_rows)) return HATQ_EWORKSPACE;
    }
    return enqueue(W, x, x_type, x_rows, x_stride, ends, src, rows, y, y_type, y_stride, ws,
                   static_cast<hipStream_t>(stream));
}

int32_t check_mlp(const hatq_linear_weights *W_in, const hatq_linear_weights *W_out) {
    int32_t s = check_weights(W_in);
    if (s == HATQ_OK) s = check_weights(W_out);
    if (s != HATQ_OK) return s;
    const bool fit = W_in->gated && !W_out->gated && W_in->experts == W_out->experts && W_in->cout == W_out->cin;
    return fit ? HATQ_OK : HATQ_EINVAL;
}

// hatq_expert_mlp's workspace: ends (at 0), src, pos, the order's own, hidden and output
// rows, and the codes of one layer at a time.  Where the hidden rows become codes before
// the second product starts, the output rows take their place (less memory, and lines
// that the memory-side cache still holds).  bytes = 0 for sizes that are not supported.
struct MlpPlaces {
    size_t src, pos, order, hidden, rows, scratch, bytes;
};
MlpPlaces mlp_places(const hatq_linear_weights *W_in, const hatq_linear_weights *W_out, int32_t tokens, int32_t topk) {
    MlpPlaces p{};
    const size_t order = hatq_expert_order_ws_bytes(tokens, topk, W_in->experts);
    if (order == 0 || tokens <= 0) return p;
    const int32_t pairs = tokens * topk;
    const size_t hidden = align256((size_t)pairs * W_in->cout * 4), rows = align256((size_t)pairs * W_out->cout * 4);
    static const int32_t grouped = 0;   // (any ends: the choice of kernels does not read them)
    const bool reads_hidden = hatq::linear_takes_tokens(
        product_args(W_out, nullptr, nullptr, pairs, &grouped, nullptr, pairs, nullptr, HATQ_F32, W_out->cout));
    p.src = align256((size_t)W_in->experts * 4);
    p.pos = p.src + align256((size_t)pairs * 4);
    p.order = p.pos + align256((size_t)pairs * 4);
    p.hidden = p.order + order;
    p.rows = reads_hidden ? p.hidden + hidden : p.hidden;
    p.scratch = p.rows + (reads_hidden || rows > hidden ? rows : hidden);
    const size_t in = hatq_linear_ws_bytes(W_in, tokens), out = hatq_linear_ws_bytes(W_out, pairs);
    p.bytes = p.scratch + (in > out ? in : out);
    return p;
}

}  // namespace

extern "C" {

size_t hatq_linear_weights_bytes(int32_t experts, int32_t cin, int32_t cout, int32_t gated, int32_t hblock) {
    if (check_shape(experts, cin, cout, gated, hblock) != HATQ_OK) return 0;
    return places(experts, cin, cout, gated).bytes;
}

int32_t hatq_prepare_linear(int32_t experts, int32_t cin, int32_t cout, int32_t gated, int32_t hblock, const void *w,
                            int32_t w_type, const float *bias, void *dst, size_t dst_bytes,
                            hatq_linear_weights *out, void *stream) {
    return prepare(experts, cin, cout, gated, hblock, w, w_type, nullptr, nullptr, bias, dst, dst_bytes, out, stream);
}

int32_t hatq_pack_linear(int32_t experts, int32_t cin, int32_t cout, int32_t gated, int32_t hblock,
                         const int8_t *codes, const float *w_scale, const float *bias, void *dst, size_t dst_bytes,
                         hatq_linear_weights *out, void *stream) {
    if (!codes) return HATQ_EINVAL;
    return prepare(experts, cin, cout, gated, hblock, nullptr, HATQ_F32, codes, w_scale, bias, dst, dst_bytes, out,
                   stream);
}

int32_t hatq_token_quant(const void *x, int32_t x_type, int32_t rows, int32_t cin, int64_t x_stride, int32_t hblock,
                         int8_t *xq, float *act_scale, void *stream) {
    if (rows < 0 || cin <= 0) return HATQ_EINVAL;
    int32_t s = check_block(hblock, cin);
    if (s != HATQ_OK) return s;
    if (cin > kMaxWidth || rows > hatq::kMaxRows) return HATQ_EUNSUPPORTED;
    if (rows == 0) return HATQ_OK;
    if ((s = check_rows(x, x_type, rows, cin, x_stride)) != HATQ_OK) return s;
    if (!xq || !act_scale || !aligned(xq, 16) || !aligned(act_scale, 4)) return HATQ_EINVAL;
    hatq_linear_weights W{};
    W.cin = cin;
    W.k_stride = k_stride_of(cin);
    W.hblock = hblock;
    return hip_status(hatq::launch_token_quant(token_args(&W, x, x_type, rows, x_stride, xq, act_scale),
                                               static_cast<hipStream_t>(stream)));
}

int32_t hatq_linear_int8(const hatq_linear_weights *W, const int8_t *xq, const float *act_scale, int32_t rows,
                         void *y, int32_t y_type, int64_t y_stride, void *stream) {
    const int32_t s = check_product(W, false, nullptr, nullptr, rows, rows, y, y_type, y_stride);
    if (s != HATQ_OK || rows == 0) return s;
    if (!xq || !act_scale || !aligned(xq, 16) || !aligned(act_scale, 4)) return HATQ_EINVAL;
    return product(W, xq, act_scale, rows, nullptr, nullptr, rows, y, y_type, y_stride,
                   static_cast<hipStream_t>(stream));
}

size_t hatq_linear_ws_bytes(const hatq_linear_weights *W, int32_t rows) {
    if (check_weights(W) != HATQ_OK || rows <= 0 || rows > hatq::kMaxRows) return 0;
    return align256((size_t)rows * W->k_stride) + align256((size_t)rows * 4);
}

int32_t hatq_linear_forward(const hatq_linear_weights *W, const void *x, int32_t x_type, int32_t rows,
                            int64_t x_stride, void *y, int32_t y_type, int64_t y_stride, void *ws, size_t ws_bytes,
                            void *stream) {
    return forward(W, false, x, x_type, rows, x_stride, nullptr, nullptr, rows, y, y_type, y_stride, ws, ws_bytes,
                   stream);
}

int32_t hatq_experts_int8(const hatq_linear_weights *W, const int8_t *xq, const float *act_scale, int32_t x_rows,
                          const int32_t *ends, const int32_t *src, int32_t rows, void *y, int32_t y_type,
                          int64_t y_stride, void *stream) {
    const int32_t s = check_product(W, true, ends, src, rows, x_rows, y, y_type, y_stride);
    if (s != HATQ_OK || rows == 0) return s;
    if (!xq || !act_scale || !aligned(xq, 16) || !aligned(act_scale, 4)) return HATQ_EINVAL;
    return product(W, xq, act_scale, x_rows, ends, src, rows, y, y_type, y_stride, static_cast<hipStream_t>(stream));
}

int32_t hatq_experts_forward(const hatq_linear_weights *W, const void *x, int32_t x_type, int32_t x_rows,
                             int64_t x_stride, const int32_t *ends, const int32_t *src, int32_t rows, void *y,
                             int32_t y_type, int64_t y_stride, void *ws, size_t ws_bytes, void *stream) {
    return forward(W, true, x, x_type, x_rows, x_stride, ends, src, rows, y, y_type, y_stride, ws, ws_bytes, stream);
}

size_t hatq_expert_order_ws_bytes(int32_t tokens, int32_t topk, int32_t experts) {
    if (tokens < 0 || topk <= 0 || experts <= 0 || experts > hatq::kMaxExperts) return 0;
    const int64_t pairs = (int64_t)tokens * topk;
    if (pairs > hatq::kMaxRows) return 0;
    return align256(hatq::expert_order_ws_ints(pairs, experts) * 4 + 1);
}

int32_t hatq_expert_order(const int32_t *ids, int32_t tokens, int32_t topk, int32_t experts, int32_t *ends,
                          int32_t *src, int32_t *pos, void *ws, size_t ws_bytes, void *stream) {
    if (tokens < 0 || topk <= 0 || experts <= 0) return HATQ_EINVAL;
    const size_t need = hatq_expert_order_ws_bytes(tokens, topk, experts);
    if (need == 0) return HATQ_EUNSUPPORTED;
    if (!ends || !aligned(ends, 4)) return HATQ_EINVAL;
    if (tokens > 0 && (!ids || !src || !pos || !aligned(ids, 4) || !aligned(src, 4) || !aligned(pos, 4)))
        return HATQ_EINVAL;
    if (!ws || !aligned(ws, 256)) return HATQ_EINVAL;
    if (ws_bytes < need) return HATQ_EWORKSPACE;
    const hatq::OrderArgs a{ids, ends, src, pos, static_cast<int32_t *>(ws), tokens, topk, experts};
    return hip_status(hatq::launch_expert_order(a, static_cast<hipStream_t>(stream)));
}

int32_t hatq_expert_combine(const float *h, int32_t h_rows, int32_t cols, int64_t h_stride, const int32_t *pos,
                            const float *weights, int32_t tokens, int32_t topk, void *y, int32_t y_type,
                            int64_t y_stride, void *stream) {
    if (h_rows < 0 || cols <= 0 || tokens < 0 || topk <= 0) return HATQ_EINVAL;
    if (cols > kMaxCols) return HATQ_EUNSUPPORTED;
    if (tokens == 0) return HATQ_OK;
    int32_t s;
    if ((s = check_rows(y, y_type, tokens, cols, y_stride)) != HATQ_OK) return s;
    if (h_rows > 0 && (s = check_rows(h, HATQ_F32, h_rows, cols, h_stride)) != HATQ_OK) return s;
    if (!pos || !weights || !aligned(pos, 4) || !aligned(weights, 4)) return HATQ_EINVAL;
    if (tokens > hatq::kMaxRows || h_rows > hatq::kMaxRows) return HATQ_EUNSUPPORTED;
    hatq::CombineArgs a{};
    a.h = h;
    a.pos = pos;
    a.weights = weights;
    a.y = y;
    a.h_stride = h_stride;
    a.y_stride = y_stride;
    a.y_type = y_type;
    a.h_rows = h_rows;
    a.cols = cols;
    a.tokens = tokens;
    a.topk = topk;
    return hip_status(hatq::launch_expert_combine(a, static_cast<hipStream_t>(stream)));
}

size_t hatq_expert_mlp_ws_bytes(const hatq_linear_weights *W_in, const hatq_linear_weights *W_out, int32_t tokens,
                                int32_t topk) {
    if (check_mlp(W_in, W_out) != HATQ_OK) return 0;
    const MlpPlaces p = mlp_places(W_in, W_out, tokens, topk);
    return p.bytes;
}

int32_t hatq_expert_mlp(const hatq_linear_weights *W_in, const hatq_linear_weights *W_out, const void *x,
                        int32_t x_type, int32_t tokens, int64_t x_stride, const int32_t *ids, const float *weights,
                        int32_t topk, void *y, int32_t y_type, int64_t y_stride, void *ws, size_t ws_bytes,
                        void *stream) {
    int32_t s = check_mlp(W_in, W_out);
    if (s != HATQ_OK) return s;
    if (tokens < 0 || topk <= 0) return HATQ_EINVAL;
    if (tokens == 0) return HATQ_OK;
    const MlpPlaces p = mlp_places(W_in, W_out, tokens, topk);
    if (p.bytes == 0) return HATQ_EUNSUPPORTED;
    if ((s = check_rows(x, x_type, tokens, W_in->cin, x_stride)) != HATQ_OK) return s;
    if ((s = check_rows(y, y_type, tokens, W_out->cout, y_stride)) != HATQ_OK) return s;
    if (!ids || !weights || !aligned(ids, 4) || !aligned(weights, 4)) return HATQ_EINVAL;
    if (!ws || !aligned(ws, 256)) return HATQ_EINVAL;
    if (ws_bytes < p.bytes) return HATQ_EWORKSPACE;
    int8_t *base = static_cast<int8_t *>(ws);
    int32_t *ends = reinterpret_cast<int32_t *>(base), *src = reinterpret_cast<int32_t *>(base + p.src),
            *pos = reinterpret_cast<int32_t *>(base + p.pos);
    float *hidden = reinterpret_cast<float *>(base + p.hidden), *rows = reinterpret_cast<float *>(base + p.rows);
    const int32_t pairs = tokens * topk;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const hatq::OrderArgs o{ids, ends, src, pos, reinterpret_cast<int32_t *>(base + p.order), tokens, topk,
                            W_in->experts};
    int8_t *xq = base + p.scratch;
    float *sx = reinterpret_cast<float *>(xq + align256((size_t)tokens * W_in->k_stride));
    const hatq::TokenArgs t = token_args(W_in, x, x_type, tokens, x_stride, xq, sx);
    if (hatq::launch_order_quant(o, t, st) != hipSuccess) return HATQ_EHIP;
    if ((s = product(W_in, xq, sx, tokens, ends, src, pairs, hidden, HATQ_F32, W_in->cout, st)) != HATQ_OK) return s;
    if ((s = enqueue(W_out, hidden, HATQ_F32, pairs, W_in->cout, ends, nullptr, pairs, rows, HATQ_F32, W_out->cout,
                     base + p.scratch, st)) != HATQ_OK)
        return s;
    const hatq::CombineArgs c{rows, pos, weights, y, W_out->cout, y_stride, y_type, pairs, W_out->cout, tokens, topk};
    return hip_status(hatq::launch_expert_combine(c, st));
}

}  // extern "C"
