// C-ABI entry points of the linear layers of 4-bit weights: host-side validation and launch
// order.  Every argument check runs before the first HIP call, so invalid calls launch
// nothing, touch no output and need no GPU.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/hatq.h"
#include "linear4.h"

namespace {

constexpr int32_t kMaxWidth = 1 << 16;           // cin, held channels
constexpr int64_t kMaxBytes = (int64_t)1 << 46;  // of one tensor

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t align256(size_t v) { return (v + 255) & ~size_t(255); }
bool known_type(int32_t t) { return t == HATQ_F32 || t == HATQ_BF16 || t == HATQ_F16; }
int32_t type_size(int32_t t) { return t == HATQ_F32 ? 4 : 2; }

// log2 of a transform block the token kernels take, or -1.
int32_t log_block(int32_t b) {
    for (int32_t l = 0; l <= 7; ++l)
        if (b == 1 << l) return l;
    return -1;
}

int32_t k_stride_of(int32_t cin) { return (cin + 127) / 128 * 128; }
int32_t cout_pad_of(int32_t cout, int32_t gated) { return (cout + 15) / 16 * 16 * (gated ? 2 : 1); }

int32_t check_shape(int32_t cin, int32_t cout, int32_t gated, int32_t hblock, int32_t group) {
    if (cin <= 0 || cout <= 0 || (gated != 0 && gated != 1) || (group != 64 && group != 128)) return HATQ_EINVAL;
    if (hblock == 192 || hblock == 320) return HATQ_EUNSUPPORTED;
    if (log_block(hblock) < 0) return HATQ_EINVAL;
    if (cin > kMaxWidth || cout > kMaxWidth / (gated ? 2 : 1) || cin % hblock != 0) return HATQ_EUNSUPPORTED;
    return HATQ_OK;
}

struct Places {
    size_t scale, bias, bytes;   // offsets into the buffer (codes first), its size
};
Places places(int32_t cin, int32_t cout, int32_t gated, int32_t group) {
    const size_t cols = (size_t)cout_pad_of(cout, gated), k = (size_t)k_stride_of(cin);
    Places p;
    p.scale = align256(cols * k / 2);
    p.bias = p.scale + align256(cols * (k / group) * 2);
    p.bytes = p.bias + align256(cols * 4);
    return p;
}

int32_t check_weights(const hatq_linear4_weights *W) {
    if (!W) return HATQ_EINVAL;
    const int32_t s = check_shape(W->cin, W->cout, W->gated, W->hblock, W->group);
    if (s != HATQ_OK) return s;
    if (W->k_stride != k_stride_of(W->cin) || W->cout_pad != cout_pad_of(W->cout, W->gated)) return HATQ_EINVAL;
    if (!W->wpack || !W->w_scale || !W->bias) return HATQ_EINVAL;
    if (!aligned(W->wpack, 16) || !aligned(W->w_scale, 16) || !aligned(W->bias, 16)) return HATQ_EINVAL;
    return HATQ_OK;
}

// A tensor of `rows` rows of `cols` elements of `type` at `stride`.
int32_t check_rows(const void *p, int32_t type, int32_t rows, int32_t cols, int64_t stride) {
    if (!p || !known_type(type) || stride < cols) return HATQ_EINVAL;
    if (!aligned(p, (uintptr_t)type_size(type))) return HATQ_EINVAL;
    if (stride > kMaxBytes / type_size(type) / rows) return HATQ_EINVAL;
    return HATQ_OK;
}

int32_t prepare(int32_t cin, int32_t cout, int32_t gated, int32_t hblock, int32_t group, const void *w, int32_t w_type,
                const int8_t *codes, const uint16_t *scale, const float *bias, void *dst, size_t dst_bytes,
                hatq_linear4_weights *out, void *stream) {
    const int32_t s = check_shape(cin, cout, gated, hblock, group);
    if (s != HATQ_OK) return s;
    if (!dst || !out || !aligned(dst, 256)) return HATQ_EINVAL;
    if (codes ? (!scale || !aligned(scale, 2))
              : (!w || !known_type(w_type) || !aligned(w, (uintptr_t)type_size(w_type))))
        return HATQ_EINVAL;
    if (bias && !aligned(bias, 4)) return HATQ_EINVAL;
    const Places p = places(cin, cout, gated, group);
    if (dst_bytes < p.bytes) return HATQ_EWORKSPACE;
    uint8_t *base = static_cast<uint8_t *>(dst);
    hatq::Linear4PrepArgs a{};
    a.w = w;
    a.codes = codes;
    a.scale_in = scale;
    a.bias_in = bias;
    a.wpack = base;
    a.w_scale = reinterpret_cast<uint16_t *>(base + p.scale);
    a.bias = reinterpret_cast<float *>(base + p.bias);
    a.w_type = w_type;
    a.cin = cin;
    a.cout = cout;
    a.gated = gated;
    a.hblock = hblock;
    a.group = group;
    a.k_stride = k_stride_of(cin);
    a.cout_pad = cout_pad_of(cout, gated);
    if (hatq::launch_linear4_prepare(a, static_cast<hipStream_t>(stream)) != hipSuccess) return HATQ_EHIP;
    *out = {cin, cout, gated, hblock, group, a.k_stride, a.cout_pad, a.wpack, a.w_scale, a.bias};
    return HATQ_OK;
}

// The codes of a call's tokens, 16 rows at a time.
size_t code_bytes(const hatq_linear4_weights *W, int32_t rows) { return align256(((size_t)rows + 15) / 16 * 16 * W->k_stride); }

}  // namespace

extern "C" {

size_t hatq_linear4_weights_bytes(int32_t cin, int32_t cout, int32_t gated, int32_t hblock, int32_t group) {
    if (check_shape(cin, cout, gated, hblock, group) != HATQ_OK) return 0;
    return places(cin, cout, gated, group).bytes;
}

int32_t hatq_prepare_linear4(int32_t cin, int32_t cout, int32_t gated, int32_t hblock, int32_t group, const void *w,
                             int32_t w_type, const float *bias, void *dst, size_t dst_bytes,
                             hatq_linear4_weights *out, void *stream) {
    return prepare(cin, cout, gated, hblock, group, w, w_type, nullptr, nullptr, bias, dst, dst_bytes, out, stream);
}

int32_t hatq_pack_linear4(int32_t cin, int32_t cout, int32_t gated, int32_t hblock, int32_t group,
                          const int8_t *codes, const uint16_t *w_scale, const float *bias, void *dst,
                          size_t dst_bytes, hatq_linear4_weights *out, void *stream) {
    if (!codes) return HATQ_EINVAL;
    return prepare(cin, cout, gated, hblock, group, nullptr, HATQ_F32, codes, w_scale, bias, dst, dst_bytes, out,
                   stream);
}

size_t hatq_linear4_ws_bytes(const hatq_linear4_weights *W, int32_t rows) {
    if (check_weights(W) != HATQ_OK || rows <= 0 || rows > hatq::kMaxRows) return 0;
    if (hatq::linear4_takes_tokens(rows, W->cout, W->gated, W->k_stride)) return 0;
    return code_bytes(W, rows) + align256((size_t)rows * 4);
}

int32_t hatq_linear4_forward(const hatq_linear4_weights *W, const void *x, int32_t x_type, int32_t rows,
                             int64_t x_stride, void *y, int32_t y_type, int64_t y_stride, void *ws, size_t ws_bytes,
                             void *stream) {
    int32_t s = check_weights(W);
    if (s != HATQ_OK) return s;
    if (rows < 0) return HATQ_EINVAL;
    if (rows > hatq::kMaxRows) return HATQ_EUNSUPPORTED;
    if (rows == 0) return HATQ_OK;
    if ((s = check_rows(y, y_type, rows, W->cout, y_stride)) != HATQ_OK) return s;
    if ((s = check_rows(x, x_type, rows, W->cin, x_stride)) != HATQ_OK) return s;
    const bool tokens = hatq::linear4_takes_tokens(rows, W->cout, W->gated, W->k_stride);
    if (!tokens) {
        if (!ws || !aligned(ws, 256)) return HATQ_EINVAL;
        if (ws_bytes < hatq_linear4_ws_bytes(W, rows)) return HATQ_EWORKSPACE;
    }
    hatq::TokenArgs t{};
    t.x = x;
    t.xq = static_cast<int8_t *>(ws);
    t.sx = tokens ? nullptr : reinterpret_cast<float *>(t.xq + code_bytes(W, rows));
    t.x_stride = x_stride;
    t.x_type = x_type;
    t.rows = rows;
    t.cin = W->cin;
    t.k_stride = W->k_stride;
    t.log_b = log_block(W->hblock);
    t.by16 = 1;
    hatq::Linear4Args a{};
    a.xq = t.xq;
    a.sx = t.sx;
    a.wp = W->wpack;
    a.w_scale = W->w_scale;
    a.bias = W->bias;
    a.y = y;
    a.y_stride = y_stride;
    a.y_type = y_type;
    a.rows = rows;
    a.cout = W->cout;
    a.k_stride = W->k_stride;
    a.gated = W->gated;
    a.group = W->group;
    a.inv_b = 1.0f / (float)W->hblock;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (tokens) return hatq::launch_linear4_tokens(a, t, st) == hipSuccess ? HATQ_OK : HATQ_EHIP;
    if (hatq::launch_token_quant(t, st) != hipSuccess) return HATQ_EHIP;
    return hatq::launch_linear4(a, st) == hipSuccess ? HATQ_OK : HATQ_EHIP;
}

}  // extern "C"
