// C-ABI entry points of the 4-bit cache and the attention over it: host-side validation and
// launch order.  Every argument check runs before the first HIP call, so invalid calls
// launch nothing, touch no output and need no GPU.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/hatq.h"
#include "cache4.h"

namespace {

constexpr int32_t kMaxRows = 1 << 24;
constexpr int32_t kMaxHeads = 1024;
constexpr int64_t kMaxPositions = (int64_t)1 << 30;     // of a sequence
constexpr int64_t kMaxBytes = (int64_t)1 << 46;         // of one tensor

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t align256(size_t v) { return (v + 255) & ~size_t(255); }
int32_t hip_status(hipError_t e) { return e == hipSuccess ? HATQ_OK : HATQ_EHIP; }

int32_t log2_of(int32_t v) {
    for (int32_t l = 0; l <= 30; ++l)
        if (v == 1 << l) return l;
    return -1;
}

int32_t check_shape(int32_t pages, int32_t page_size, int32_t heads, int32_t dim, int32_t hblock) {
    if (pages <= 0 || heads <= 0 || dim <= 0) return HATQ_EINVAL;
    const int32_t page = log2_of(page_size), block = log2_of(hblock);
    if (page < 4 || page > 16) return HATQ_EINVAL;
    if (hblock == 192 || hblock == 320) return HATQ_EUNSUPPORTED;
    if (block < 0 || block > 7) return HATQ_EINVAL;
    if (heads > kMaxHeads || dim > 256 || dim % hblock != 0 || (int64_t)pages * page_size > INT32_MAX)
        return HATQ_EUNSUPPORTED;
    return HATQ_OK;
}

int32_t check_cache(const hatq_cache4 *C) {
    if (!C) return HATQ_EINVAL;
    const int32_t s = check_shape(C->pages, C->page_size, C->heads, C->dim, C->hblock);
    if (s != HATQ_OK) return s;
    return C->buf && aligned(C->buf, 256) ? HATQ_OK : HATQ_EINVAL;
}

hatq::Cache4 cache_of(const hatq_cache4 *C) {
    return {static_cast<uint8_t *>(C->buf), C->pages, log2_of(C->page_size), C->heads, C->dim, log2_of(C->hblock)};
}

// Sizes of the rows' places, without the pointers.
int32_t check_sizes(const hatq_cache4 *C, int32_t rows, int32_t width, int32_t batch, bool ragged) {
    if (rows < 0 || width <= 0 || batch <= 0) return HATQ_EINVAL;
    if (!ragged && rows % batch != 0) return HATQ_EINVAL;
    if (rows > kMaxRows || batch > kMaxRows || (int64_t)width * C->page_size > kMaxPositions) return HATQ_EUNSUPPORTED;
    return HATQ_OK;
}

int32_t check_places(const int32_t *table, const int32_t *lens, const int32_t *ends) {
    if (!table || !lens || !aligned(table, 4) || !aligned(lens, 4) || !aligned(ends, 4)) return HATQ_EINVAL;
    return HATQ_OK;
}

// A tensor [rows][heads][dim].  out: its heads may not overlap.
int32_t check_heads(const hatq_heads *x, int32_t rows, int32_t heads, int32_t dim, bool out) {
    if (!x || !x->p || x->type < HATQ_F32 || x->type > HATQ_F16) return HATQ_EINVAL;
    const int64_t size = x->type == HATQ_F32 ? 4 : 2;
    if (!aligned(x->p, (uintptr_t)size) || x->row_stride < 0 || x->head_stride < 0) return HATQ_EINVAL;
    if (x->row_stride > kMaxBytes / size / rows || x->head_stride > kMaxBytes / size / heads) return HATQ_EINVAL;
    if (out) {
        // rows of heads, or heads of rows
        const bool by_row = x->head_stride >= dim && x->row_stride >= (heads - 1) * x->head_stride + dim;
        const bool by_head = x->row_stride >= dim && x->head_stride >= (rows - 1) * x->row_stride + dim;
        if (!(by_row || by_head || (rows == 1 && x->head_stride >= dim) || (heads == 1 && x->row_stride >= dim) ||
              (rows == 1 && heads == 1)))
            return HATQ_EINVAL;
    }
    return HATQ_OK;
}

hatq::Heads4 heads_of(const hatq_heads *x) { return {x->p, x->row_stride, x->head_stride, x->type}; }

int32_t cache_call(const hatq_cache4 *C, const hatq_heads *k, const hatq_heads *v, int32_t rows, const int32_t *table,
                   int32_t width, const int32_t *lens, const int32_t *ends, int32_t batch, bool out,
                   hipError_t (*launch)(const hatq::CacheArgs &, hipStream_t), void *stream) {
    int32_t s = check_cache(C);
    if (s == HATQ_OK) s = check_sizes(C, rows, width, batch, ends != nullptr);
    if (s != HATQ_OK || rows == 0) return s;
    if ((s = check_places(table, lens, ends)) != HATQ_OK) return s;
    if ((s = check_heads(k, rows, C->heads, C->dim, out)) != HATQ_OK) return s;
    if ((s = check_heads(v, rows, C->heads, C->dim, out)) != HATQ_OK) return s;
    const hatq::CacheArgs a = {cache_of(C), {table, lens, ends, width, batch, rows}, {heads_of(k), heads_of(v)}};
    return hip_status(launch(a, static_cast<hipStream_t>(stream)));
}

// The checks of an attention's sizes, and its layout.
int32_t check_attention(const hatq_cache4 *C, int32_t rows, int32_t q_heads, int32_t width, int32_t batch, bool ragged,
                        int32_t window, int32_t max_len, hatq::AttentionPlan *p) {
    int32_t s = check_cache(C);
    if (s == HATQ_OK) s = check_sizes(C, rows, width, batch, ragged);
    if (s != HATQ_OK) return s;
    if (q_heads <= 0 || q_heads % C->heads != 0 || max_len < 0 || window < 0) return HATQ_EINVAL;
    if (q_heads > kMaxHeads * 16 || (int64_t)rows * q_heads > INT32_MAX / 2) return HATQ_EUNSUPPORTED;
    if (rows == 0) return HATQ_OK;
    const int64_t most = (int64_t)width * C->page_size;
    *p = hatq::plan_attention(batch, rows, C->heads, q_heads / C->heads, C->dim,
                              max_len > 0 && max_len < most ? max_len : most, ragged, window);
    return HATQ_OK;
}

size_t attention_bytes(const hatq_cache4 *C, const hatq::AttentionPlan &p) {
    return p.splits > 1 ? align256((size_t)p.tiles * C->heads * p.splits * hatq::partial4_bytes(C->dim)) : 0;
}

}  // namespace

extern "C" {

size_t hatq_cache4_bytes(int32_t pages, int32_t page_size, int32_t heads, int32_t dim, int32_t hblock) {
    if (check_shape(pages, page_size, heads, dim, hblock) != HATQ_OK) return 0;
    return (size_t)pages * heads * page_size * ((dim + 63) / 64) * 68;
}

int32_t hatq_cache4_init(int32_t pages, int32_t page_size, int32_t heads, int32_t dim, int32_t hblock, void *buf,
                         size_t bytes, hatq_cache4 *out) {
    const int32_t s = check_shape(pages, page_size, heads, dim, hblock);
    if (s != HATQ_OK) return s;
    if (!out || !buf || !aligned(buf, 256)) return HATQ_EINVAL;
    if (bytes < hatq_cache4_bytes(pages, page_size, heads, dim, hblock)) return HATQ_EWORKSPACE;
    *out = {pages, page_size, heads, dim, hblock, buf};
    return HATQ_OK;
}

int32_t hatq_cache4_append(const hatq_cache4 *C, const hatq_heads *k, const hatq_heads *v, int32_t rows,
                           const int32_t *table, int32_t width, const int32_t *lens, const int32_t *ends,
                           int32_t batch, void *stream) {
    return cache_call(C, k, v, rows, table, width, lens, ends, batch, false, hatq::launch_cache4_append, stream);
}

int32_t hatq_cache4_read(const hatq_cache4 *C, const hatq_heads *k, const hatq_heads *v, int32_t rows,
                         const int32_t *table, int32_t width, const int32_t *lens, const int32_t *ends,
                         int32_t batch, void *stream) {
    return cache_call(C, k, v, rows, table, width, lens, ends, batch, true, hatq::launch_cache4_read, stream);
}

size_t hatq_attention4_ws_bytes(const hatq_cache4 *C, int32_t rows, int32_t q_heads, int32_t width, int32_t batch,
                                int32_t ragged, int32_t window, int32_t max_len) {
    hatq::AttentionPlan p{};
    if (check_attention(C, rows, q_heads, width, batch, ragged != 0, window, max_len, &p) != HATQ_OK || rows == 0) return 0;
    return attention_bytes(C, p);
}

int32_t hatq_attention4(const hatq_cache4 *C, const hatq_heads *q, const hatq_heads *y, int32_t rows, int32_t q_heads,
                        const int32_t *table, int32_t width, const int32_t *lens, const int32_t *ends, int32_t batch,
                        float scale, int32_t causal, int32_t window, int32_t max_len, void *ws, size_t ws_bytes,
                        void *stream) {
    hatq::AttentionPlan p{};
    int32_t s = check_attention(C, rows, q_heads, width, batch, ends != nullptr, window, max_len, &p);
    if (s != HATQ_OK) return s;
    if ((causal != 0 && causal != 1) || (window > 0 && !causal) || !std::isfinite(scale)) return HATQ_EINVAL;
    if (rows == 0) return HATQ_OK;
    if ((s = check_places(table, lens, ends)) != HATQ_OK) return s;
    if ((s = check_heads(q, rows, q_heads, C->dim, false)) != HATQ_OK) return s;
    if ((s = check_heads(y, rows, q_heads, C->dim, true)) != HATQ_OK) return s;
    if (const size_t need = attention_bytes(C, p)) {
        if (!ws || !aligned(ws, 256)) return HATQ_EINVAL;
        if (ws_bytes < need) return HATQ_EWORKSPACE;
    }
    hatq::AttentionArgs a{};
    a.c = cache_of(C);
    a.at = {table, lens, ends, width, batch, rows};
    a.q = heads_of(q);
    a.y = heads_of(y);
    a.share = q_heads / C->heads;
    a.causal = causal;
    a.window = window;
    a.scale = scale;
    a.splits = p.splits;
    a.ws = ws;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    switch ((C->dim + 63) / 64) {
        case 1: return hip_status(hatq::launch_attention4_1(a, p, st));
        case 2: return hip_status(hatq::launch_attention4_2(a, p, st));
        case 3: return hip_status(hatq::launch_attention4_3(a, p, st));
        default: return hip_status(hatq::launch_attention4_4(a, p, st));
    }
}

}  // extern "C"
