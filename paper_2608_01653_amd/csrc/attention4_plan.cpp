// How attention over a 4-bit cache is laid out: host code without a launch, from sizes alone.
#include "cache4.h"

namespace hatq {

AttentionPlan plan_attention(int32_t batch, int32_t rows, int32_t heads, int32_t share, int32_t dim, int64_t max_len,
                             bool ragged) {
    const int64_t cols = (int64_t)rows * share;
    AttentionPlan p{};
    // a sequence's columns on average
    const bool many = cols / batch >= 128;
    p.cols = many ? wide_cols(dim) : 16;
    p.tiles = ragged ? cols / p.cols + (batch < rows ? batch : rows) : batch * ((cols / batch + p.cols - 1) / p.cols);
    p.waves = dim <= 128 && !many ? 8 : 4;
    p.splits = 1;
    if (many) return p;
    // blocks that fill the card, of at least two steps of 32 positions a wave
    const int64_t steps = (max_len + 31) / 32, base = p.tiles * heads;
    int64_t splits = 512 / base;
    if (splits > steps / (2 * p.waves)) splits = steps / (2 * p.waves);
    p.splits = splits < 1 ? 1 : (int32_t)splits;
    return p;
}

}  // namespace hatq
