// How attention over a 4-bit cache is laid out: host code without a launch, from sizes alone.
#include "cache4.h"

namespace hatq {

AttentionPlan plan_attention(int32_t batch, int32_t rows, int32_t heads, int32_t share, int32_t dim, int64_t max_len,
                             bool ragged, int32_t window) {
    const int64_t cols = (int64_t)rows * share;
    AttentionPlan p{};
    const auto tiles = [&](int64_t by) {
        return ragged ? cols / by + (batch < rows ? batch : rows) : batch * ((cols / batch + by - 1) / by);
    };
    // Wide blocks for more than one narrow one's columns, where they fill the card twice.  (us, 8
    // heads of 128 channels, bf16, wide and not: 64 sequences of 2048, 16 columns each 68 and
    // 42, 24 73 and 77, 48 73 and 102, 64 125 and 131, 128 175 and 240; 4 heads, 4 sequences of
    // 4096, too few blocks, 128 columns 66 and 31, 512 70 and 63; 8192 columns 492 and 747, heads
    // of 192 channels 696 and 1239, of 64 303 and 463; of 256, whose two tiles do not fit the
    // registers, 1846 and 1571.)
    p.cols = wide_cols(dim);
    p.tiles = tiles(p.cols);
    p.waves = 4;
    p.splits = 1;
    if (p.cols > 16 && cols / batch > 16 && p.tiles * heads >= 512) return p;
    p.cols = 16;
    p.tiles = tiles(16);
    // Parts of a sequence while there is not a block for each CU, of at least two steps of 32
    // positions a wave; 8 waves a block, 16 where each of them has four steps and no other
    // block would share its CU (at 16 to 64 steps 16 are behind: 1 token of 4 sequences of 1024 15.6
    // us for 14.4), fewer where a sequence is shorter.  (us a call in a graph, 8
    // heads of 128 channels, bf16: 1 sequence of 8192 in 8 parts 18.2, in 16 16.2, in 32 16.6;
    // 8 of 4096 in 1 part 26, in 4 20.8, in 8 22.1; 32 of 921 to 4096 whole, 8 waves 35.6, 16
    // 33.6, in 2 parts 34.7; 2 of 131072, 4 heads, fp16, 32 parts, 8 waves 48.3, 16 46.8; 1 of
    // 300, 64 channels, 4 waves 8.3, 8 7.9, 16 8.9.)
    int64_t most = max_len;
    const int64_t seen = (int64_t)window + rows / batch;
    if (window > 0 && seen < most) most = seen;
    const int64_t steps = (most + 31) / 32, base = p.tiles * heads;
    int64_t splits = 256 / base;
    if (splits > steps / 16) splits = steps / 16;
    p.splits = splits < 1 ? 1 : (int32_t)splits;
    p.waves = 8;
    if (dim <= 128 && base * p.splits <= 256 && steps / p.splits >= 64) p.waves = 16;
    while (p.waves > 1 && p.waves / 2 >= steps) p.waves /= 2;
    return p;
}

}  // namespace hatq
