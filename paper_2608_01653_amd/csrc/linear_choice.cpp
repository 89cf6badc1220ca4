// Which kernel a linear product takes: host code without a launch, from sizes alone.
#include "../../include/hatq.h"
#include "linear.h"

namespace hatq {
namespace {

// Row tiles that are met: groups fill half of their last tile on average.
double met_tiles(const LinearArgs &a, int bm) {
    if (!a.ends) return (a.rows + bm - 1) / bm;
    const double groups = a.experts < a.rows ? a.experts : a.rows, t = (double)a.rows / bm + 0.5 * groups;
    return t > groups ? t : groups;
}

}  // namespace

// The small kernel reads the weights again for every 16 rows, quantizes rows once for each
// range of columns and writes runs of 16 channels: it wins while rows and columns are few,
// fitted as rows cout^1.5.  (us, two kernels and one.  bf16: 128 -> 32, 8192 rows 9.2 and
// 6.2; 512 -> 256, 4096 rows 10.4 and 7.7; 1024 -> 256, 16384 rows 22.9 and 22.3; 512 ->
// 704, 8192 rows 17.6 and 14.8; 512 -> 2048, 800 rows 9.2 and 8.5, 1500 rows 10.8 and
// 13.2; 2048 -> 256, 300 rows 9.6 and 10.0, 1500 rows 12.4 and 10.4, 2500 rows 16.8 and
// 19.1.)  By expert, while a tile of 16 rows is mostly all that an expert has.  (Float32:
// 32 experts of 512 -> 1024, 96 rows 8.1 and 6.0, 384 rows 10.0 and 7.3, 768 rows 10.4 and
// 11.5; 64 of 2048 -> 1024, 48 rows 16.2 and 14.2, 768 rows 30.8 and 29.5, 1536 rows 32.1
// and 48.9; 8 of 320 -> 320, 1536 rows 8.7 and 7.4.)  The ends are on the device, so the rule
// has to hold for any: rows that meet in one expert read its weights again for every 16.  Up
// to 8 an expert that is the better of the two all the same, from 9 on only while the product
// is small.  (bf16, rows even / by Zipf's law / all in one expert: 64 of 2048 -> 8192, 512
// rows 272 / 262 / 129 and 226 / 199 / 46, 576 rows 215 / 203 / 28 and 229 / 210 / 47, 768
// rows 216 / 206 / 28 and 211 / 240 / 55; 256 of 2048 -> 8192, 3072 rows 806 / 760 / 98 and
// 811 / 943 / 174; 256 of 1024 -> 4096, 2304 rows 215 / 196 / 34 and 207 / 251 / 56; below the
// limit 64 of 2048 -> 4096, 768 rows 117 / 118 / 19 and 103 / 127 / 32.)
bool linear_takes_tokens(const LinearArgs &a) {
    if (!a.ends && a.rows <= HATQ_TOKEN_ROWS && (int64_t)a.rows * a.k_stride <= HATQ_TOKEN_CODES) return true;
    if (a.k_stride > 2048) return false;
    const double rows = a.rows, cols = a.cout_pad;
    if (a.ends) {
        if (met_tiles(a, 16) * 16.0 * a.k_stride * cols <= 4e8 || a.rows <= 8 * (int64_t)a.experts) return true;
        return a.rows <= 12 * (int64_t)a.experts && rows * a.k_stride * cols <= 8e9;
    }
    if (a.k_stride > 1024) return rows >= 500 && rows * cols <= 4e5;
    return rows * rows * cols * cols * cols <= 7e7 * 7e7;
}

// The kernel of a call that linear_takes_tokens takes, and a lane's chunks of 8 elements: a
// wave a row and 2048 elements at most (small), or all eight waves a row.
TokenChoice choose_tokens(const LinearArgs &a) {
    if (a.k_stride <= 512) return {true, 1};
    if (a.k_stride <= 1024) return {true, 2};
    if (a.k_stride <= 2048 && (a.ends || (int64_t)a.rows * a.k_stride > HATQ_TOKEN_CODES || a.rows > HATQ_TOKEN_ROWS))
        return {true, 4};
    return {false, a.k_stride <= 4096 ? 1 : a.k_stride <= 8192 ? 2 : 4};
}

namespace {

// Estimates in microseconds, fitted to measurements of all the kernels at 2110 drawn sizes:
// contractions 100 to 9000, outputs 16 to 9000, 17 to 40000 rows, 1 to 64 experts (MI355X).
// Over these the kernel chosen is 1 % behind the fastest of them on average, and more
// than 10 % behind at 4 % of the sizes.  The bytes of the outputs are not in it.  Past 64
// experts it was not fitted, and streams too long: 256 experts of 2048 -> 8192, 2048 rows
// streamed 1410 us with their codes, 2304 rows in tiles 795.
struct TileCost {
    int bm, bn;
    double fixed, step;   // of a launch; a step of 64 bytes of the contraction, latency
    int slots;            // tiles that the card holds at once
    double rate;          // TOP/s with the card full
};
constexpr TileCost kTiles[] = {   // (kTile32x64 to kTile256x256)
    {32, 64, 4.1, 0.044, 512, 740.0},    // four groups of waves over the contraction,
    {64, 64, 4.2, 0.09, 256, 1110.0},    // and here
    {64, 128, 4.0, 0.17, 1024, 1410.0},
    {128, 128, 6.0, 0.16, 768, 1880.0},
    {128, 256, 5.5, 0.30, 512, 2180.0},
    {256, 256, 8.7, 0.77, 256, 2300.0},
};
constexpr int kTileKernels = sizeof(kTiles) / sizeof(kTiles[0]);
// bytes a microsecond of weights; fitted to repeated calls, whose weights the memory-side cache
// holds in part (a large copy moves 5.07e6, and weights that no cache holds come at 5.1e6)
constexpr double kWeightRate = 7.8e6;
constexpr double kTileRate = 6.5e4;     // and what one tile's CU takes of them
struct StreamCost {
    int bm;
    double fixed, step;   // a step: latency, eight waves on a group
    double rate;          // bytes a microsecond of codes, from the L2s
};
constexpr StreamCost kStreams[] = {{16, 3.5, 0.021, 7.8e6}, {32, 4.1, 0.072, 1.6e7}};

double weight_time(const LinearArgs &a, double tiles) {
    const double groups = a.ends && a.experts < a.rows ? a.experts : a.ends ? a.rows : 1;
    return groups * a.cout_pad * a.k_stride / (tiles * kTileRate < kWeightRate ? tiles * kTileRate : kWeightRate);
}

// Waves of the stream kernel on a group of 16 channels by 16 rows: all eight while the
// groups do not fill the card, or where each wave still has four steps; else as many as
// leave a wave some.  (Of the three, at the drawn sizes: 256 groups, 64 steps 2 % and with
// two waves 74 % behind the best; 2048 groups, 4 steps, eight 67 % and two 0 %.)
int stream_waves(const LinearArgs &a) {
    const double groups = met_tiles(a, 16) * ((a.cout + 15) / 16);
    const int steps = a.k_stride >> 6;
    if (groups < 256.0) return 8;
    if (groups < 512.0) return steps >= 16 ? 8 : 4;
    return steps >= 32 ? 8 : steps >= 16 ? 4 : 2;
}

// The stream kernel reads the rows' codes again for every 16 channels.
double stream_cost(const LinearArgs &a, const StreamCost &c, int waves) {
    const double rows = met_tiles(a, c.bm) * c.bm * (double)a.k_stride * (a.cout_pad / 16) / c.rate, w = weight_time(a, 1e9);
    const double latency = (a.k_stride >> 6) * c.step * (a.gated ? 1.4 : 1.0) * 8 / waves, t = rows > w ? rows : w;
    return c.fixed + (t > latency ? t : latency);
}

double tile_cost(const LinearArgs &a, const TileCost &c) {
    const double tiles = met_tiles(a, c.bm) * ((a.cout_pad + c.bn - 1) / c.bn), steps = a.k_stride / 64;
    // one layer's tiles are alike: the last ones of a full card run by themselves, mostly
    const double up = 256.0 * (double)((int64_t)(tiles + 255.0) / 256);
    const double whole = a.ends || tiles <= 256.0 ? tiles : up - 0.2 * (up - tiles);
    double t = whole * c.bm * c.bn * a.k_stride * 2e-6 / c.rate;
    // (where a CU holds one tile, the start and the end of one are not hidden by another)
    const double rounds = 1 + (int64_t)((tiles - 1.0) / c.slots), w = weight_time(a, tiles);
    const double latency = rounds * steps * c.step + (c.slots == 256 ? (rounds - 1) * c.fixed : 0.0);
    if (latency > t) t = latency;
    if (w > t) t = w;
    return c.fixed + t;
}

}  // namespace

LinearChoice choose_linear(const LinearArgs &a) {
    const int waves = stream_waves(a);
    LinearChoice best = {kStream16, waves};
    double cost = stream_cost(a, kStreams[0], waves);
    if (const double c = stream_cost(a, kStreams[1], 8); c < cost) {
        cost = c;
        best = {kStream32, 8};
    }
    // (a long call never streams; the products of large sizes stay far inside a double)
    if (met_tiles(a, 16) * 16 > 4096 + 16.0 * a.experts) cost = 1e300;
    for (int i = 0; i < kTileKernels; ++i) {
        const double c = tile_cost(a, kTiles[i]);
        if (c < cost) {
            cost = c;
            best = {i, 0};
        }
    }
    return best;
}

}  // namespace hatq
