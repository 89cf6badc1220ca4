// Internal launchers of the 4-bit cache and the attention over it (host side, gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hatq {

// A cache's pages, as hatq_cache4.
struct Cache4 {
    uint8_t *buf;
    int32_t pages, log_page, heads, dim;
    int32_t log_b;      // transform block 2^log_b
};

// Where the sequences' positions are: hatq_cache4_append's table, lens and ends.
struct Places4 {
    const int32_t *table, *lens, *ends;
    int32_t width, batch, rows;
};

// A tensor [rows][heads][dim] of a hatq_dtype, strides in elements.
struct Heads4 {
    void *p;
    int64_t row, head;
    int32_t type;
};

struct CacheArgs {
    Cache4 c;
    Places4 at;
    Heads4 x[2];        // keys, values
};
hipError_t launch_cache4_append(const CacheArgs &a, hipStream_t st);
hipError_t launch_cache4_read(const CacheArgs &a, hipStream_t st);

struct AttentionArgs {
    Cache4 c;
    Places4 at;
    Heads4 q, y;
    int32_t share;      // query heads of one cached head
    int32_t causal, window;
    float scale;        // of a product of the untransformed heads
    int32_t splits;     // of each sequence's positions; partial results in ws where more than one
    void *ws;
};

// How a call is laid out: host code without a launch, from sizes alone.
struct AttentionPlan {
    int32_t cols;           // columns (a query row and head) of a cached head a block takes: 16 or wide_cols
    int32_t waves, splits;  // splits: 1 where cols is more than 16
    int64_t tiles;          // blocks of columns of one cached head, over all sequences: an upper bound
};
constexpr int wide_cols(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 48 : dim <= 192 ? 32 : 16; }
AttentionPlan plan_attention(int32_t batch, int32_t rows, int32_t heads, int32_t share, int32_t dim, int64_t max_len,
                             bool ragged, int32_t window);
// Bytes of one partial result: 16 query rows of a head, their maxima and sums.
inline size_t partial4_bytes(int32_t dim) { return (size_t)((dim + 63) / 64) * 4096 + 128; }
// For heads of up to 64, 128, 192 and 256 channels.
hipError_t launch_attention4_1(const AttentionArgs &a, const AttentionPlan &p, hipStream_t st);
hipError_t launch_attention4_2(const AttentionArgs &a, const AttentionPlan &p, hipStream_t st);
hipError_t launch_attention4_3(const AttentionArgs &a, const AttentionPlan &p, hipStream_t st);
hipError_t launch_attention4_4(const AttentionArgs &a, const AttentionPlan &p, hipStream_t st);

}  // namespace hatq
