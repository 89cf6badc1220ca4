// Linear layers over tokens: token codes, weight preparation, and the order and
// the weighted sum of expert rows.  The products are in linear.hip.
#include "hatq_device.h"
#include "linear.h"
#include "linear_device.h"

namespace hatq {
namespace {

constexpr int kThreads = 256;

// ---- token codes ----------------------------------------------------------------
// S = B x per token, s = fl32(max|S| / 127), q = clamp(rne(fl32(S / s))).
//
// A token's row stays in registers between its maximum and its codes, so x is read
// once.  Chunk i of row thread t is number i * 64 * WAVES + t.  The maximum keeps NaN:
// a token with a value that is not finite gets the scale NaN and codes 0.  Bound by
// memory with the butterflies (7 adds an element at order 128) close behind: 4096 tokens
// of 4096, bf16, 12.1 us, 4.2 TB/s; 8192 of them 20.8 us, 4.8 TB/s.
// Row `row` by its thread t; red: WAVES floats of LDS for each row of the block.
template <int WAVES, int CH, typename T>
__device__ __forceinline__ void token_quant_row(const TokenArgs &a, int64_t row, int t, float *red) {
    constexpr int RT = 64 * WAVES;   // threads of a row
    const bool in = row < a.rows;    // (a block of several waves a row has a barrier for all)
    if (WAVES == 1 && !in) return;
    const T *x = static_cast<const T *>(a.x) + (in ? row : 0) * a.x_stride;
    const int chunks = a.k_stride >> 3;

    Raw8<T> raw[CH] = {};
    load_chunks<T, CH, RT>(x, a.cin, t, raw);
    float v[CH * 8];
    chunk_values<T, CH, RT>(x, a.cin, t, raw, v);
    const float sigma = token_butterfly(v, t, a.log_b);
    float m = token_max(v);
    if constexpr (WAVES > 1) {
        if ((t & 63) == 0) red[t >> 6] = m;
        __syncthreads();
        m = red[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = __builtin_elementwise_maximum(m, red[w]);
        if (!in) return;
    }
    const float s = token_scale(m);
    if (t == 0) a.sx[row] = s;
    const float r = sigma * (1.0f / s);
    const bool plain = token_plain(s);
    // (by 16 rows: 16 codes of a row, then those of the next)
    int8_t *q = a.xq + (a.by16 ? (row >> 4) * 16 * a.k_stride + (row & 15) * 16 : row * a.k_stride);
    const int pair = a.by16 ? 256 : 16;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * RT + t;
        const uint2 codes = token_codes8(&v[8 * i], sigma, s, r, plain);
        if (c < chunks) *reinterpret_cast<uint2 *>(q + (c >> 1) * pair + (c & 1) * 8) = codes;
    }
}

// One row a block of WAVES waves, or four of one wave.
template <int WAVES, int CH, typename T>
__global__ void __launch_bounds__(WAVES == 1 ? kThreads : 64 * WAVES) token_quant_kernel(const TokenArgs a) {
    __shared__ float red[WAVES];
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t row = WAVES == 1 ? block * (kThreads / 64) + (threadIdx.x >> 6) : block;
    token_quant_row<WAVES, CH, T>(a, row, WAVES == 1 ? threadIdx.x & 63 : threadIdx.x, red);
}

template <int WAVES, int CH>
hipError_t token_launch(const TokenArgs &a, hipStream_t st) {
    const dim3 grid = grid_of(WAVES == 1 ? (a.rows + 3) / 4 : a.rows);
    const int threads = WAVES == 1 ? kThreads : 64 * WAVES;
    if (a.x_type == kF32) token_quant_kernel<WAVES, CH, float><<<grid, threads, 0, st>>>(a);
    else if (a.x_type == kBf16) token_quant_kernel<WAVES, CH, bf16_t><<<grid, threads, 0, st>>>(a);
    else token_quant_kernel<WAVES, CH, _Float16><<<grid, threads, 0, st>>>(a);
    return hipGetLastError();
}

// ---- weights --------------------------------------------------------------------
// Held channel of packed column p, or -1 in the padding.  A gated layer's columns
// go 32 gates, 32 values in turn, so one wave's accumulators hold both.
__device__ __forceinline__ int held_channel(const LinearPrepArgs &a, int p) {
    if (!a.gated) return p < a.cout ? p : -1;
    const int c = (p >> 6) * 32 + (p & 31);
    return c >= a.cout ? -1 : (p & 32) ? a.cout + c : c;
}

template <typename T>
__device__ double transformed(const T *w, int d, int b) {
    const int first = d & ~(b - 1), i = d & (b - 1);
    double acc = 0.0;
    for (int j = 0; j < b; ++j) {
        const double e = (double)to_float(w[first + j]);
        acc += (__popc(i & j) & 1) ? -e : e;
    }
    return acc;
}

// One block per packed column of an expert.  The maximum keeps NaN, as the tokens' does: a
// channel that is not finite gets the scale NaN and codes 0.
template <typename T>
__global__ void __launch_bounds__(kThreads) linear_prepare_kernel(const LinearPrepArgs a) {
    const int p = blockIdx.x, e = blockIdx.y;
    const int held = a.gated ? 2 * a.cout : a.cout;
    const int ch = held_channel(a, p);
    const int64_t row = (int64_t)e * held + ch;
    const T *w = static_cast<const T *>(a.w) + row * a.cin;
    float s = 0.0f;
    if (ch >= 0) {
        float m = 0.0f;
        for (int d = threadIdx.x; d < a.cin; d += kThreads)
            m = __builtin_elementwise_maximum(m, fabsf((float)transformed(w, d, a.hblock)));
        const float of_lane[2] = {m, 0.0f};
        m = token_max(of_lane);
        __shared__ float red[kThreads / 64];
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
        __syncthreads();
        m = red[0];
#pragma unroll
        for (int k = 1; k < kThreads / 64; ++k) m = __builtin_elementwise_maximum(m, red[k]);
        s = token_scale(m);
    }
    int8_t *out = a.wpack + ((int64_t)e * a.cout_pad + (p & ~15)) * a.k_stride + (p & 15) * 16;
    for (int d = threadIdx.x; d < a.k_stride; d += kThreads) {
        int8_t q = 0;
        if (s == s && ch >= 0 && d < a.cin) q = (int8_t)(int)rintf(clamp127((float)transformed(w, d, a.hblock) / s));
        out[(int64_t)(d >> 6) * 1024 + ((d >> 4) & 3) * 256 + (d & 15)] = q;
    }
    if (threadIdx.x == 0) {
        a.w_scale[(int64_t)e * a.cout_pad + p] = s;
        a.bias[(int64_t)e * a.cout_pad + p] = ch >= 0 && a.bias_in ? a.bias_in[row] : 0.0f;
    }
}

// Codes that are there already: a block takes 256 of 16 columns, reads runs of columns and
// writes runs of the packed order, by way of LDS.
__global__ void __launch_bounds__(kThreads) linear_pack_kernel(const LinearPrepArgs a) {
    __shared__ v4i tile[16][17];
    const int e = blockIdx.z, column = threadIdx.x >> 4, chunk = threadIdx.x & 15;
    const int p = blockIdx.y * 16 + column, c = blockIdx.x * 16 + chunk, ch = held_channel(a, p);
    const int64_t row = (int64_t)e * (a.gated ? 2 * a.cout : a.cout) + ch;
    const int8_t *from = a.codes + row * a.cin + c * 16;
    const bool whole = (reinterpret_cast<uintptr_t>(a.codes) & 15) == 0 && a.cin % 16 == 0;
    v4i q = {0, 0, 0, 0};
    if (ch >= 0 && c * 16 < a.cin) {
        if (whole) {
            q = *reinterpret_cast<const v4i *>(from);
        } else {
            int8_t *b = reinterpret_cast<int8_t *>(&q);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c * 16 + j < a.cin) b[j] = from[j];
        }
    }
    tile[chunk][column] = q;
    __syncthreads();
    const int to = blockIdx.x * 16 + column;   // the chunk that this thread writes, of column `chunk`
    int8_t *out = a.wpack + ((int64_t)e * a.cout_pad + blockIdx.y * 16) * a.k_stride;
    if (to < a.k_stride >> 4) *reinterpret_cast<v4i *>(out + (int64_t)to * 256 + chunk * 16) = tile[column][chunk];
    if (blockIdx.x == 0 && chunk == 0) {
        a.w_scale[(int64_t)e * a.cout_pad + p] = ch >= 0 ? a.scale_in[row] : 0.0f;
        a.bias[(int64_t)e * a.cout_pad + p] = ch >= 0 && a.bias_in ? a.bias_in[row] : 0.0f;
    }
}

// ---- the order of expert rows -----------------------------------------------------
// A stable counting sort of `pairs` ids.  Block b owns a contiguous segment, wave w of it
// a contiguous part.  The first row of expert e in block b is the rows of the experts
// before e plus the rows of e in the blocks before b; each wave then ranks its pairs 64
// at a time in order.  Ranks come from ballots, not from atomics, so equal ids keep
// their order.  Up to kOrderOne pairs every block counts all of them itself, in one launch;
// beyond, a first launch leaves the blocks' counts in a table.  Not bound by memory: a call
// is one or two launches (96 pairs 6.5 us through the binding) and then the counting by
// LDS atomics, where lanes with the same expert wait for each other (32768 pairs of 32
// experts 9.3 us, of 8 experts 12.3); through the table 65536 pairs of 32 8.5 us, 262144 of
// 64 15.9, 2^24 of 256 267 (200 MB).
constexpr int kOrderWaves = 8;
constexpr int kOrderThreads = 64 * kOrderWaves;
constexpr int kOrderBlocks = 256;
constexpr int kOrderSegment = 1024;   // pairs of a block, more when that would take over kOrderBlocks
constexpr int kOrderOne = 32768;

__host__ __device__ __forceinline__ int64_t order_segment(int64_t pairs) {
    const int64_t per = (pairs + kOrderBlocks - 1) / kOrderBlocks;
    const int64_t seg = per > kOrderSegment ? per : kOrderSegment;
    return (seg + kOrderThreads - 1) / kOrderThreads * kOrderThreads;
}

// f(first index, ids) over [begin, end) by `step` threads, this one the t-th, N ids of a
// thread loaded at once; -1 past the end.
template <int N, typename F>
__device__ __forceinline__ void order_ids(const int32_t *ids, int64_t begin, int64_t end, int t, int step, F f) {
    for (int64_t b = begin; b < end; b += step * N) {
        int id[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int64_t i = b + k * step + t;
            id[k] = i < end ? ids[i] : -1;
        }
        f(b + t, id);
    }
}

struct Span {
    int64_t begin, end;
};
__device__ __forceinline__ Span order_span(int64_t pairs, int block, int wave) {
    const int64_t seg = order_segment(pairs), part = seg / kOrderWaves;
    const int64_t b = block * seg + wave * part, e = b + part;
    return {b < pairs ? b : pairs, e < pairs ? e : pairs};
}

// counts[w][e] of this block's waves (zeroed, and a barrier on both sides).
__device__ __forceinline__ void order_counts(const OrderArgs &a, int64_t pairs, int *counts) {
    const int w = threadIdx.x >> 6;
    const Span s = order_span(pairs, blockIdx.x, w);
    order_ids<2>(a.ids, s.begin, s.end, threadIdx.x & 63, 64, [&](int64_t, const int *id) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if ((unsigned)id[k] < (unsigned)a.experts) atomicAdd(&counts[w * a.experts + id[k]], 1);
    });
}

__global__ void __launch_bounds__(kOrderThreads) order_count_kernel(const OrderArgs a) {
    extern __shared__ int lds[];
    for (int i = threadIdx.x; i < kOrderWaves * a.experts; i += kOrderThreads) lds[i] = 0;
    __syncthreads();
    order_counts(a, (int64_t)a.tokens * a.topk, lds);
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += kOrderThreads) {
        int n = 0;
        for (int w = 0; w < kOrderWaves; ++w) n += lds[w * a.experts + e];
        a.ws[(int64_t)blockIdx.x * a.experts + e] = n;
    }
}

// Block blockIdx.x of `blocks`.  lds: [experts] rows in all blocks, in the blocks before;
// counts [waves][experts].
template <bool TABLE>
__device__ void order_place(const OrderArgs &a, int blocks, int *lds) {
    const int E = a.experts;
    int *total = lds, *before = lds + E, *counts = lds + 2 * E;
    const int64_t pairs = (int64_t)a.tokens * a.topk;
    for (int i = threadIdx.x; i < (2 + kOrderWaves) * E; i += kOrderThreads) lds[i] = 0;
    __syncthreads();
    order_counts(a, pairs, counts);
    if (TABLE) {
        for (int i = threadIdx.x; i < blocks * E; i += kOrderThreads) {
            const int b = i / E, e = i - b * E, n = a.ws[i];
            atomicAdd(&total[e], n);
            if (b < (int)blockIdx.x) atomicAdd(&before[e], n);
        }
    } else {
        const int64_t mine = blockIdx.x * order_segment(pairs);
        order_ids<16>(a.ids, 0, mine, threadIdx.x, kOrderThreads, [&](int64_t, const int *id) {
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if ((unsigned)id[k] < (unsigned)E) atomicAdd(&before[id[k]], 1);
        });
        order_ids<16>(a.ids, mine, pairs, threadIdx.x, kOrderThreads, [&](int64_t, const int *id) {
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if ((unsigned)id[k] < (unsigned)E) atomicAdd(&total[id[k]], 1);
        });
    }
    __syncthreads();
    // exclusive scan over the block's threads, each with PER experts in a row
    constexpr int PER = kMaxExperts / kOrderThreads;
    int n[PER], sum = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int e = threadIdx.x * PER + k;
        n[k] = e < E ? total[e] + (TABLE ? 0 : before[e]) : 0;
        sum += n[k];
    }
    const int scan = wave_scan(sum, [](int x, int y) { return x + y; });
    __shared__ int wave_sum[kOrderWaves];
    if ((threadIdx.x & 63) == 63) wave_sum[threadIdx.x >> 6] = scan;
    __syncthreads();
    int first = scan - sum, all = 0;
    for (int w = 0; w < kOrderWaves; ++w) {
        if (w < (int)(threadIdx.x >> 6)) first += wave_sum[w];
        all += wave_sum[w];
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int e = threadIdx.x * PER + k;
        if (e >= E) break;
        // the waves' first rows of this expert
        int at = first + before[e];
        for (int w = 0; w < kOrderWaves; ++w) {
            const int c = counts[w * E + e];
            counts[w * E + e] = at;
            at += c;
        }
        first += n[k];
        if (blockIdx.x == 0) a.ends[e] = first;
    }
    __syncthreads();
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    volatile int *next = counts + w * E;   // read and written by turns within the wave
    const Span s = order_span(pairs, blockIdx.x, w);
    order_ids<2>(a.ids, s.begin, s.end, lane, 64, [&](int64_t i0, const int *ids) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int id = ids[k];
            const int64_t i = i0 + k * 64;
            const bool in = (unsigned)id < (unsigned)E;
            uint64_t same = __ballot(in);
#pragma unroll
            for (int bit = 0; bit < 10; ++bit) {
                const uint64_t set = __ballot((id >> bit) & 1);
                same &= (id >> bit) & 1 ? set : ~set;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1));
            int row = -1;
            if (in) row = next[id] + rank;
            __builtin_amdgcn_wave_barrier();   // every lane has read before the last of each id writes
            if (in && rank + 1 == __popcll(same)) next[id] = row + 1;
            __builtin_amdgcn_wave_barrier();
            if (in) a.src[row] = (int)((unsigned)i / (unsigned)a.topk);
            if (i < s.end) a.pos[i] = row;
        }
    });
    for (int64_t i = all + (int64_t)blockIdx.x * kOrderThreads + threadIdx.x; i < pairs; i += (int64_t)blocks * kOrderThreads)
        a.src[i] = -1;
}

template <bool TABLE>
__global__ void __launch_bounds__(kOrderThreads) order_place_kernel(const OrderArgs a) {
    extern __shared__ int lds[];
    order_place<TABLE>(a, gridDim.x, lds);
}

// The order of the rows in the first blocks, the codes of the tokens in the rest: neither
// needs the other.
template <int WAVES, int CH, typename T>
__global__ void __launch_bounds__(kOrderThreads) order_quant_kernel(const OrderArgs o, int blocks, const TokenArgs a) {
    extern __shared__ int lds[];
    if ((int)blockIdx.x < blocks) return order_place<false>(o, blocks, lds);
    constexpr int ROWS = kOrderThreads / (64 * WAVES);   // of a block
    token_quant_row<WAVES, CH, T>(a, (blockIdx.x - blocks) * ROWS + threadIdx.x / (64 * WAVES),
                                  threadIdx.x % (64 * WAVES), reinterpret_cast<float *>(lds) + threadIdx.x / (64 * WAVES) * WAVES);
}

// ---- the weighted sum of expert rows ------------------------------------------------
// Four channels a thread, its rows in ascending order; bound by the rows' bytes (16384 rows
// of 2048 into 4096 of bf16, 151 MB: 25 us, 6.0 TB/s).
template <typename T>
__global__ void __launch_bounds__(kThreads) combine_kernel(const CombineArgs a) {
    const int groups = (a.cols + 3) / 4;
    const int64_t n = (int64_t)a.tokens * groups;
    for (int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x; u < n; u += (int64_t)gridDim.x * kThreads) {
        const int tok = (int)(u / groups), c = (int)(u - (int64_t)tok * groups) * 4;
        const bool whole = c + 4 <= a.cols;
        const int32_t *pos = a.pos + (int64_t)tok * a.topk;
        const float *wt = a.weights + (int64_t)tok * a.topk;
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int j = 0; j < a.topk; ++j) {
            const int p = pos[j];
            if ((unsigned)p >= (unsigned)a.h_rows) continue;
            const float g = wt[j];
            const float *h = a.h + p * a.h_stride + c;
            if (whole) {
                float f[4];
                load4(h, f);
#pragma unroll
                for (int k = 0; k < 4; ++k) s[k] = __builtin_fmaf(g, f[k], s[k]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < a.cols) s[k] = __builtin_fmaf(g, h[k], s[k]);
            }
        }
        T *y = static_cast<T *>(a.y) + tok * a.y_stride + c;
        if (whole) {
            store4(y, s);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (c + k < a.cols) y[k] = from_float<T>(s[k]);
        }
    }
}

}  // namespace

hipError_t launch_token_quant(const TokenArgs &a, hipStream_t st) {
    const int chunks = a.k_stride >> 3;
    // Two chunks a lane and the waves a row takes.  (bf16, order 128, us: 4096 rows of
    // 4096 13.8 on four waves, 14.8 on two of four chunks, 15.4 on one of eight, 20.6 on
    // eight of one; 1 row of 4096 3.1, 4.1, 6.1, 3.1; 4096 rows of 2048 7.7 on two waves,
    // 7.8 on one, 11.5 on four.)
    if (chunks <= 64) return token_launch<1, 1>(a, st);
    if (chunks <= 128) return token_launch<1, 2>(a, st);
    if (chunks <= 256) return token_launch<2, 2>(a, st);
    if (chunks <= 512) return token_launch<4, 2>(a, st);
    if (chunks <= 1024) return token_launch<8, 2>(a, st);
    if (chunks <= 2048) return token_launch<16, 2>(a, st);
    if (chunks <= 4096) return token_launch<16, 4>(a, st);
    return token_launch<16, 8>(a, st);
}

hipError_t launch_linear_prepare(const LinearPrepArgs &a, hipStream_t st) {
    const dim3 grid(a.cout_pad, a.experts);
    if (a.codes)
        linear_pack_kernel<<<dim3((a.k_stride + 255) / 256, a.cout_pad / 16, a.experts), kThreads, 0, st>>>(a);
    else if (a.w_type == kBf16) linear_prepare_kernel<bf16_t><<<grid, kThreads, 0, st>>>(a);
    else if (a.w_type == kF16) linear_prepare_kernel<_Float16><<<grid, kThreads, 0, st>>>(a);
    else linear_prepare_kernel<float><<<grid, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_expert_order(const OrderArgs &a, hipStream_t st) {
    const int64_t pairs = (int64_t)a.tokens * a.topk, seg = order_segment(pairs);
    const int blocks = pairs > seg ? (int)((pairs + seg - 1) / seg) : 1;
    const size_t counts = sizeof(int) * kOrderWaves * a.experts, all = counts + 2 * sizeof(int) * a.experts;
    if (pairs <= kOrderOne) {
        order_place_kernel<false><<<blocks, kOrderThreads, all, st>>>(a);
    } else {
        order_count_kernel<<<blocks, kOrderThreads, counts, st>>>(a);
        order_place_kernel<true><<<blocks, kOrderThreads, all, st>>>(a);
    }
    return hipGetLastError();
}

template <int WAVES, int CH>
static hipError_t order_quant(const OrderArgs &o, int blocks, const TokenArgs &a, hipStream_t st) {
    constexpr int ROWS = kOrderThreads / (64 * WAVES);
    const int grid = blocks + (a.rows + ROWS - 1) / ROWS;
    size_t bytes = sizeof(int) * (2 + kOrderWaves) * o.experts;
    if (bytes < sizeof(float) * kOrderWaves) bytes = sizeof(float) * kOrderWaves;
    if (a.x_type == kF32) order_quant_kernel<WAVES, CH, float><<<grid, kOrderThreads, bytes, st>>>(o, blocks, a);
    else if (a.x_type == kBf16) order_quant_kernel<WAVES, CH, bf16_t><<<grid, kOrderThreads, bytes, st>>>(o, blocks, a);
    else order_quant_kernel<WAVES, CH, _Float16><<<grid, kOrderThreads, bytes, st>>>(o, blocks, a);
    return hipGetLastError();
}

hipError_t launch_order_quant(const OrderArgs &o, const TokenArgs &a, hipStream_t st) {
    const int64_t pairs = (int64_t)o.tokens * o.topk, seg = order_segment(pairs);
    const int blocks = pairs > seg ? (int)((pairs + seg - 1) / seg) : 1, chunks = a.k_stride >> 3;
    if (pairs > kOrderOne || chunks > 1024) {
        const hipError_t e = launch_expert_order(o, st);
        return e == hipSuccess ? launch_token_quant(a, st) : e;
    }
    if (chunks <= 64) return order_quant<1, 1>(o, blocks, a, st);
    if (chunks <= 128) return order_quant<1, 2>(o, blocks, a, st);
    if (chunks <= 256) return order_quant<2, 2>(o, blocks, a, st);
    if (chunks <= 512) return order_quant<4, 2>(o, blocks, a, st);
    return order_quant<8, 2>(o, blocks, a, st);
}

hipError_t launch_expert_combine(const CombineArgs &a, hipStream_t st) {
    const int64_t n = (int64_t)a.tokens * ((a.cols + 3) / 4);
    const int64_t blocks = (n + kThreads - 1) / kThreads;
    const int grid = (int)(blocks < 65536 ? blocks : 65536);
    if (a.y_type == kF32) combine_kernel<float><<<grid, kThreads, 0, st>>>(a);
    else if (a.y_type == kBf16) combine_kernel<bf16_t><<<grid, kThreads, 0, st>>>(a);
    else combine_kernel<_Float16><<<grid, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

size_t expert_order_ws_ints(int64_t pairs, int32_t experts) {
    const int64_t seg = order_segment(pairs);
    return pairs > kOrderOne ? (size_t)((pairs + seg - 1) / seg) * experts : 0;
}

}  // namespace hatq
