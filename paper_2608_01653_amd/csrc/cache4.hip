// New tokens' keys and values into a 4-bit cache, and back from it.
#include "cache4_device.h"

namespace hatq {
namespace {

constexpr int kThreads = 512;

// s = bf16(fl32(m / 7)), at least 2^-100, as a float.  With the largest magnitude below 2^102
// a scale is within [2^-100, 2^100], so that a weight relative to weight times scale, as the
// attention keeps it, is an ordinary float32 whatever the scales are.
constexpr float kLeastScale = 0x1p-100f, kMostValue = 0x1p102f;
__device__ __forceinline__ float cache_scale(float m) {
    return fmaxf(__uint_as_float(bf16_pair(m / 7.0f, 0.0f) << 16), kLeastScale);
}

// A lane's place: a chunk of one head of one row, of keys (the first half of a block's threads) or
// values.  The four chunks of a head are adjacent lanes, so its transform and maxima stay inside a
// quad; eight adjacent rows, mostly an octet of the cache, are in one half of a wave, whose stores
// and loads then meet in few lines of it; a block has up to eight heads (2^log_heads), and as many
// more rows where there are fewer.  (Keys and values in one block, since an octet's lines hold
// both: in blocks of their own 90 us for 83, 32768 rows of 8 heads of 128 bf16 in and out.)
struct Unit {
    int row, head, chunk;
    bool in;
};
__device__ __forceinline__ Unit this_unit(const CacheArgs &a, int log_heads) {
    const int t = threadIdx.x & 255, u = t >> 5;
    const int row = (blockIdx.x * (8 >> log_heads) + (u >> log_heads)) * 8 + ((t >> 2) & 7);
    const int head = (blockIdx.y << log_heads) + (u & ((1 << log_heads) - 1));
    return {row, head, t & 3, row < a.at.rows && head < a.c.heads};
}

template <int NB>
__device__ __forceinline__ uint8_t *octet_of(const Cache4 &c, int page, int head, int pos) {
    const int in_page = pos & ((1 << c.log_page) - 1);
    return c.buf + page_offset<NB>(c, page, head) + (in_page >> 3) * (NB * kOctet);
}

// S = B x of a head, A = max |S| of each 64 channels, s = bf16(fl32(A / 7)), codes
// clamp(rne(fl32(S / s)), -7, 7); a head with a value that is not below 2^102 gets scales
// NaN and codes 0.  bf16 scales: the range of the floats that come in, at 2 bytes for 32 of
// codes; the codes are made with the rounded scale, so the rounding (2^-8) costs nothing
// but the clamp of a maximum up to 7.03 steps away.
// Codes without a division for each: with r within 2^-23 of 1 / s, v r and v / s differ by at
// most 7.03 (2^-23 + 2^-24) < 2^-19, so k = rne(v r) is rne(fl(v / s)) where v r is within
// 0.5 - 2^-16 of k; a chunk with a value nearer to the middle of two codes divides, or clears
// its codes if the head is not fine.
// LB: log2 of the transform's block, -1 where it is known at run time only.
// Bound by the instructions next to the bytes: 32768 rows of 8 heads of 128, bf16, of a fused
// query-key-value product: 49 us for 170 MB (a copy of as many 33), 616 vector instructions a
// wave that take 33 us by themselves (224 of them the 7 butterfly stages of 32 values a lane).
template <int NB, int LB>
__global__ void __launch_bounds__(kThreads) cache4_append_kernel(const CacheArgs a, int log_heads) {
    const Unit n = this_unit(a, log_heads);
    if (!n.in) return;
    const int which = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    const Heads4 x = which ? a.x[1] : a.x[0];
    float v[NB][16];
    Row4 r;
    int page;
    load_head<NB>(x, n.row * x.row + n.head * x.head, n.chunk, a.c.dim, v, [&] {
        r = row_place(a.at, n.row);
        page = r.seq < 0 ? -1 : page_of(a.c, a.at, r.seq, r.pos);
    });
    if (page < 0) return;
    const float sigma = head_butterfly(v, LB < 0 ? a.c.log_b : LB, ChunksAdjacent{});
    float m[NB], all = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        m[b] = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; j += 2)
            m[b] = __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(v[b][j]), fabsf(v[b][j + 1])), m[b]);
        m[b] = __builtin_elementwise_maximum(m[b], lane_xor<1>(m[b]));
        m[b] = __builtin_elementwise_maximum(m[b], lane_xor<2>(m[b]));
        all = __builtin_elementwise_maximum(all, m[b]);
    }
    const bool fine = all < kMostValue;
    uint8_t *const octet = octet_of<NB>(a.c, page, n.head, r.pos);
    const int pos8 = r.pos & 7;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const float s = cache_scale(m[b]);
        const float inv = sigma * __builtin_amdgcn_rcpf(s);
        const float magic = which ? HATQ_MAGIC + 8.0f : HATQ_MAGIC;     // (values are held as code + 8)
        uint32_t q[16];
        float off = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            float d[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float k = __builtin_fmaf(v[b][j + e], inv, magic);
                d[e] = __builtin_fmaf(v[b][j + e], inv, -(k - magic));
                q[j + e] = __float_as_uint(k);      // its low bits: the code
            }
            off = __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(d[0]), fabsf(d[1])), off);
        }
        if (!(fine && off <= 0.5f - 0x1p-16f)) {
            asm volatile("");   // a branch: else the compiler divides for every chunk and selects
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float k = __builtin_amdgcn_fmed3f(rintf((sigma * v[b][j]) / s), -7.0f, 7.0f);
                q[j] = (uint32_t)((fine ? (int)k : 0) + (which ? 8 : 0));
            }
        }
        // (half bytes: the codes of four bytes' low halves, and of their high ones)
        const auto halves = [&](int l0, int l1, int l2, int l3, int h0, int h1, int h2, int h3) {
            const uint32_t low = pack_low_bytes(q[l0], q[l1], q[l2], q[l3]), high = pack_low_bytes(q[h0], q[h1], q[h2], q[h3]);
            return (low & 0x0f0f0f0fu) | ((high << 4) & 0xf0f0f0f0u);
        };
        if (which == 0) {
            *reinterpret_cast<uint2 *>(octet + key_at(b, n.chunk, pos8)) =
                make_uint2(halves(0, 1, 2, 3, 4, 5, 6, 7), halves(8, 9, 10, 11, 12, 13, 14, 15));
        } else {
            const uint32_t w[2] = {halves(0, 2, 4, 6, 1, 3, 5, 7), halves(8, 10, 12, 14, 9, 11, 13, 15)};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<uint16_t *>(octet + value_at<NB>(b, 4 * n.chunk + i, pos8)) = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
        if (n.chunk == 0)
            *reinterpret_cast<uint16_t *>(octet + scale_at<NB>(which, b, pos8)) =
                fine ? (uint16_t)(__float_as_uint(s) >> 16) : (uint16_t)0x7fc0;
    }
}

// x' = B (s c) / b: what the codes stand for, 0 where there is no page.  As many rows as above: 33 to 36
// us for 170 MB, 5 TB/s, with 550 vector instructions a wave that take 29.
template <int NB, int LB>
__global__ void __launch_bounds__(kThreads) cache4_read_kernel(const CacheArgs a, int log_heads) {
    const Unit n = this_unit(a, log_heads);
    if (!n.in) return;
    const Row4 r = row_place(a.at, n.row);
    if (r.seq < 0) return;
    const int page = page_of(a.c, a.at, r.seq, r.pos);
    const int which = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    float v[NB][16];
    if (page >= 0) {
        const uint8_t *const octet = octet_of<NB>(a.c, page, n.head, r.pos);
        const int pos8 = r.pos & 7;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const uint32_t bits = *reinterpret_cast<const uint16_t *>(octet + scale_at<NB>(which, b, pos8));
            const float s = __uint_as_float(bits << 16);
            int q[16];
            if (which == 0) {
                const uint2 w = *reinterpret_cast<const uint2 *>(octet + key_at(b, n.chunk, pos8));
#pragma unroll
                for (int j = 0; j < 16; ++j) q[j] = (int)((j >> 3 ? w.y : w.x) << (28 - (j & 3) * 8 - (j & 4))) >> 28;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t w = *reinterpret_cast<const uint16_t *>(octet + value_at<NB>(b, 4 * n.chunk + i, pos8));
#pragma unroll
                    for (int j = 0; j < 4; ++j) q[4 * i + j] = (int)((w >> (4 * j)) & 15) - 8;
                }
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) v[b][j] = (float)q[j] * s;
        }
    } else {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) v[b][j] = 0.0f;
    }
    const float sigma = head_butterfly(v, LB < 0 ? a.c.log_b : LB, ChunksAdjacent{});
    const Heads4 x = which ? a.x[1] : a.x[0];
    const float inv_b = sigma * __uint_as_float((uint32_t)(127 - a.c.log_b) << 23);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[b][j] *= inv_b;
        store_head16(x, n.row * x.row + n.head * x.head, b * 64 + n.chunk * 16, a.c.dim, v[b]);
    }
}

int log_heads_of(const CacheArgs &a) { return a.c.heads >= 5 ? 3 : a.c.heads >= 3 ? 2 : a.c.heads - 1; }
dim3 unit_grid(const CacheArgs &a) {
    const int log = log_heads_of(a), rows = 64 >> log;
    return dim3((a.at.rows + rows - 1) / rows, (a.c.heads + (1 << log) - 1) >> log);
}

// A kernel for the call's blocks of channels and its transform: of 64 and 128 as constants, 722 ->
// 600 vector instructions a wave.
#define HATQ_CACHE_LAUNCH(kernel, nb)                                                            \
    do {                                                                                          \
        if constexpr (nb % 2 == 0)                                                                \
            if (a.c.log_b == 7) { kernel<nb, 7><<<grid, kThreads, 0, st>>>(a, log); break; }      \
        if (a.c.log_b == 6) kernel<nb, 6><<<grid, kThreads, 0, st>>>(a, log);                     \
        else kernel<nb, -1><<<grid, kThreads, 0, st>>>(a, log);                                   \
    } while (0)

template <int NB>
void append(const CacheArgs &a, hipStream_t st) {
    const dim3 grid = unit_grid(a);
    const int log = log_heads_of(a);
    HATQ_CACHE_LAUNCH(cache4_append_kernel, NB);
}
template <int NB>
void read(const CacheArgs &a, hipStream_t st) {
    const dim3 grid = unit_grid(a);
    const int log = log_heads_of(a);
    HATQ_CACHE_LAUNCH(cache4_read_kernel, NB);
}

}  // namespace

hipError_t launch_cache4_append(const CacheArgs &a, hipStream_t st) {
    switch ((a.c.dim + 63) / 64) {
        case 1: append<1>(a, st); break;
        case 2: append<2>(a, st); break;
        case 3: append<3>(a, st); break;
        default: append<4>(a, st); break;
    }
    return hipGetLastError();
}

hipError_t launch_cache4_read(const CacheArgs &a, hipStream_t st) {
    switch ((a.c.dim + 63) / 64) {
        case 1: read<1>(a, st); break;
        case 2: read<2>(a, st); break;
        case 3: read<3>(a, st); break;
        default: read<4>(a, st); break;
    }
    return hipGetLastError();
}

}  // namespace hatq
