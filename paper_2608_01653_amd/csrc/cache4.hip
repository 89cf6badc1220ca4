// New tokens' keys and values into a 4-bit cache, and back from it.
#include "cache4_device.h"

namespace hatq {
namespace {

constexpr int kThreads = 256;

// s = bf16(fl32(m / 7)), at least 2^-100, as a float.  With the largest magnitude below 2^102
// a scale is within [2^-100, 2^100], so that a weight relative to weight times scale, as the
// attention keeps it, is an ordinary float32 whatever the scales are.
constexpr float kLeastScale = 0x1p-100f, kMostValue = 0x1p102f;
__device__ __forceinline__ float cache_scale(float m) {
    return fmaxf(__uint_as_float(bf16_pair(m / 7.0f, 0.0f) << 16), kLeastScale);
}

// A lane's place: chunk `threadIdx.x & 3` of one head of one row, of keys or values.  The
// four chunks of a head are adjacent lanes, so its transform and maxima stay inside a quad.
struct Unit {
    int which, head, chunk;
    int64_t row;
};
__device__ __forceinline__ Unit unit_of(const CacheArgs &a, int64_t u) {
    const int64_t of_keys = (int64_t)a.at.rows * a.c.heads, n = u >= of_keys ? u - of_keys : u;
    const int64_t row = n / a.c.heads;
    return {u >= of_keys, (int)(n - row * a.c.heads), (int)(threadIdx.x & 3), row};
}
__device__ __forceinline__ int64_t this_unit() {
    return (((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kThreads + threadIdx.x) >> 2;
}

template <int NB>
__device__ __forceinline__ uint8_t *octet_of(const Cache4 &c, int page, int head, int pos) {
    const int in_page = pos & ((1 << c.log_page) - 1);
    return c.buf + page_offset<NB>(c, page, head) + (in_page >> 3) * (NB * kOctet);
}

// S = B x of a head, A = max |S| of each 64 channels, s = bf16(fl32(A / 7)), codes
// clamp(rne(fl32(S / s)), -7, 7); a head with a value that is not below 2^102 gets scales
// NaN and codes 0.  bf16 scales: the range of the floats that come in, at 2 bytes for 32 of
// codes; the codes are made with the rounded scale, so the rounding (2^-9) costs nothing
// but the clamp of a maximum up to 7.03 steps away.
template <int NB>
__global__ void __launch_bounds__(kThreads) cache4_append_kernel(const CacheArgs a) {
    const int64_t u = this_unit();
    if (u >= 2 * (int64_t)a.at.rows * a.c.heads) return;
    const Unit n = unit_of(a, u);
    const Row4 r = row_place(a.at, (int)n.row);
    if (r.seq < 0) return;
    const int page = page_of(a.c, a.at, r.seq, r.pos);
    if (page < 0) return;
    const Heads4 &x = a.x[n.which];
    float v[NB][16];
#pragma unroll
    for (int b = 0; b < NB; ++b) load_head16(x, n.row * x.row + n.head * x.head, b * 64 + n.chunk * 16, a.c.dim, v[b]);
    head_butterfly(v, a.c.log_b, ChunksAdjacent{});
    float m[NB], all = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        m[b] = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) m[b] = __builtin_elementwise_maximum(m[b], fabsf(v[b][j]));
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
        uint32_t q[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float t = __builtin_amdgcn_fmed3f(rintf(v[b][j] / s), -7.0f, 7.0f);
            q[j] = fine ? (uint32_t)(int)t : 0u;
        }
        if (n.which == 0) {
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j >> 3] |= (q[j] & 15) << ((j & 3) * 8 + (j & 4));
            *reinterpret_cast<uint2 *>(octet + key_at(b, n.chunk, pos8)) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) w |= ((q[4 * i + j] + 8) & 15) << (4 * j);
                *reinterpret_cast<uint16_t *>(octet + value_at<NB>(b, 4 * n.chunk + i, pos8)) = (uint16_t)w;
            }
        }
        if (n.chunk == 0)
            *reinterpret_cast<uint16_t *>(octet + scale_at<NB>(n.which, b, pos8)) =
                fine ? (uint16_t)(__float_as_uint(s) >> 16) : (uint16_t)0x7fc0;
    }
}

// x' = B (s c) / b: what the codes stand for, 0 where there is no page.
template <int NB>
__global__ void __launch_bounds__(kThreads) cache4_read_kernel(const CacheArgs a) {
    const int64_t u = this_unit();
    if (u >= 2 * (int64_t)a.at.rows * a.c.heads) return;
    const Unit n = unit_of(a, u);
    const Row4 r = row_place(a.at, (int)n.row);
    if (r.seq < 0) return;
    const int page = page_of(a.c, a.at, r.seq, r.pos);
    float v[NB][16];
    if (page >= 0) {
        const uint8_t *const octet = octet_of<NB>(a.c, page, n.head, r.pos);
        const int pos8 = r.pos & 7;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const uint32_t bits = *reinterpret_cast<const uint16_t *>(octet + scale_at<NB>(n.which, b, pos8));
            const float s = __uint_as_float(bits << 16);
            int q[16];
            if (n.which == 0) {
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
    head_butterfly(v, a.c.log_b, ChunksAdjacent{});
    const Heads4 &x = a.x[n.which];
    const float inv_b = __uint_as_float((uint32_t)(127 - a.c.log_b) << 23);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[b][j] *= inv_b;
        store_head16(x, n.row * x.row + n.head * x.head, b * 64 + n.chunk * 16, a.c.dim, v[b]);
    }
}

dim3 unit_grid(const CacheArgs &a) {
    const int64_t units = 2 * (int64_t)a.at.rows * a.c.heads, n = (units * 4 + kThreads - 1) / kThreads;
    const int64_t x = n < (1 << 20) ? n : 1 << 20;
    return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

}  // namespace

hipError_t launch_cache4_append(const CacheArgs &a, hipStream_t st) {
    const dim3 grid = unit_grid(a);
    switch ((a.c.dim + 63) / 64) {
        case 1: cache4_append_kernel<1><<<grid, kThreads, 0, st>>>(a); break;
        case 2: cache4_append_kernel<2><<<grid, kThreads, 0, st>>>(a); break;
        case 3: cache4_append_kernel<3><<<grid, kThreads, 0, st>>>(a); break;
        default: cache4_append_kernel<4><<<grid, kThreads, 0, st>>>(a); break;
    }
    return hipGetLastError();
}

hipError_t launch_cache4_read(const CacheArgs &a, hipStream_t st) {
    const dim3 grid = unit_grid(a);
    switch ((a.c.dim + 63) / 64) {
        case 1: cache4_read_kernel<1><<<grid, kThreads, 0, st>>>(a); break;
        case 2: cache4_read_kernel<2><<<grid, kThreads, 0, st>>>(a); break;
        case 3: cache4_read_kernel<3><<<grid, kThreads, 0, st>>>(a); break;
        default: cache4_read_kernel<4><<<grid, kThreads, 0, st>>>(a); break;
    }
    return hipGetLastError();
}

}  // namespace hatq
