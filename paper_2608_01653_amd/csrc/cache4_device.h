// Device-side layout of the 4-bit cache and the transforms of its heads (gfx950).
//
// A head's channels are taken 64 at a time, NB blocks of them, zeros past the end, and
// its positions 8 at a time.  One octet of positions of one head, 544 NB bytes:
//   keys    [NB][4 chunks][4][2][8 bytes]: chunk u holds channels 16 u .. 16 u + 15 of the
//           block, [r][h] position 4 h + r.  Byte b of the chunk's word w holds the codes of
//           channels 8 w + b (low half) and 8 w + 4 + b (high half) in two's complement.
//   values  [NB][16 runs][8 positions][2 bytes]: run l holds channels 4 l .. 4 l + 3, the
//           lowest in the lowest bits, code + 8.
//   scales  keys [NB][8 positions], values [NB][8 positions], bf16
// A wave's 16-byte load at each of 64 addresses is then a matrix operand of 32 positions by
// 64 channels with no exchange between lanes: for the keys, positions are rows and channels
// the contraction; for the values, channels are rows and positions the contraction.
#pragma once

#include "cache4.h"
#include "hatq_device.h"
#include "linear_device.h"

namespace hatq {

constexpr int kOctet = 544;     // bytes a block of 64 channels of 8 positions of a head
constexpr int kKeyCodes = 256;

// Byte offsets inside an octet: 16 codes of a key's chunk, 4 of a value's run, a scale.
__device__ __forceinline__ int key_at(int block, int chunk, int pos8) {
    return block * kKeyCodes + chunk * 64 + (pos8 & 3) * 16 + (pos8 >> 2) * 8;
}
template <int NB>
__device__ __forceinline__ int value_at(int block, int run, int pos8) {
    return NB * kKeyCodes + block * 256 + run * 16 + pos8 * 2;
}
template <int NB>
__device__ __forceinline__ int scale_at(int which, int block, int pos8) {
    return NB * 512 + (which * NB + block) * 16 + pos8 * 2;
}

// Byte offset of a page's first octet of one head; an octet of it is octet * NB * kOctet on.
template <int NB>
__device__ __forceinline__ int64_t page_offset(const Cache4 &c, int page, int head) {
    return ((int64_t)page * c.heads + head) * ((int64_t)(NB * kOctet) << (c.log_page - 3));
}

// The sequence of a row of the call, -1 past the last one, and its position, -1 before the
// first one.
struct Row4 {
    int seq, pos;
};
__device__ __forceinline__ Row4 row_place(const Places4 &at, int row) {
    int seq, begin, count;
    if (!at.ends) {
        count = at.rows / at.batch;
        seq = row / count;
        begin = seq * count;
    } else {
        int lo = 0, hi = at.batch;      // the first sequence whose end is past the row
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (at.ends[mid] > row) hi = mid;
            else lo = mid + 1;
        }
        seq = lo;
        if (seq >= at.batch) return {-1, -1};
        begin = seq ? at.ends[seq - 1] : 0;
        count = at.ends[seq] - begin;
    }
    const int64_t pos = (int64_t)at.lens[seq] - count + (row - begin);
    return {seq, pos < 0 || pos > 0x7fffffff ? -1 : (int)pos};
}

// The page of a position, or -1: past the table, or a page that the cache does not have.
__device__ __forceinline__ int page_of(const Cache4 &c, const Places4 &at, int seq, int pos) {
    const int slot = pos >> c.log_page;
    if (pos < 0 || slot >= at.width) return -1;
    const int page = at.table[(int64_t)seq * at.width + slot];
    return (unsigned)page < (unsigned)c.pages ? page : -1;
}

// A head's values from element `at` on: 16 channels of each block, chunk `chunk` of it, zeros
// past the head's end; all loads under way before the first value is used, and `between`,
// which does not read them, before that.
template <int NB, typename T, typename F>
__device__ __forceinline__ void load_head(const T *p, int chunk, int dim, float (&v)[NB][16], F between) {
    Raw8<T> raw[NB][2];
    T one[16];      // (of a chunk that the head's end cuts: one block's at most)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int c0 = b * 64 + chunk * 16;
        if (c0 + 16 <= dim) {
            load_raw(p + c0, raw[b][0]);
            load_raw(p + c0 + 8, raw[b][1]);
        }
    }
    between();
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int c0 = b * 64 + chunk * 16;
        if (c0 + 16 <= dim) {
            raw_values(raw[b][0], v[b]);
            raw_values(raw[b][1], v[b] + 8);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[b][j] = 0.0f;
            if (c0 < dim) {
#pragma unroll
                for (int j = 0; j < 16; ++j) one[j] = p[min(c0 + j, dim - 1)];
#pragma unroll
                for (int j = 0; j < 16; ++j) v[b][j] = c0 + j < dim ? to_float(one[j]) : 0.0f;
            }
        }
    }
}
template <int NB, typename F>
__device__ __forceinline__ void load_head(const Heads4 &x, int64_t at, int chunk, int dim, float (&v)[NB][16], F between) {
    if (x.type == kF32) load_head<NB>(static_cast<const float *>(x.p) + at, chunk, dim, v, between);
    else if (x.type == kBf16) load_head<NB>(static_cast<const bf16_t *>(x.p) + at, chunk, dim, v, between);
    else load_head<NB>(static_cast<const _Float16 *>(x.p) + at, chunk, dim, v, between);
}

template <typename T>
__device__ __forceinline__ void put16(T *p, int c0, int dim, const float *v) {
    if (c0 + 16 <= dim) {
#pragma unroll
        for (int j = 0; j < 16; j += 16 / (int)sizeof(T)) store16(p + c0 + j, v + j);
        return;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j)
        if (c0 + j < dim) p[c0 + j] = from_float<T>(v[j]);
}
__device__ __forceinline__ void store_head16(const Heads4 &x, int64_t at, int c0, int dim, const float *v) {
    if (x.type == kF32) put16(static_cast<float *>(x.p) + at, c0, dim, v);
    else if (x.type == kBf16) put16(static_cast<bf16_t *>(x.p) + at, c0, dim, v);
    else put16(static_cast<_Float16 *>(x.p) + at, c0, dim, v);
}

// Chunks of a head in adjacent lanes (the cache's own kernels), or 16 lanes apart, as a
// matrix instruction has them (the attention): the stage with the chunk ^ MASK of 16 values.
// Returns the sign of the values held relative to the transform's.
struct ChunksAdjacent {
    template <int MASK>
    static __device__ __forceinline__ float stage(float (&v)[16]) {
        const float c = (threadIdx.x & MASK) ? -1.0f : 1.0f;
        token_cross<MASK>(v, c);
        return c;
    }
};
struct ChunksApart {
    // A swap of two values between the lanes of a pair leaves each lane with both partners of
    // one of the values; their sum and difference go back the same way.
    template <int MASK>
    static __device__ __forceinline__ void swap(float &x, float &y) {
        const uint32_t u = __float_as_uint(x), w = __float_as_uint(y);
        if constexpr (MASK == 1) {
            const auto r = __builtin_amdgcn_permlane16_swap(u, w, false, false);
            x = __uint_as_float(r[0]);
            y = __uint_as_float(r[1]);
        } else {
            const auto r = __builtin_amdgcn_permlane32_swap(u, w, false, false);
            x = __uint_as_float(r[0]);
            y = __uint_as_float(r[1]);
        }
    }
    template <int MASK>
    static __device__ __forceinline__ float stage(float (&v)[16]) {
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            swap<MASK>(v[j], v[j + 1]);
            float sum = v[j] + v[j + 1], less = v[j] - v[j + 1];
            swap<MASK>(sum, less);
            v[j] = sum;
            v[j + 1] = less;
        }
        return 1.0f;
    }
};

// The order-2^lb butterfly of heads held 16 channels a lane and block, ascending stages;
// returns the sign of the values held relative to the transform's.
template <int NB, typename C>
__device__ __forceinline__ float head_butterfly(float (&v)[NB][16], int lb, C) {
    float sigma = 1.0f;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        if (lb >= 1) reg_stage<1>(v[n]);
        if (lb >= 2) reg_stage<2>(v[n]);
        if (lb >= 3) reg_stage<4>(v[n]);
        if (lb >= 4) reg_stage<8>(v[n]);
        // (the same sign for every block)
        if (lb >= 5) sigma = C::template stage<1>(v[n]);
        if (lb >= 6) sigma *= C::template stage<2>(v[n]);
    }
    if constexpr (NB % 2 == 0) {    // (a block of 128 divides the head: no odd one)
        if (lb >= 7) {
#pragma unroll
            for (int n = 0; n < NB; n += 2)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float a = v[n][j], b = v[n + 1][j];
                    v[n][j] = a + b;
                    v[n + 1][j] = a - b;
                }
        }
    }
    return sigma;
}

}  // namespace hatq
