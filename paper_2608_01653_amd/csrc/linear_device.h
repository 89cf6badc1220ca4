// Device-side element types of the linear layers over tokens (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hatq_device.h"

namespace hatq {

constexpr int kF32 = 0, kBf16 = 1, kF16 = 2;   // hatq_dtype

struct bf16_t {
    uint16_t bits;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(_Float16 v) { return (float)v; }
__device__ __forceinline__ float to_float(bf16_t v) { return __uint_as_float((uint32_t)v.bits << 16); }

// Two floats rounded to nearest even, NaN kept, as bf16 (low half from a).
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    typedef float v2f __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), v2bf));
}

template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ _Float16 from_float<_Float16>(float v) { return (_Float16)v; }
template <>
__device__ __forceinline__ bf16_t from_float<bf16_t>(float v) { return {(uint16_t)bf16_pair(v, v)}; }

// Vectors at any element's address: the hardware's loads and stores of 8 and 16 bytes need
// no alignment, so odd row strides and offset views take the same path.  (7075 rows, 512 ->
// 2198, bf16 rows of 4396 bytes: 31.7 us, 51.6 with stores of an element.)
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef _Float16 f16x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef _Float16 f16x8_any __attribute__((ext_vector_type(8), aligned(2)));

// Four adjacent elements.
__device__ __forceinline__ void load4(const float *p, float *v) {
    const f32x4_any a = *reinterpret_cast<const f32x4_any *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = a[j];
}

// Eight adjacent elements as they lie in memory, and their values.
template <typename T>
struct Raw8 {
    uint32_t w[2 * sizeof(T)];
};
template <typename T>
__device__ __forceinline__ void load_raw(const T *p, Raw8<T> &r) {
    const u32x4_any *q = reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
        const u32x4_any a = q[k];
#pragma unroll
        for (int j = 0; j < 4; ++j) r.w[4 * k + j] = a[j];
    }
}
__device__ __forceinline__ void raw_values(const Raw8<float> &r, float *v) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(r.w[j]);
}
__device__ __forceinline__ void raw_values(const Raw8<bf16_t> &r, float *v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(r.w[j] << 16);
        v[2 * j + 1] = __uint_as_float(r.w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void raw_values(const Raw8<_Float16> &r, float *v) {
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const v2h h = __builtin_bit_cast(v2h, r.w[j]);
        v[2 * j] = (float)h[0];
        v[2 * j + 1] = (float)h[1];
    }
}

// A token's chunks of 8 elements, number i * THREADS + t, of n elements at p (n = 0: an
// empty token, p is not read): the loads, all of them under way at once, and then the
// values, zeros past the end.  A chunk that the end cuts is read by elements.
template <typename T, int CH, int THREADS>
__device__ __forceinline__ void load_chunks(const T *p, int n, int t, Raw8<T> (&raw)[CH]) {
    if (n < 8) return;   // (no whole chunk)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int e = (i * THREADS + t) * 8;
        load_raw(p + (e + 8 <= n ? e : 0), raw[i]);
    }
}
template <typename T, int CH, int THREADS>
__device__ __forceinline__ void chunk_values(const T *p, int n, int t, const Raw8<T> (&raw)[CH], float (&v)[8 * CH]) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int e = (i * THREADS + t) * 8;
        raw_values(raw[i], &v[8 * i]);
        if (e + 8 > n) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[8 * i + j] = 0.0f;
            if (e < n) {
                T one[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) one[j] = p[min(e + j, n - 1)];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[8 * i + j] = e + j < n ? to_float(one[j]) : 0.0f;
            }
        }
    }
}

__device__ __forceinline__ void store4(float *p, const float *v) {
    *reinterpret_cast<f32x4_any *>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ void store4(bf16_t *p, const float *v) {
    *reinterpret_cast<u32x2_any *>(p) = u32x2_any{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
}
__device__ __forceinline__ void store4(_Float16 *p, const float *v) {
    *reinterpret_cast<f16x4_any *>(p) = f16x4_any{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
}

// One 16-byte piece.
__device__ __forceinline__ void store16(float *p, const float *v) { store4(p, v); }
__device__ __forceinline__ void store16(bf16_t *p, const float *v) {
    *reinterpret_cast<u32x4_any *>(p) =
        u32x4_any{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
}
__device__ __forceinline__ void store16(_Float16 *p, const float *v) {
    f16x8_any h;
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = (_Float16)v[j];
    *reinterpret_cast<f16x8_any *>(p) = h;
}

// Inclusive scans over the wave, of values >= 0, by DPP moves: rows of 16 lanes, then
// lane 15 of each row to the next row, then lane 31 to the upper half.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_or_0(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
template <typename F>
__device__ __forceinline__ int wave_scan(int v, F f) {
    v = f(v, dpp_or_0<0x111, 0xF>(v));   // row_shr 1, 2, 4, 8
    v = f(v, dpp_or_0<0x112, 0xF>(v));
    v = f(v, dpp_or_0<0x114, 0xF>(v));
    v = f(v, dpp_or_0<0x118, 0xF>(v));
    v = f(v, dpp_or_0<0x142, 0xA>(v));   // row_bcast 15
    return f(v, dpp_or_0<0x143, 0xC>(v));   // row_bcast 31
}

// ---- token codes --------------------------------------------------------------------
// A lane holds chunks of 8 adjacent elements, neighbouring lanes neighbouring chunks:
// index bits 0-2 are registers, bits 3-6 lanes of one 16-lane row, so the butterflies of
// a block of up to 128 stay inside a DPP row.

// The butterfly with lane ^ MASK, v + c v' for c = 1 or -1, of eight registers: the lane move
// is part of the fused multiply-add.  (Written out, since the compiler keeps a move, a wait
// and an add for each.)  A lane move may read a register two instructions after its write,
// so s_nop 1 comes first; the eight registers are independent.
#define HATQ_EIGHT(LINE, ctrl) LINE(0, 8, ctrl) LINE(1, 9, ctrl) LINE(2, 10, ctrl) LINE(3, 11, ctrl) LINE(4, 12, ctrl) \
    LINE(5, 13, ctrl) LINE(6, 14, ctrl) LINE(7, 15, ctrl)
#define HATQ_SELF(i, t, ctrl) "v_fmac_f32_dpp %" #i ", %" #i ", %8 " ctrl " row_mask:0xf bank_mask:0xf\n\t"
#define HATQ_MOVE(i, t, ctrl) "v_mov_b32_dpp %" #t ", %" #i " " ctrl " row_mask:0xf bank_mask:0xf\n\t"
#define HATQ_FROM(i, t, ctrl) "v_fmac_f32_dpp %" #i ", %" #t ", %16 " ctrl " row_mask:0xf bank_mask:0xf\n\t"
#define HATQ_INOUT(v) "+&v"(v[0]), "+&v"(v[1]), "+&v"(v[2]), "+&v"(v[3]), "+&v"(v[4]), "+&v"(v[5]), "+&v"(v[6]), "+&v"(v[7])
#define HATQ_OUT(v) "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
template <int MASK>
__device__ __forceinline__ void cross8(float *v, float c) {
    static_assert(MASK == 1 || MASK == 2 || MASK == 4 || MASK == 8, "lane mask");
    if constexpr (MASK == 1) asm("s_nop 1\n\t" HATQ_EIGHT(HATQ_SELF, "quad_perm:[1,0,3,2]") : HATQ_INOUT(v) : "v"(c));
    if constexpr (MASK == 2) asm("s_nop 1\n\t" HATQ_EIGHT(HATQ_SELF, "quad_perm:[2,3,0,1]") : HATQ_INOUT(v) : "v"(c));
    if constexpr (MASK == 8) asm("s_nop 1\n\t" HATQ_EIGHT(HATQ_SELF, "row_ror:8") : HATQ_INOUT(v) : "v"(c));
    if constexpr (MASK == 4) {   // i -> 7 - i inside 8 lanes, then i -> i ^ 3
        float t[8];
        asm("s_nop 1\n\t" HATQ_EIGHT(HATQ_MOVE, "row_half_mirror") HATQ_EIGHT(HATQ_FROM, "quad_perm:[3,2,1,0]")
            : HATQ_INOUT(v), HATQ_OUT(t) : "v"(c));
    }
}
#undef HATQ_EIGHT
#undef HATQ_SELF
#undef HATQ_MOVE
#undef HATQ_FROM
#undef HATQ_INOUT
#undef HATQ_OUT

template <int MASK, int R>
__device__ __forceinline__ void token_cross(float (&v)[R], float c) {
    static_assert(R % 8 == 0, "chunks of 8");
#pragma unroll
    for (int r = 0; r < R; r += 8) cross8<MASK>(v + r, c);
}

// The order-2^lb butterfly of every chunk; returns the sign of the values held relative
// to the transform's (hatq_device.h, cross_stage).
template <int R>
__device__ __forceinline__ float token_butterfly(float (&v)[R], int lane, int lb) {
    float sigma = 1.0f;
    if (lb >= 1) reg_stage<1>(v);
    if (lb >= 2) reg_stage<2>(v);
    if (lb >= 3) reg_stage<4>(v);
    if (lb >= 4) {
        const float c = (lane & 1) ? -1.0f : 1.0f;
        token_cross<1>(v, c);
        sigma *= c;
    }
    if (lb >= 5) {
        const float c = (lane & 2) ? -1.0f : 1.0f;
        token_cross<2>(v, c);
        sigma *= c;
    }
    if (lb >= 6) {
        const float c = (lane & 4) ? -1.0f : 1.0f;
        token_cross<4>(v, c);
        sigma *= c;
    }
    if (lb >= 7) {
        const float c = (lane & 8) ? -1.0f : 1.0f;
        token_cross<8>(v, c);
        sigma *= c;
    }
    return sigma;
}

// max |v| of the wave, NaN where one of them is (v_maximum, not v_max).
template <int R>
__device__ __forceinline__ float token_max(const float (&v)[R]) {
    float m = 0.0f;
#pragma unroll
    for (int r = 0; r < R; r += 2)
        m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(fabsf(v[r]), fabsf(v[r + 1])), m);
    m = __builtin_elementwise_maximum(m, lane_xor<1>(m));
    m = __builtin_elementwise_maximum(m, lane_xor<2>(m));
    m = __builtin_elementwise_maximum(m, lane_xor<4>(m));
    m = __builtin_elementwise_maximum(m, lane_xor<8>(m));
    const uint32_t u = __float_as_uint(m);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    m = __builtin_elementwise_maximum(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t w = __float_as_uint(m);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return __builtin_elementwise_maximum(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// s = fl32(m / 127), 1 where that is 0, NaN where m is not finite.
__device__ __forceinline__ float token_scale(float m) {
    const float s = m / 127.0f;
    return !(m < __builtin_inff()) ? __builtin_nanf("") : s == 0.0f ? 1.0f : s;
}

// Codes of one chunk, rne(fl32(sigma v / s)), as 8 bytes.  u = fl(v r + 1.5 2^23), r =
// sigma / s, rounds the exact product to the nearest integer k in one fma and d =
// fl(v r - k) in another; |v r - v / s| <= 127 2^-24, d is within 2^-25 of its exact
// value and fl(v / s) within 2^-18 of v / s, so |d| <= 0.5 - 2^-16 gives k = rne(fl(v /
// s)).  A chunk with an element nearer to a half-integer, and any with s outside
// [2^-125, 2^125] (`plain` false), divides.  Where s is NaN the codes are 0.
__device__ __forceinline__ uint2 token_codes8(const float *v, float sigma, float s, float r, bool plain) {
    uint32_t u[8];
    float m = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        float d[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float k = __builtin_fmaf(v[j + e], r, HATQ_MAGIC);
            u[j + e] = __float_as_uint(k);   // |v r| < 127.5: a code
            d[e] = __builtin_fmaf(v[j + e], r, -(k - HATQ_MAGIC));
        }
        m = fmaxf(fmaxf(fabsf(d[0]), fabsf(d[1])), m);
    }
    if (!(plain && m <= 0.5f - 0x1p-16f)) {
        asm volatile("");   // a branch: else the compiler divides for every chunk and selects
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float q = clamp127(rintf((sigma * v[j]) / s));
            u[j] = s == s ? (uint32_t)(int32_t)q : 0u;
        }
    }
    return make_uint2(pack_low_bytes(u[0], u[1], u[2], u[3]), pack_low_bytes(u[4], u[5], u[6], u[7]));
}
__device__ __forceinline__ bool token_plain(float s) { return s >= 0x1p-125f && s <= 0x1p125f; }

}  // namespace hatq
