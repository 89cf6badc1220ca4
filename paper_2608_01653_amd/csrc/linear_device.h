// Device-side element types of the linear layers over tokens (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

// Eight adjacent elements, 16-byte aligned.
__device__ __forceinline__ void load8(const float *p, float *v) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t *p, float *v) {
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const _Float16 *p, float *v) {
    typedef _Float16 v8h __attribute__((ext_vector_type(8)));
    const v8h h = *reinterpret_cast<const v8h *>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)h[j];
}

// Four adjacent elements, aligned to their size.
__device__ __forceinline__ void store4(float *p, const float *v) {
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store4(bf16_t *p, const float *v) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
}
__device__ __forceinline__ void store4(_Float16 *p, const float *v) {
    typedef _Float16 v4h __attribute__((ext_vector_type(4)));
    *reinterpret_cast<v4h *>(p) = v4h{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
}

// One 16-byte piece.
__device__ __forceinline__ void store16(float *p, const float *v) { store4(p, v); }
__device__ __forceinline__ void store16(bf16_t *p, const float *v) {
    *reinterpret_cast<uint4 *>(p) =
        make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}
__device__ __forceinline__ void store16(_Float16 *p, const float *v) {
    typedef _Float16 v8h __attribute__((ext_vector_type(8)));
    v8h h;
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = (_Float16)v[j];
    *reinterpret_cast<v8h *>(p) = h;
}

}  // namespace hatq
