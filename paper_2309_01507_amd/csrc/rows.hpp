// Elements of rows: vector types, and loads and stores of float32 and bf16 at any boundary.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lpmm {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---- elements ----------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }
template <bool BF16>
__device__ __forceinline__ float w4_load1(const void* p, int64_t i) {
    if constexpr (BF16) return __uint_as_float(uint32_t(static_cast<const uint16_t*>(p)[i]) << 16);
    else return static_cast<const float*>(p)[i];
}
template <bool BF16>
__device__ __forceinline__ void w4_store1(void* p, int64_t i, float v) {
    if constexpr (BF16) static_cast<uint16_t*>(p)[i] = to_bf16(v);
    else static_cast<float*>(p)[i] = v;
}

// 16 bytes at the alignment of an element: gfx950 reads and writes them in one piece wherever they lie
struct __attribute__((packed, aligned(2))) Vec16 { uint32_t v[4]; };
struct __attribute__((packed, aligned(4))) Vec16f { float v[4]; };

// 8 elements from p[i] on; those at or beyond `end` are 0 and not read
template <bool BF16>
__device__ __forceinline__ void w4_load8(const void* p, int64_t i, int64_t end, float out[8]) {
    if (i + 8 <= end) {
        if constexpr (BF16) {
            const Vec16 u = *reinterpret_cast<const Vec16*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                out[2 * e] = __uint_as_float(u.v[e] << 16);
                out[2 * e + 1] = __uint_as_float(u.v[e] & 0xFFFF0000u);
            }
        } else {
            const Vec16f a = *reinterpret_cast<const Vec16f*>(static_cast<const float*>(p) + i);
            const Vec16f b = *reinterpret_cast<const Vec16f*>(static_cast<const float*>(p) + i + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { out[e] = a.v[e]; out[4 + e] = b.v[e]; }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = i + e < end ? w4_load1<BF16>(p, i + e) : 0.0f;
    }
}

}  // namespace lpmm
