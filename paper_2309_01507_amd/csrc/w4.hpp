// Weights in 4 bits with group scales: compress, decompress, the product with them and its two gradients (format and
// formulas: include/lpmm4.h).
//
// E2M1 codes are exact in bf16 and gfx950 converts two of them with one instruction, so a product of bf16 inputs with codes
// goes through the matrix instructions without any rounding; the group's scale is applied to the group's fp32 sum.  fp32
// inputs are taken apart into three bf16 numbers that add up to them exactly, so the same instructions serve them at a third of the rate.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lpmm {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kW4Chunk = 128;            // codes of a row come in runs of 128: 16 words, 64 bytes

struct W4Mat {
    const uint32_t* codes;
    const float* scales;
    int n, k;
    int words;                           // of a row: kp / 8
    int groups;                          // of a row
};

// word d of a run of 128 stands at place (d % 4) * 4 + d / 4, and the word at place p is word (p % 4) * 4 + p / 4: its own inverse
__device__ __forceinline__ int w4_place(int d) { return (d & 3) * 4 + (d >> 2); }

// ---- elements ----------------------------------------------------------------------------------------------------------

template <bool BF16> struct W4Elem;
template <> struct W4Elem<true> { typedef uint16_t type; };
template <> struct W4Elem<false> { typedef float type; };

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

// ---- compress ----------------------------------------------------------------------------------------------------------

constexpr float kW4Least = 0x1p-100f;

// Maximum of unsigned words over the 4, 8 or 16 lanes of a group (all active)
template <int LANES>
__device__ __forceinline__ uint32_t group_umax(uint32_t x) {
    auto step = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    x = step(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0xB1, 0xF, 0xF, false)));      // lane ^ 1
    x = step(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x4E, 0xF, 0xF, false)));      // lane ^ 2
    if constexpr (LANES >= 8) x = step(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x141, 0xF, 0xF, false)));
    if constexpr (LANES >= 16) x = step(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x140, 0xF, 0xF, false)));
    return x;
}

// The largest float not above m * s: |w| > m * s holds exactly where |w| is larger than this.  (m s is within the normal range.)
__device__ __forceinline__ float w4_threshold(float m, float s) {
    const float p = m * s;
    return __builtin_fmaf(m, s, -p) < 0.0f ? __uint_as_float(__float_as_uint(p) - 1u) : p;
}

// A lane takes the 8 elements of one word; 16 lanes a run of 128.
template <bool BF16, int GROUP>
__global__ __launch_bounds__(256) void w4_quant_kernel(const void* w, int64_t w_stride, int n, int k, int runs, int groups,
                                                       uint32_t* codes, float* scales) {
    const uint32_t unit = blockIdx.x * 16u + (threadIdx.x >> 4);          // run of 128, counted over all rows
    const int row = int(unit / uint32_t(runs)), run = int(unit % uint32_t(runs)), d = threadIdx.x & 15;
    if (row >= n) return;                                                 // 16 lanes at a time
    const int at = run * kW4Chunk + d * 8;
    float x[8];
    w4_load8<BF16>(w, int64_t(row) * w_stride + at, int64_t(row) * w_stride + k, x);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t a = __float_as_uint(x[e]) & 0x7FFFFFFFu;           // magnitudes order like their bits, NaN above all
        top = a > top ? a : top;
    }
    top = group_umax<GROUP / 8>(top);
    float s = __uint_as_float(top) / 6.0f;
    if (top < __float_as_uint(kW4Least)) s = 0.0f;
    uint32_t word = 0;
    if (top >= 0x7F800000u) {
        s = __builtin_nanf("");
    } else if (s != 0.0f) {
        const float t0 = w4_threshold(0.25f, s), t1 = w4_threshold(0.75f, s), t2 = w4_threshold(1.25f, s),
                    t3 = w4_threshold(1.75f, s), t4 = w4_threshold(2.5f, s), t5 = w4_threshold(3.5f, s),
                    t6 = w4_threshold(5.0f, s);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = fabsf(x[e]);
            const bool c4 = a > t3;
            const bool c2 = a > (c4 ? t5 : t1);
            const bool c1 = a > (c4 ? (c2 ? t6 : t4) : (c2 ? t2 : t0));
            uint32_t c = (c4 ? 4u : 0u) + (c2 ? 2u : 0u) + (c1 ? 1u : 0u);
            if (c != 0) c |= (__float_as_uint(x[e]) >> 31) << 3;
            word |= c << (4 * e);
        }
    }
    codes[int64_t(unit) * 16 + w4_place(d)] = word;
    if (d % (GROUP / 8) == 0 && at < k) scales[int64_t(row) * groups + at / GROUP] = s;
}

// ---- decompress --------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void w4_values8(uint32_t word, float out[8]) {
    f32x2 v;
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 0); out[0] = v.x; out[1] = v.y;
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 1); out[2] = v.x; out[3] = v.y;
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 2); out[4] = v.x; out[5] = v.y;
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 3); out[6] = v.x; out[7] = v.y;
}

template <bool BF16>
__global__ __launch_bounds__(256) void w4_dequant_kernel(W4Mat m, int runs, int group_shift, void* w, int64_t w_stride) {
    const uint32_t unit = blockIdx.x * 16u + (threadIdx.x >> 4);
    const int row = int(unit / uint32_t(runs)), run = int(unit % uint32_t(runs)), d = threadIdx.x & 15;
    const int at = run * kW4Chunk + d * 8;
    if (row >= m.n || at >= m.k) return;
    float v[8];
    w4_values8(m.codes[int64_t(unit) * 16 + w4_place(d)], v);
    const float s = m.scales[int64_t(row) * m.groups + (at >> group_shift)];
    const int64_t base = int64_t(row) * w_stride + at;
    if (at + 8 <= m.k) {
        if constexpr (BF16) {
            Vec16 u;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                u.v[e] = uint32_t(to_bf16(v[2 * e] * s)) | uint32_t(to_bf16(v[2 * e + 1] * s)) << 16;
            *reinterpret_cast<Vec16*>(static_cast<uint16_t*>(w) + base) = u;
        } else {
            Vec16f a, b;
#pragma unroll
            for (int e = 0; e < 4; ++e) { a.v[e] = v[e] * s; b.v[e] = v[4 + e] * s; }
            *reinterpret_cast<Vec16f*>(static_cast<float*>(w) + base) = a;
            *reinterpret_cast<Vec16f*>(static_cast<float*>(w) + base + 4) = b;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < m.k) w4_store1<BF16>(w, base + e, v[e] * s);
    }
}

// ---- operands of the matrix instructions -----------------------------------------------------------------------------------

__device__ __forceinline__ bf16x8 w4_codes_bf16(uint32_t word) {
    union { bf16x2 h[4]; bf16x8 v; } u;
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.0f, 0);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.0f, 1);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.0f, 2);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.0f, 3);
    return u.v;
}

// A float as three bf16 numbers with that sum: the upper 8 bits of the significand, of what is left, and of what is left then (24
// bits in all), cut off, not rounded, so that nothing overflows.  Infinities and NaN stand in the first, with nothing left.
__device__ __forceinline__ void split3(float x, uint32_t out[3]) {
    const uint32_t hi = __float_as_uint(x) & 0xFFFF0000u;
    float r = x - __uint_as_float(hi);
    if ((hi & 0x7F800000u) == 0x7F800000u) r = 0.0f;
    const uint32_t mid = __float_as_uint(r) & 0xFFFF0000u;
    out[0] = hi | ((__float_as_uint(x) & 0xFFFFu) != 0 && (hi & 0x7FFFFFFFu) == 0x7F800000u ? 0x00400000u : 0u);   // a NaN stays one
    out[1] = mid;
    out[2] = __float_as_uint(r - __uint_as_float(mid)) & 0xFFFF0000u;
}

template <bool BF16> constexpr int kW4Terms = BF16 ? 1 : 3;

// 8 elements of a row as operands: elements at or beyond `end` are 0 and not read
template <bool BF16>
__device__ __forceinline__ void w4_operand8(const void* p, int64_t i, int64_t end, bf16x8 out[]) {
    if constexpr (BF16) {
        union { uint32_t w[4]; bf16x8 v; } u;
        if (i + 8 <= end) {
            const Vec16 q = *reinterpret_cast<const Vec16*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) u.w[e] = q.v[e];
        } else {
            const uint16_t* x = static_cast<const uint16_t*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = i + 2 * e < end ? x[i + 2 * e] : 0, hi = i + 2 * e + 1 < end ? x[i + 2 * e + 1] : 0;
                u.w[e] = lo | hi << 16;
            }
        }
        out[0] = u.v;
    } else {
        float x[8];
        w4_load8<false>(p, i, end, x);
        union { uint32_t w[4]; bf16x8 v; } u[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t a[3], b[3];
            split3(x[2 * e], a);
            split3(x[2 * e + 1], b);
#pragma unroll
            for (int j = 0; j < 3; ++j) u[j].w[e] = a[j] >> 16 | b[j];
        }
#pragma unroll
        for (int j = 0; j < 3; ++j) out[j] = u[j].v;
    }
}

// ---- y = x W^T ---------------------------------------------------------------------------------------------------------------
//
// A workgroup takes 16 rows of W and 16 tokens; its waves share the runs of 128 and add up in LDS.  A lane's 16 bytes of
// codes are its operands of four 16x16x32 products: lane l holds row l % 16, and its word s the elements 32 s + 8 (l / 16) .. + 7.
template <bool BF16, int GROUP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void w4_linear_kernel(W4Mat m, const void* x, int t, int64_t x_stride, void* y,
                                                               int64_t y_stride) {
    constexpr int TERMS = kW4Terms<BF16>;
    __shared__ f32x4 s_part[WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
    const int n = blockIdx.x * 16 + col, tok = blockIdx.y * 16 + col;
    const int row = n < m.n ? n : m.n - 1;
    const uint32_t* w = m.codes + int64_t(row) * m.words + quarter * 4;
    const float* sc = m.scales + int64_t(row) * m.groups;
    const int64_t x0 = int64_t(tok) * x_stride;
    f32x4 acc = {0, 0, 0, 0};
    for (int run = wave; run < m.words / 16; run += WAVES) {
        const uint4 q = *reinterpret_cast<const uint4*>(w + run * 16);
        const uint32_t words[4] = {q.x, q.y, q.z, q.w};
        f32x4 part = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int at = run * kW4Chunk + s * 32 + quarter * 8;
            bf16x8 a[TERMS] = {};
            if (tok < t) w4_operand8<BF16>(x, x0 + at, x0 + m.k, a);
            const bf16x8 b = w4_codes_bf16(words[s]);
#pragma unroll
            for (int j = 0; j < TERMS; ++j) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[j], b, part, 0, 0, 0);
            if ((s + 1) * 32 % GROUP == 0) {
                const int g = (run * kW4Chunk + s * 32) / GROUP;
                const float scale = g < m.groups ? sc[g] : 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] = __builtin_fmaf(scale, part[i], acc[i]);
                part = f32x4{0, 0, 0, 0};
            }
        }
    }
    s_part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int i = 1; i < WAVES; ++i) acc += s_part[i][lane];
        if (n < m.n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int tt = blockIdx.y * 16 + quarter * 4 + i;
                if (tt < t) w4_store1<BF16>(y, int64_t(tt) * y_stride + n, acc[i]);
            }
        }
    }
}

}  // namespace lpmm
