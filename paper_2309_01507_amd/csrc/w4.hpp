// Weights in 4 bits with group scales: compress, decompress, the product with them and its two gradients (format and
// formulas: include/lpmm4.h).
//
// E2M1 codes are exact in bf16 and gfx950 converts two of them with one instruction, so a product of bf16 inputs with codes
// goes through the matrix instructions without any rounding; the group's scale is applied to the group's fp32 sum.  fp32
// inputs are taken apart into three bf16 numbers that add up to them, so the same instructions serve them at a third of the rate.
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

// A lane takes the 8 elements of one word, 16 lanes a run of 128: the group's maximum is a butterfly over 4 to 16 of them and w is read once.  Bound
// by memory: 32000 x 4096 fp32, groups of 128: 117 us, 5.1 TB/s (call after call from a graph; between other kernels, in front of a profiler, 143); 1024 x 50257
// bf16, groups of 32: 39 us, 3.5 TB/s (rows off 16-byte boundaries, and
// the eight exact comparisons of an element).
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

// A lane writes the 8 values of one word.  Bound by memory: 32000 x 4096 fp32 115 us, 5.2 TB/s (between other kernels 127);
// 1024 x 50257 bf16 22 us, 6.2 TB/s.
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

// Floats as three bf16 numbers each with that sum, exactly from 2^-110 on (below, within the least bf16 number): the value rounded to 8 bits of significand, what is left (at most 16 bits)
// rounded to 8, and what is left then.  Two at a time, packed.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2 p = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ void split3_pair(float a, float b, uint32_t out[3]) {
    out[0] = pack_bf16(a, b);
    a -= low_bf16(out[0]);
    b -= high_bf16(out[0]);
    out[1] = pack_bf16(a, b);
    out[2] = pack_bf16(a - low_bf16(out[1]), b - high_bf16(out[1]));
}
// The same where values may be too large to round up, infinite or NaN: cut off instead of rounded, nothing left of what is not finite
__device__ __forceinline__ void split3_any(float x, uint32_t out[3]) {
    const uint32_t hi = __float_as_uint(x) & 0xFFFF0000u;
    const bool finite = (hi & 0x7F800000u) != 0x7F800000u;
    const float r = finite ? x - __uint_as_float(hi) : 0.0f;
    const uint32_t mid = __float_as_uint(r) & 0xFFFF0000u;
    out[0] = hi | (!finite && (__float_as_uint(x) & 0xFFFFu) != 0 ? 0x00400000u : 0u);       // a NaN stays one
    out[1] = mid;
    out[2] = __float_as_uint(r - __uint_as_float(mid)) & 0xFFFF0000u;
}
// 8 floats as words of 2 for each of the three terms
__device__ __forceinline__ void split3_8(const float x[8], uint32_t out[3][4]) {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t a = __float_as_uint(x[e]) & 0x7FFFFFFFu;
        most = a > most ? a : most;
    }
    if (__builtin_expect(most < 0x7F000000u, 1)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t w[3];
            split3_pair(x[2 * e], x[2 * e + 1], w);
#pragma unroll
            for (int j = 0; j < 3; ++j) out[j][e] = w[j];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t a[3], b[3];
            split3_any(x[2 * e], a);
            split3_any(x[2 * e + 1], b);
#pragma unroll
            for (int j = 0; j < 3; ++j) out[j][e] = a[j] >> 16 | b[j];
        }
    }
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
        uint32_t w[3][4];
        split3_8(x, w);
#pragma unroll
        for (int j = 0; j < 3; ++j) out[j] = __builtin_bit_cast(bf16x8, make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]));
    }
}

// ---- y = x W^T ---------------------------------------------------------------------------------------------------------------
//
// At most 16 MT tokens.  A workgroup takes tiles of 16 rows of W, one after the other; its waves share the runs of 128 in pieces of A next to each
// other and add up in LDS.  A lane's 16 bytes of codes are its operands of four 16x16x32 products: lane l holds row l % 16, and its word s
// the elements 32 s + 8 (l / 16) .. + 7.  The operands of x stay in registers from tile to tile where the waves cover a row at once
// (K <= 128 A WAVES); the next tile's codes are requested before this one's are used (EARLY: where registers
// hold them).  Bound by the latency of one round trip for few tiles (1 x 4096 x 4096 bf16, groups of 128: 4.9 us, 1.8 TB/s; 16 tokens 7.3; beyond what
// the registers hold of a row x is read again for each chunk: 7 x 4096 x 11008 10.9 us), by reading the codes for many (7 x 32000 x 4096, groups of 64: 18 to 19 us,
// 3.9 TB/s).  fp32 holds three terms of x: with a
// row of them in registers nothing is read ahead and some spill, 53 us there (groups of 128 33), with one run a wave x is read again for each tile, 67.  (bf16 in groups of
// 32 with two runs a wave spills 6.)
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));      // 16 and 8 bytes at the alignment of a float
typedef float f32x2u __attribute__((ext_vector_type(2), aligned(4)));

template <bool BF16, int GROUP, int MT, int WAVES, int A, int SIMD_WAVES, bool EARLY>
__global__ __launch_bounds__(64 * WAVES, SIMD_WAVES) void w4_linear_kernel(W4Mat m, const void* x, int t, int64_t x_stride, void* y,
                                                                  int64_t y_stride) {
    constexpr int TERMS = kW4Terms<BF16>, GROUPS = kW4Chunk / GROUP, SCALES = GROUPS * A;
    __shared__ f32x4 s_part[2][WAVES][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
    const int tiles = (m.n + 15) >> 4, runs = m.words / 16;
    const int chunks = (runs + WAVES * A - 1) / (WAVES * A);
    uint4 q[A];
    float sc[SCALES];
    auto load_w = [&](int tile, int chunk) {
        const int row = min(tile * 16 + col, m.n - 1), run0 = (chunk * WAVES + wave) * A;
        const uint32_t* w = m.codes + int64_t(row) * m.words + quarter * 4;
        const float* scale = m.scales + int64_t(row) * m.groups;
        const int g0 = run0 * GROUPS;
#pragma unroll
        for (int u = 0; u < A; ++u) q[u] = run0 + u < runs ? *reinterpret_cast<const uint4*>(w + (run0 + u) * 16) : make_uint4(0, 0, 0, 0);
        if (g0 + SCALES <= m.groups) {
            if constexpr (SCALES >= 4) {
#pragma unroll
                for (int i = 0; i < SCALES; i += 4) {
                    const f32x4u v = *reinterpret_cast<const f32x4u*>(scale + g0 + i);
                    sc[i] = v.x; sc[i + 1] = v.y; sc[i + 2] = v.z; sc[i + 3] = v.w;
                }
            } else if constexpr (SCALES == 2) {
                const f32x2u v = *reinterpret_cast<const f32x2u*>(scale + g0);
                sc[0] = v.x; sc[1] = v.y;
            } else {
                sc[0] = scale[g0];
            }
        } else {
#pragma unroll
            for (int i = 0; i < SCALES; ++i) sc[i] = g0 + i < m.groups ? scale[g0 + i] : 0.0f;
        }
    };
    bf16x8 a[A][4][MT][TERMS];
    auto load_x = [&](int chunk) {
#pragma unroll
        for (int u = 0; u < A; ++u)
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int b = 0; b < MT; ++b) {
                    const int at = ((chunk * WAVES + wave) * A + u) * kW4Chunk + s * 32 + quarter * 8, tok = b * 16 + col;
#pragma unroll
                    for (int j = 0; j < TERMS; ++j) a[u][s][b][j] = bf16x8{};
                    if (tok < t && at < m.k) w4_operand8<BF16>(x, int64_t(tok) * x_stride + at, int64_t(tok) * x_stride + m.k, a[u][s][b]);
                }
    };
    f32x4 acc[MT] = {};
    int tile = blockIdx.x, chunk = 0, buffer = 0;
    load_w(tile, 0);
    load_x(0);
    while (true) {
        uint4 q_now[A];
        float sc_now[SCALES];
#pragma unroll
        for (int u = 0; u < A; ++u) q_now[u] = q[u];
#pragma unroll
        for (int i = 0; i < SCALES; ++i) sc_now[i] = sc[i];
        const bool end = chunk + 1 == chunks;
        const int next = end ? tile + int(gridDim.x) : tile, next_chunk = end ? 0 : chunk + 1;
        if (EARLY && next < tiles) load_w(next, next_chunk);
#pragma unroll
        for (int u = 0; u < A; ++u) {
            const uint32_t words[4] = {q_now[u].x, q_now[u].y, q_now[u].z, q_now[u].w};
            f32x4 part[MT];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const bf16x8 v = w4_codes_bf16(words[s]);
#pragma unroll
                for (int b = 0; b < MT; ++b) {
                    if (s * 32 % GROUP == 0) part[b] = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < TERMS; ++j) part[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[u][s][b][j], v, part[b], 0, 0, 0);
                    if ((s + 1) * 32 % GROUP == 0) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[b][i] = __builtin_fmaf(sc_now[u * GROUPS + s * 32 / GROUP], part[b][i], acc[b][i]);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);         // codes of later runs are not converted ahead, into registers that are not there
        }
        if (!EARLY && next < tiles) load_w(next, next_chunk);
        if (chunks > 1 && next < tiles) load_x(next_chunk);
        if (end) {
#pragma unroll
            for (int b = 0; b < MT; ++b) {
                s_part[buffer][wave][b][lane] = acc[b];
                acc[b] = f32x4{0, 0, 0, 0};
            }
            __syncthreads();               // the other buffer is written next, and this one only behind the next barrier
            if (wave < MT) {               // a wave adds up 16 tokens
                f32x4 sum = s_part[buffer][0][wave][lane];
#pragma unroll
                for (int i = 1; i < WAVES; ++i) sum += s_part[buffer][i][wave][lane];
                const int n = tile * 16 + col;
                if (n < m.n) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int tok = wave * 16 + quarter * 4 + i;
                        if (tok < t) w4_store1<BF16>(y, int64_t(tok) * y_stride + n, sum[i]);
                    }
                }
            }
            buffer ^= 1;
        }
        if (next >= tiles) break;
        tile = next;
        chunk = next_chunk;
    }
}

}  // namespace lpmm
