// Matrices in 8-bit floating point with a power of two for each block of 128: bringing them there and back, for the rows of a matrix,
// for its transpose, or both from one reading (format and formulas: include/lpmm4.h).
//
// The power is found from the bits of the block's largest element, and multiplying by it is exact, so the rounding to E4M3 by the
// hardware's conversion is the only one.
#pragma once

#include "rows.hpp"

namespace lpmm {

constexpr int kF8Block = 128;

struct F8Mat {
    const uint8_t* codes;
    const uint8_t* scales;
    int rows;
    int bytes;                           // of a row of codes: columns rounded up to whole blocks
    int shift;                           // log2 of the rows of a block: 0 or 7
    // Scales of blocks of one row stand next to those of the rows below, so that a wave's operand finds its own in one line; those of blocks of 128
    // rows next to those of the blocks to the right.
    int scale_bytes;                     // of a row of scales
    __host__ __device__ __forceinline__ int64_t scale_at(int row, int block) const {
        return shift == 0 ? int64_t(block) * scale_bytes + row : int64_t(row >> shift) * scale_bytes + block;
    }
};

// ---- scales ------------------------------------------------------------------------------------------------------------------------

// A magnitude's bits for the block's maximum: what is not finite does not count
__device__ __forceinline__ uint32_t f8_magnitude(float x) {
    const uint32_t a = __float_as_uint(x) & 0x7FFFFFFFu;
    return a < 0x7F800000u ? a : 0u;
}
// exponent + 127 of the least power of two that brings `top` to at most 448 = 1.75 * 2^8
__device__ __forceinline__ uint32_t f8_scale(uint32_t top) {
    const int e = int((top + 0x1FFFFFu) >> 23) - 8;
    return e > 0 ? uint32_t(e) : 0u;
}
__device__ __forceinline__ float f8_inverse(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }
__device__ __forceinline__ float f8_power(uint32_t scale) { return __uint_as_float(scale ? scale << 23 : 0x00400000u); }

// Codes of 4 values times `inverse`.  Infinities, for which there is no code, become NaN.
__device__ __forceinline__ uint32_t f8_codes4(float a, float b, float c, float d, float inverse) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, w, true);
    return uint32_t(w);
}

__device__ __forceinline__ uint32_t umax32(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Maximum over groups of 16 lanes
__device__ __forceinline__ uint32_t umax16(uint32_t x) {
    x = umax32(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0xB1, 0xF, 0xF, false)));      // lane ^ 1
    x = umax32(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x4E, 0xF, 0xF, false)));      // lane ^ 2
    x = umax32(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x141, 0xF, 0xF, false)));     // mirrored among 8
    x = umax32(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x140, 0xF, 0xF, false)));     // and 16
    return x;
}

// The largest finite magnitude's bits of a block that 16 lanes hold: all lanes look at what is not finite only where there is such
__device__ __forceinline__ uint32_t f8_top16(const float v[8]) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = umax32(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    top = umax16(top);
    if (top >= 0x7F800000u) {
        top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = umax32(top, f8_magnitude(v[e]));
        top = umax16(top);
    }
    return top;
}

// ---- to 8 bits ---------------------------------------------------------------------------------------------------------------------

// Blocks of 1 x 128: 16 lanes a block, 8 elements each; a wave takes four blocks of a row, a workgroup of four rows, and goes on to others where a launch cannot have so many.
// rows_up: rows rounded up to a multiple of 4, so that the rest of a row of scales is written too.  Bound by memory: 4096 x 11008 bf16 27.5 us, 4.9
// TB/s, of inputs that no cache holds, 22.9 of one that was just read.
template <bool BF16>
__global__ __launch_bounds__(256) void f8_quant_kernel(const void* x, int64_t stride, int rows, int cols, int blocks, uint8_t* codes, uint8_t* scales,
                                                       int rows_up) {
    const uint32_t across = uint32_t(blocks + 3) >> 2, groups = uint32_t(rows_up >> 2) * across;
    const int d = threadIdx.x & 15;
    for (uint32_t group = blockIdx.x; group < groups; group += gridDim.x) {
        const int row = int(group / across) * 4 + (threadIdx.x >> 6), block = int(group % across) * 4 + (threadIdx.x >> 4 & 3);
        if (block >= blocks) continue;                                    // 16 lanes at a time
        if (row >= rows) {
            if (d == 0) scales[int64_t(block) * rows_up + row] = 0;
            continue;
        }
        const int at = block * kF8Block + d * 8;
        float v[8];
        w4_load8<BF16>(x, int64_t(row) * stride + at, int64_t(row) * stride + cols, v);
        const uint32_t scale = f8_scale(f8_top16(v));
        const float inverse = f8_inverse(scale);
        uint2 w;
        w.x = f8_codes4(v[0], v[1], v[2], v[3], inverse);
        w.y = f8_codes4(v[4], v[5], v[6], v[7], inverse);
        *reinterpret_cast<uint2*>(codes + (int64_t(row) * blocks + block) * kF8Block + d * 8) = w;
        if (d == 0) scales[int64_t(block) * rows_up + row] = uint8_t(scale);
    }
}

// A tile of 128 x 128 a workgroup, for 128 x 128 blocks and for a matrix together with its transpose.  A thread takes 8 rows by 8
// columns: the maxima of rows, columns or all go over lanes and LDS, the transposed codes through LDS, 8 rows a piece.
// TILE: rows of a block, 1 or 128.  codes or codes_t may be null.  Bound by memory: 4096 x 11008 bf16 and its transpose 50 us, 3.6 TB/s, of inputs
// that no cache holds (a workgroup loads, waits, writes and ends), 37.6 of one that was just written; 4096 x 4096 fp32 in blocks of 128 x 128 18.2 us, 4.6 TB/s, and 16.9.
template <bool BF16, int TILE>
__global__ __launch_bounds__(256) void f8_quant_tile_kernel(const void* x, int64_t stride, int rows, int cols, int across, uint8_t* codes, uint8_t* scales,
                                                            int code_bytes, int scale_bytes, uint8_t* codes_t, uint8_t* scales_t, int code_bytes_t,
                                                            int scale_bytes_t) {
    __shared__ uint32_t s_top[4][kF8Block];
    __shared__ uint2 s_codes[kF8Block * 16];                              // [column][8 rows a piece]
    const int p = threadIdx.x & 15, g = threadIdx.x >> 4, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int block_r = int(blockIdx.x) / across, block_c = int(blockIdx.x) - block_r * across, r0 = block_r * kF8Block + g * 8, c0 = block_c * kF8Block + p * 8;
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + i < rows) {
            w4_load8<BF16>(x, int64_t(r0 + i) * stride + c0, int64_t(r0 + i) * stride + cols, v[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
        }
    }
    uint32_t row_scale[8], col_scale[8];
    if constexpr (TILE == 1) {
        uint32_t col_top[8] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t a = f8_magnitude(v[i][e]);
                top = umax32(top, a);
                col_top[e] = umax32(col_top[e], a);
            }
            row_scale[i] = f8_scale(umax16(top));
        }
        if (codes_t) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                col_top[e] = umax32(col_top[e], __shfl_xor(col_top[e], 16, 64));
                col_top[e] = umax32(col_top[e], __shfl_xor(col_top[e], 32, 64));
            }
            if (lane < 16) {
#pragma unroll
                for (int e = 0; e < 8; ++e) s_top[wave][p * 8 + e] = col_top[e];
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint32_t top = 0;
#pragma unroll
                for (int w = 0; w < 4; ++w) top = umax32(top, s_top[w][p * 8 + e]);
                col_scale[e] = f8_scale(top);
            }
        }
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = umax32(top, f8_magnitude(v[i][e]));
        top = umax16(top);
        top = umax32(top, __shfl_xor(top, 16, 64));
        top = umax32(top, __shfl_xor(top, 32, 64));
        if (lane == 0) s_top[0][wave] = top;
        __syncthreads();
        top = umax32(umax32(s_top[0][0], s_top[0][1]), umax32(s_top[0][2], s_top[0][3]));
#pragma unroll
        for (int i = 0; i < 8; ++i) row_scale[i] = col_scale[i] = f8_scale(top);
    }
    if (codes) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i >= rows) break;
            const float inverse = f8_inverse(row_scale[i]);
            uint2 w;
            w.x = f8_codes4(v[i][0], v[i][1], v[i][2], v[i][3], inverse);
            w.y = f8_codes4(v[i][4], v[i][5], v[i][6], v[i][7], inverse);
            *reinterpret_cast<uint2*>(codes + int64_t(r0 + i) * code_bytes + c0) = w;
            if (TILE == 1 && p == 0) scales[int64_t(block_c) * scale_bytes + r0 + i] = uint8_t(row_scale[i]);
        }
        if (TILE == 1 && p == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r0 + i >= rows && r0 + i < scale_bytes) scales[int64_t(block_c) * scale_bytes + r0 + i] = 0;
        }
        if (TILE > 1 && g == 0) {
            if (p == 0) scales[int64_t(block_r) * scale_bytes + block_c] = uint8_t(row_scale[0]);
            else if (block_c == across - 1 && block_c + p < scale_bytes) scales[int64_t(block_r) * scale_bytes + block_c + p] = 0;
        }
    }
    if (codes_t) {
        // piece g of column c at g ^ (c / 8): the 16 lanes of a store hit all banks
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float inverse = f8_inverse(col_scale[e]);
            uint2 w;
            w.x = f8_codes4(v[0][e], v[1][e], v[2][e], v[3][e], inverse);
            w.y = f8_codes4(v[4][e], v[5][e], v[6][e], v[7][e], inverse);
            s_codes[(p * 8 + e) * 16 + (g ^ p)] = w;
        }
        if (TILE == 1 && g == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c0 + e < scale_bytes_t) scales_t[int64_t(block_r) * scale_bytes_t + c0 + e] = uint8_t(c0 + e < cols ? col_scale[e] : 0u);
        }
        if (TILE > 1 && g == 0) {
            if (p == 0) scales_t[int64_t(block_c) * scale_bytes_t + block_r] = uint8_t(col_scale[0]);
            else if ((block_r + 1) * kF8Block >= rows && block_r + p < scale_bytes_t) scales_t[int64_t(block_c) * scale_bytes_t + block_r + p] = 0;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int id = threadIdx.x + j * 256, c = id >> 3, q = id & 7;          // 16 rows of a column
            if (block_c * kF8Block + c >= cols) continue;
            const uint2 a = s_codes[c * 16 + ((2 * q) ^ (c >> 3))], b = s_codes[c * 16 + ((2 * q + 1) ^ (c >> 3))];
            *reinterpret_cast<uint4*>(codes_t + int64_t(block_c * kF8Block + c) * code_bytes_t + block_r * kF8Block + q * 16) = make_uint4(a.x, a.y, b.x, b.y);
        }
    }
}

// ---- and back ----------------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void f8_values4(uint32_t w, float power, float out[4]) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), true);
    out[0] = lo.x * power; out[1] = lo.y * power; out[2] = hi.x * power; out[3] = hi.y * power;
}

// 16 lanes a block: 8 neighbours each, in fp32 two times 4, so that a wave's stores of 16 bytes are next to each other.  Bound by memory: 4096 x 11008 to bf16
// 26.9 us, 5.0 TB/s, of codes that no cache holds, 22.3 of those just written.
template <bool BF16>
__global__ __launch_bounds__(256) void f8_dequant_kernel(F8Mat m, int cols, int blocks, void* out, int64_t stride) {
    const uint32_t unit = blockIdx.x * 16u + (threadIdx.x >> 4);
    const int row = int(unit / uint32_t(blocks)), block = int(unit % uint32_t(blocks)), d = threadIdx.x & 15;
    if (row >= m.rows) return;
    const float power = f8_power(m.scales[m.scale_at(row, block)]);
    const uint8_t* codes = m.codes + int64_t(unit) * kF8Block;
    constexpr int STEP = BF16 ? 8 : 4;
#pragma unroll
    for (int part = 0; part < 8 / STEP; ++part) {
        const int in = part * 64 + d * STEP, at = block * kF8Block + in;
        if (at >= cols) continue;
        const int64_t base = int64_t(row) * stride + at;
        float v[8];
        if constexpr (BF16) {
            const uint2 w = *reinterpret_cast<const uint2*>(codes + in);
            f8_values4(w.x, power, v);
            f8_values4(w.y, power, v + 4);
        } else {
            f8_values4(*reinterpret_cast<const uint32_t*>(codes + in), power, v);
        }
        if (at + STEP <= cols) {
            if constexpr (BF16) {
                Vec16 u;
#pragma unroll
                for (int e = 0; e < 4; ++e) u.v[e] = uint32_t(to_bf16(v[2 * e])) | uint32_t(to_bf16(v[2 * e + 1])) << 16;
                *reinterpret_cast<Vec16*>(static_cast<uint16_t*>(out) + base) = u;
            } else {
                Vec16f u;
#pragma unroll
                for (int e = 0; e < 4; ++e) u.v[e] = v[e];
                *reinterpret_cast<Vec16f*>(static_cast<float*>(out) + base) = u;
            }
        } else {
#pragma unroll
            for (int e = 0; e < STEP; ++e)
                if (at + e < cols) w4_store1<BF16>(out, base + e, v[e]);
        }
    }
}

}  // namespace lpmm
