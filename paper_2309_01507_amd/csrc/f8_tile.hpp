// The product of two matrices in 8 bits: c[i][j] = sum_k a[i][k] b[j][k].
//
// Results of 16 bits: v_mfma_scale_f32_32x32x64_f8f6f4 multiplies codes and applies both blocks' powers.  It adds up the 64 products of a step
// with terms cut off some 2^-13 below the largest (measured: 1.5e-5 of the result's size, for every fp8 form), which is far below the
// half step of 2^-9 that rounding to bf16 costs.  Results of 32 bits: the codes times their powers become bf16, which holds them
// exactly, and v_mfma_f32_32x32x16_bf16 adds them up in fp32, at half the rate.
//
// Operand layout of v_mfma_scale_f32_32x32x64_f8f6f4: lane l holds, of row (A) or column (B) l % 32, 32 bytes of the half l / 32 of the
// reduction's 64, and the power of these (a byte of a register).  The result stands as that of v_mfma_f32_32x32x16_bf16 does.  Which of a
// block's elements meet in which step is free, as long as both operands agree.
#pragma once

#include "f8.hpp"
#include "tile.hpp"

namespace lpmm {

typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x16 mfma_f8(uint4 a0, uint4 a1, uint4 b0, uint4 b1, f32x16 c, int scale_a, int scale_b) {
    const i32x8 a = {int(a0.x), int(a0.y), int(a0.z), int(a0.w), int(a1.x), int(a1.y), int(a1.z), int(a1.w)};
    const i32x8 b = {int(b0.x), int(b0.y), int(b0.z), int(b0.w), int(b1.x), int(b1.y), int(b1.z), int(b1.w)};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, scale_a, 0, scale_b);
}

// 8 codes times their power as bf16
__device__ __forceinline__ bf16x8 f8_bf16(uint32_t lo, uint32_t hi, float power) {
    union { bf16x2 h[4]; bf16x8 v; } u;
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, false);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, true);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, false);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, true);
    return u.v;
}

// ROWS rows of a block of 128 codes (8 pieces of 16 bytes), loaded straight into LDS by WAVES waves.  Row r of LDS holds row
// of(r) of the tile: where EACH rows of 32 lanes make a wave's part, lane's row r % 32 of each is next to the others, so that a lane's results are
// neighbours.
template <int ROWS, int WAVES, int EACH>
struct StageF8 {
    static constexpr int kPieces = ROWS * 8, kOwn = kPieces / 64 / WAVES;
    static_assert(kPieces % (64 * WAVES) == 0 && ROWS % (32 * EACH) == 0, "whole KiB per wave");
    Buffer buffer;
    uint32_t off[kOwn];
    static __device__ __forceinline__ int of(int r) { return r / (32 * EACH) * (32 * EACH) + (r % 32) * EACH + r / 32 % EACH; }
    __device__ __forceinline__ void setup(const F8Mat& m, int first, int wave) {
        const int lane = threadIdx.x & 63, rows = min(m.rows - first, ROWS);
        buffer.set(m.codes + int64_t(first) * m.bytes, int64_t(rows) * m.bytes);
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            const int r = (j * WAVES + wave) * 8 + (lane >> 3), o = lane & 7;
            off[j] = uint32_t(of(r)) * uint32_t(m.bytes) + uint32_t(lds_piece<3>(r, o) - r * 8) * 16;
        }
    }
    __device__ __forceinline__ void load(int at, uint4* lds, int wave) const {
#pragma unroll
        for (int j = 0; j < kOwn; ++j) buffer.to_lds16(off[j], at, lds + (j * WAVES + wave) * 64);
    }
};

// EACH neighbouring results of a row, those before `left`
template <bool BF16, int EACH>
__device__ __forceinline__ void f8_store(void* out, int64_t at, int left, const float v[EACH]) {
    if (left >= EACH) {
        if constexpr (BF16) {
            struct __attribute__((packed, aligned(2))) Pack { uint16_t v[EACH]; } u;
#pragma unroll
            for (int e = 0; e < EACH; ++e) u.v[e] = to_bf16(v[e]);
            *reinterpret_cast<Pack*>(static_cast<uint16_t*>(out) + at) = u;
        } else {
            struct __attribute__((packed, aligned(4))) Pack { float v[EACH]; } u;
#pragma unroll
            for (int e = 0; e < EACH; ++e) u.v[e] = v[e];
            *reinterpret_cast<Pack*>(static_cast<float*>(out) + at) = u;
        }
    } else {
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (e < left) w4_store1<BF16>(out, at + e, v[e]);
    }
}

// A workgroup of WM x WN waves takes WM MT 32 rows of a and WN NT 32 rows of b; blocks of 128 go through LDS, one ahead.  FAST: results of 16
// bits.  blockIdx.y: which of the reduction's parts of `per` blocks; their sums go to parts[y][row][column] as fp32 where there are several.
template <bool FAST, bool BF16, int WM, int WN, int MT, int NT>
__global__ __launch_bounds__(64 * WM * WN, 2) void f8_tile_kernel(F8Mat a, F8Mat b, void* c, int64_t stride, int m_tiles, int n_tiles, int per, float* parts) {
    constexpr int BM = WM * MT * 32, BN = WN * NT * 32, WAVES = WM * WN;
    typedef StageF8<BM, WAVES, 1> StageA;
    typedef StageF8<BN, WAVES, NT> StageB;
    __shared__ uint4 s_a0[StageA::kPieces], s_a1[StageA::kPieces];
    __shared__ uint4 s_b0[StageB::kPieces], s_b1[StageB::kPieces];
    int m_tile, n_tile;
    if (!tile_of(blockIdx.x, m_tiles, n_tiles, m_tile, n_tile)) return;
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, half = lane >> 5;
    const int m0 = m_tile * BM, n0 = n_tile * BN, mw = (wave % WM) * MT * 32, nw = (wave / WM) * NT * 32;
    StageA stage_a;
    StageB stage_b;
    stage_a.setup(a, m0, wave);
    stage_b.setup(b, n0, wave);
    const uint8_t* scale_a[MT];
    const uint8_t* scale_b[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) scale_a[i] = a.scales + int64_t(min(m0 + mw + i * 32 + col, a.rows - 1) >> a.shift) * a.scale_bytes;
#pragma unroll
    for (int j = 0; j < NT; ++j) scale_b[j] = b.scales + int64_t(min(n0 + nw + col * NT + j, b.rows - 1) >> b.shift) * b.scale_bytes;
    const int blocks = a.bytes / kF8Block, first = blockIdx.y * per, last = min(blocks, first + per);
    f32x16 acc[MT][NT] = {};
    uint32_t sa[MT], sb[NT], sa_next[MT], sb_next[NT];
    auto load_scales = [&](int block) {
#pragma unroll
        for (int i = 0; i < MT; ++i) sa_next[i] = scale_a[i][block];
#pragma unroll
        for (int j = 0; j < NT; ++j) sb_next[j] = scale_b[j][block];
    };
    auto step = [&](bool more, int block, const uint4* now_a, const uint4* now_b, uint4* next_a, uint4* next_b) {
#pragma unroll
        for (int i = 0; i < MT; ++i) sa[i] = sa_next[i];
#pragma unroll
        for (int j = 0; j < NT; ++j) sb[j] = sb_next[j];
        if (more) {
            stage_a.load((block + 1) * kF8Block, next_a, wave);
            stage_b.load((block + 1) * kF8Block, next_b, wave);
            load_scales(block + 1);
        }
        if constexpr (FAST) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                uint4 vb[NT][2];
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 2; ++q) vb[j][q] = now_b[lds_piece<3>(nw + j * 32 + col, s * 4 + q * 2 + half)];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const uint4 v0 = now_a[lds_piece<3>(mw + i * 32 + col, s * 4 + half)], v1 = now_a[lds_piece<3>(mw + i * 32 + col, s * 4 + 2 + half)];
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = mfma_f8(v0, v1, vb[j][0], vb[j][1], acc[i][j], int(sa[i]), int(sb[j]));
                }
            }
        } else {
            float pa[MT], pb[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) pa[i] = f8_power(sa[i]);
#pragma unroll
            for (int j = 0; j < NT; ++j) pb[j] = f8_power(sb[j]);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                uint4 vb[NT];
                bf16x8 xb[NT][2];
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    vb[j] = now_b[lds_piece<3>(nw + j * 32 + col, 2 * s + half)];
                    xb[j][0] = f8_bf16(vb[j].x, vb[j].y, pb[j]);
                    xb[j][1] = f8_bf16(vb[j].z, vb[j].w, pb[j]);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const uint4 v = now_a[lds_piece<3>(mw + i * 32 + col, 2 * s + half)];
                    const bf16x8 x0 = f8_bf16(v.x, v.y, pa[i]), x1 = f8_bf16(v.z, v.w, pa[i]);
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        acc[i][j] = mfma32(x0, xb[j][0], acc[i][j]);
                        acc[i][j] = mfma32(x1, xb[j][1], acc[i][j]);
                    }
                }
            }
        }
        __syncthreads();
    };
    if (first < last) {
        stage_a.load(first * kF8Block, s_a0, wave);
        stage_b.load(first * kF8Block, s_b0, wave);
        load_scales(first);
    }
    __syncthreads();
    int block = first;
    for (; block + 2 < last; block += 2) {
        step(true, block, s_a0, s_b0, s_a1, s_b1);
        step(true, block + 1, s_a1, s_b1, s_a0, s_b0);
    }
    if (block < last) step(block + 1 < last, block, s_a0, s_b0, s_a1, s_b1);
    if (block + 1 < last) step(false, block + 1, s_a1, s_b1, s_a0, s_b0);
    const int n = n0 + nw + col * NT;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int m = m0 + mw + i * 32 + mfma32_row(e, half);
            float v[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) v[j] = acc[i][j][e];
            if (m < a.rows) {
                if (parts) f8_store<false, NT>(parts, (int64_t(blockIdx.y) * a.rows + m) * b.rows + n, b.rows - n, v);
                else f8_store<BF16, NT>(c, int64_t(m) * stride + n, b.rows - n, v);
            }
        }
}

// The parts' sums, in the order of the parts
template <bool BF16>
__global__ __launch_bounds__(256) void f8_join_kernel(const float* parts, int count, int rows, int cols, void* c, int64_t stride) {
    const int64_t all = int64_t(rows) * cols, at = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (at >= all) return;
    float v = parts[at];
    for (int p = 1; p < count; ++p) v += parts[p * all + at];
    w4_store1<BF16>(c, at / cols * stride + at % cols, v);
}

// ---- few tokens --------------------------------------------------------------------------------------------------------------------
//
// Operand layout of v_mfma_scale_f32_16x16x128_f8f6f4: lane l holds, of row (A) or column (B) l % 16, 32 bytes of the quarter l / 16 of the
// reduction's 128; of the result column l % 16, rows 4 (l / 16) + i for i = 0..3.
__device__ __forceinline__ f32x4 mfma16_f8(const uint32_t a[8], const uint32_t b[8], f32x4 c, int scale_a, int scale_b) {
    const i32x8 va = {int(a[0]), int(a[1]), int(a[2]), int(a[3]), int(a[4]), int(a[5]), int(a[6]), int(a[7])};
    const i32x8 vb = {int(b[0]), int(b[1]), int(b[2]), int(b[3]), int(b[4]), int(b[5]), int(b[6]), int(b[7])};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 0, 0, 0, scale_a, 0, scale_b);
}

// y = x W^T for at most 16 tokens: a workgroup takes NT 16 rows of W, its waves every WAVES-th block.  x comes as it is and is brought to 8 bits in the
// registers that are the operand: a block of a token lies in 4 lanes.  FAST goes with BF16.
template <bool BF16, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void f8_few_kernel(F8Mat w, const void* x, int t, int k, int64_t x_stride, void* y, int64_t y_stride) {
    __shared__ float s_sum[WAVES][NT * 4 * 64];
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 15, quarter = lane >> 4;
    const int n0 = blockIdx.x * NT * 16, blocks = w.bytes / kF8Block;
    const uint8_t* codes[NT];
    const uint8_t* scales[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n = min(n0 + j * 16 + col, w.rows - 1);
        codes[j] = w.codes + int64_t(n) * w.bytes + quarter * 32;
        scales[j] = w.scales + int64_t(n >> w.shift) * w.scale_bytes;
    }
    const int64_t row = int64_t(col) * x_stride;
    uint4 q[NT][2];
    uint32_t sc[NT];
    float v[32];
    auto load = [&](int block) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            q[j][0] = *reinterpret_cast<const uint4*>(codes[j] + int64_t(block) * kF8Block);
            q[j][1] = *reinterpret_cast<const uint4*>(codes[j] + int64_t(block) * kF8Block + 16);
            sc[j] = scales[j][block];
        }
        const int at = block * kF8Block + quarter * 32;
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            if (col < t && at + o * 8 < k) {
                w4_load8<BF16>(x, row + at + o * 8, row + k, v + o * 8);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[o * 8 + e] = 0.0f;
            }
        }
    };
    f32x4 acc[NT] = {};
    for (int block = wave; block < blocks; block += WAVES) {
        load(block);
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 32; ++e) top = umax32(top, f8_magnitude(v[e]));
        top = umax32(top, __shfl_xor(top, 16, 64));
        top = umax32(top, __shfl_xor(top, 32, 64));
        const uint32_t scale = f8_scale(top);
        const float inverse = f8_inverse(scale);
        uint32_t xa[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) xa[e] = f8_codes4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3], inverse);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const uint32_t wb[8] = {q[j][0].x, q[j][0].y, q[j][0].z, q[j][0].w, q[j][1].x, q[j][1].y, q[j][1].z, q[j][1].w};
            if constexpr (BF16) {
                acc[j] = mfma16_f8(xa, wb, acc[j], int(scale), int(sc[j]));
            } else {
                const float px = f8_power(scale), pw = f8_power(sc[j]);
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f8_bf16(xa[2 * s], xa[2 * s + 1], px), f8_bf16(wb[2 * s], wb[2 * s + 1], pw), acc[j], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) s_sum[wave][(j * 4 + i) * 64 + lane] = acc[j][i];
    __syncthreads();
    for (int id = threadIdx.x; id < NT * 256; id += 64 * WAVES) {
        float sum = s_sum[0][id];
#pragma unroll
        for (int o = 1; o < WAVES; ++o) sum += s_sum[o][id];
        const int j = id >> 8, i = id >> 6 & 3, n = n0 + j * 16 + (id & 15), tok = 4 * (id >> 4 & 3) + i;
        if (n < w.rows && tok < t) w4_store1<BF16>(y, int64_t(tok) * y_stride + n, sum);
    }
}

}  // namespace lpmm
