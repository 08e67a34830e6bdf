// The product of two matrices in 8 bits: c[i][j] = sum_k a[i][k] b[j][k].
//
// Results of 16 bits: v_mfma_scale_f32_32x32x64_f8f6f4 multiplies codes and applies both blocks' powers.  It adds up eight neighbouring products at once, each cut off at 2^-13 of the
// largest 2^(ea + eb) among them (exponents of the codes, -6 for those below the normal numbers; measured, for v_mfma_scale_f32_16x16x128_f8f6f4 as well), and goes on in fp32.  That
// is at most 2^-10 of the products' magnitudes (2^-7 where the largest of eight has a code below the normal numbers); of normally distributed operands it takes 1.5e-5 of the result's
// norm, where rounding to bf16 takes 1.7e-3, and is taken for twice the rate.  Results of 32 bits: the codes times their powers become bf16, which holds them
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

// 32 codes, of two pieces
__device__ __forceinline__ i32x8 f8_operand(uint4 lo, uint4 hi) {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    return __builtin_shufflevector(__builtin_bit_cast(i32x4, lo), __builtin_bit_cast(i32x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ f32x16 mfma_f8(i32x8 a, i32x8 b, f32x16 c, int scale_a, int scale_b) {
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
    uint32_t off, step;                                        // of the first piece, and from one of the wave's pieces to the next
    static __device__ __forceinline__ int of(int r) { return r / (32 * EACH) * (32 * EACH) + (r % 32) * EACH + r / 32 % EACH; }
    __device__ __forceinline__ void setup(const F8Mat& m, int first, int wave) {
        const int lane = threadIdx.x & 63, rows = min(m.rows - first, ROWS), r = wave * 8 + (lane >> 3), o = lane & 7;
        buffer.set(m.codes + int64_t(first) * m.bytes, int64_t(rows) * m.bytes);
        off = uint32_t(of(r)) * uint32_t(m.bytes) + uint32_t(lds_piece<3>(r, o) - r * 8) * 16;
        step = uint32_t(m.bytes);
    }
    __device__ __forceinline__ void load(int at, uint4* lds, int wave) const {
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            // rows j * WAVES * 8 further on; the swizzle repeats every 16 rows
            static_assert(WAVES % 4 == 0, "whole parts of 32 rows");
            const int r = j * WAVES * 8;
            buffer.to_lds16(off + uint32_t(of_step(r, wave)) * step, at, lds + (j * WAVES + wave) * 64);
        }
    }
    // of(r + w) - of(w) for the wave's first row w, r a multiple of 32
    static __device__ __forceinline__ int of_step(int r, int wave) {
        const int w = wave * 8;
        return of(r + w) - of(w);
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
//
// Bound by the matrix unit and by what it waits for: from a graph of 20 calls 8192^3 to bf16 426 us, 2.6 PFLOP/s (with both operands kept in registers 275, with the meetings left out 356, with the loads
// left out 384); 4096 x 11008 x 4096 162 us, 2.28 PFLOP/s, and 168 to 195, behind the kernel that brings x to 8 bits, by the profiler; fp32 4096^3 110 us, 1.25 (the bf16 unit's half rate; a conversion for each 8 codes of each wave).  256 x 256 reads each
// code from LDS a fourth as often as it is multiplied with 64.  Codes go straight into LDS, one block ahead: through registers 64 x 64 tiles took 242 us for the first, and two
// blocks ahead, or halves of a block between meetings, spilled or gained nothing.  Scales are one byte a row and block, loaded a block ahead without a condition: a
// conditional load makes the wave wait for all others, and bytes that stand a row of blocks apart take a line each.
template <bool FAST, int WM, int WN, int MT, int NT>
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
    uint32_t scale_a[MT], scale_b[NT];                               // where their rows' scales begin: arrays of less than 2^29 bytes
#pragma unroll
    for (int i = 0; i < MT; ++i) scale_a[i] = uint32_t(a.scale_at(min(m0 + mw + i * 32 + col, a.rows - 1), 0));
#pragma unroll
    for (int j = 0; j < NT; ++j) scale_b[j] = uint32_t(b.scale_at(min(n0 + nw + col * NT + j, b.rows - 1), 0));
    const int blocks = a.bytes / kF8Block, first = blockIdx.y * per, last = min(blocks, first + per);
    f32x16 acc[MT][NT] = {};
    uint32_t sa[MT], sb[NT], sa_next[MT], sb_next[NT];              // this block's scales, and the next one's
    auto load_scales = [&](int block) {
        const uint8_t* in_a = a.scales + a.scale_at(0, min(block, blocks - 1));
        const uint8_t* in_b = b.scales + b.scale_at(0, min(block, blocks - 1));
#pragma unroll
        for (int i = 0; i < MT; ++i) sa_next[i] = in_a[scale_a[i]];
#pragma unroll
        for (int j = 0; j < NT; ++j) sb_next[j] = in_b[scale_b[j]];
    };
    auto take_scales = [&]() {
#pragma unroll
        for (int i = 0; i < MT; ++i) sa[i] = sa_next[i];
#pragma unroll
        for (int j = 0; j < NT; ++j) sb[j] = sb_next[j];
    };
    // operands of half a block
    auto read_a = [&](int s, int i, const uint4* lds) {
        return f8_operand(lds[lds_piece<3>(mw + col, s * 4 + half) + i * 256], lds[lds_piece<3>(mw + col, s * 4 + 2 + half) + i * 256]);
    };
    auto read_b = [&](int s, int j, const uint4* lds) {
        return f8_operand(lds[lds_piece<3>(nw + col, s * 4 + half) + j * 256], lds[lds_piece<3>(nw + col, s * 4 + 2 + half) + j * 256]);
    };
    auto load = [&](int block, uint4* to_a, uint4* to_b) {
        stage_a.load(block * kF8Block, to_a, wave);
        stage_b.load(block * kF8Block, to_b, wave);
    };
    // This wave's loads have arrived and its reads have ended, and so have all others'
    auto meet = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0070);
        __syncthreads();
    };
    load(first, s_a0, s_b0);
    load_scales(first);
    auto step = [&](bool more, int block, const uint4* now_a, const uint4* now_b, uint4* next_a, uint4* next_b) {
        take_scales();
        load_scales(block + 1);
        if (more) load(block + 1, next_a, next_b);
        float pa[MT], pb[NT];
        if constexpr (!FAST) {
#pragma unroll
            for (int i = 0; i < MT; ++i) pa[i] = f8_power(sa[i]);
#pragma unroll
            for (int j = 0; j < NT; ++j) pb[j] = f8_power(sb[j]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            i32x8 va[MT], vb[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) vb[j] = read_b(s, j, now_b);
#pragma unroll
            for (int i = 0; i < MT; ++i) va[i] = read_a(s, i, now_a);
            if constexpr (FAST) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = mfma_f8(va[i], vb[j], acc[i][j], int(sa[i]), int(sb[j]));
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) asm volatile("" : "+v"(acc[i][j]));
                __builtin_amdgcn_sched_barrier(0);
                continue;
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                bf16x8 xb[NT][2];
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    xb[j][0] = f8_bf16(vb[j][4 * q], vb[j][4 * q + 1], pb[j]);
                    xb[j][1] = f8_bf16(vb[j][4 * q + 2], vb[j][4 * q + 3], pb[j]);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const bf16x8 x0 = f8_bf16(va[i][4 * q], va[i][4 * q + 1], pa[i]), x1 = f8_bf16(va[i][4 * q + 2], va[i][4 * q + 3], pa[i]);
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        acc[i][j] = mfma32(x0, xb[j][0], acc[i][j]);
                        acc[i][j] = mfma32(x1, xb[j][1], acc[i][j]);
                    }
                }
            }
        }
        meet();
    };
    meet();
    int block = first;
    for (; block + 2 < last; block += 2) {
        step(true, block, s_a0, s_b0, s_a1, s_b1);
        step(true, block + 1, s_a1, s_b1, s_a0, s_b0);
    }
    step(block + 1 < last, block, s_a0, s_b0, s_a1, s_b1);
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
                else f8_store<FAST, NT>(c, int64_t(m) * stride + n, b.rows - n, v);
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
constexpr int kF8FewTokens = 16, kF8FewBytes = 65536;          // codes of x that LDS holds beside a second workgroup

// y = x W^T for at most 16 tokens whose codes fit into LDS.  WK x WN waves: 16 NT rows of W each, every WK-th block; a workgroup goes on to other rows
// as long as there are any.  Codes of W come from memory into the registers that are the operand, AHEAD blocks in front of their use; the first
// are on their way while the workgroup brings x to 8 bits.  The waves' sums of a row meet in LDS.
//
// Bound by reading W: one token through 32000 x 4096 bf16 22 us, 6.0 TB/s, through 11008 x 4096 9.6 us, 4.7, through 4096 x 4096 4.9 us, 3.4 (one round trip to memory, x and the
// join), with W behind L2 but not out of the memory's own cache.  Every workgroup brings the same x to 8 bits, which a kernel in front would do once, for a launch (so it began: 1 x 4096 x 4096 9.9 us);
// each token more costs 0.35 us of conversions.  Loads of four units at once took as long.
template <bool BF16, int WK, int WN, int NT, int AHEAD>
__global__ __launch_bounds__(64 * WK * WN) void f8_few_kernel(F8Mat w, const void* x, int t, int k, int64_t x_stride, void* y, int64_t y_stride) {
    constexpr int THREADS = 64 * WK * WN, ROWS = WN * NT * 16, PART = NT * 4 * 64;
    extern __shared__ uint4 s_x[];                                        // codes of x: [block][token], swizzled; then a scale for each
    __shared__ float s_sum[2][WK * WN * PART];
    const int blocks = w.bytes / kF8Block, lane = threadIdx.x & 63, wave = wave_number(), wk = wave % WK, wn = wave / WK;
    const int col = lane & 15, quarter = lane >> 4, tiles = (w.rows + ROWS - 1) / ROWS;
    uint8_t* s_scale = reinterpret_cast<uint8_t*>(s_x + blocks * t * 8);
    uint4 q[AHEAD][NT][2];
    uint32_t sw[AHEAD][NT];
    // the wave's steps: blocks wk, wk + WK, ... of one tile, then of the next
    int to_tile = blockIdx.x, to_block = wk;
    auto load = [&](int slot) {
        if (to_tile >= tiles) return;
        const uint8_t* in = w.scales + w.scale_at(0, to_block);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = min(to_tile * ROWS + (wn * NT + j) * 16 + col, w.rows - 1);
            const uint8_t* at = w.codes + int64_t(n) * w.bytes + to_block * kF8Block + quarter * 32;
            q[slot][j][0] = *reinterpret_cast<const uint4*>(at);
            q[slot][j][1] = *reinterpret_cast<const uint4*>(at + 16);
            sw[slot][j] = in[w.scale_at(n, 0)];
        }
        to_block += WK;
        if (to_block >= blocks) {
            to_block = wk;
            to_tile += gridDim.x;
        }
    };
    if (wk < blocks) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) load(i);
    }
    constexpr int AT_ONCE = THREADS / 16;                                 // 16 lanes a block of a token
    const int more_blocks = AT_ONCE / t, more_tokens = AT_ONCE - more_blocks * t;
    int block = int(threadIdx.x >> 4) / t, token = int(threadIdx.x >> 4) - block * t;
    for (; block < blocks; block += more_blocks, token += more_tokens) {
        if (token >= t) {
            token -= t;
            if (++block >= blocks) break;
        }
        const int d = threadIdx.x & 15, at = block * kF8Block + d * 8;
        const int64_t row = int64_t(token) * x_stride;
        float v[8];
        w4_load8<BF16>(x, row + at, row + k, v);
        const uint32_t scale = f8_scale(f8_top16(v));
        const float inverse = f8_inverse(scale);
        uint2 c;
        c.x = f8_codes4(v[0], v[1], v[2], v[3], inverse);
        c.y = f8_codes4(v[4], v[5], v[6], v[7], inverse);
        reinterpret_cast<uint2*>(s_x + block * t * 8)[lds_piece<3>(token, d >> 1) * 2 + (d & 1)] = c;
        if (d == 0) s_scale[block * t + token] = uint8_t(scale);
    }
    __syncthreads();
    int parity = 0;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, parity ^= 1) {
        f32x4 acc[NT] = {};
        for (int block = wk; block < blocks; block += WK) {
            uint4 x0 = make_uint4(0, 0, 0, 0), x1 = x0;
            uint32_t sx = 127;
            if (col < t) {
                const uint4* from = s_x + block * t * 8;
                x0 = from[lds_piece<3>(col, quarter * 2)];
                x1 = from[lds_piece<3>(col, quarter * 2 + 1)];
                sx = s_scale[block * t + col];
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if constexpr (BF16) {
                    acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f8_operand(x0, x1), f8_operand(q[0][j][0], q[0][j][1]), acc[j], 0, 0, 0, int(sx), 0,
                                                                              int(sw[0][j]));
                } else {
                    const float px = f8_power(sx), pw = f8_power(sw[0][j]);
                    const uint4 w0 = q[0][j][0], w1 = q[0][j][1];
                    acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f8_bf16(x0.x, x0.y, px), f8_bf16(w0.x, w0.y, pw), acc[j], 0, 0, 0);
                    acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f8_bf16(x0.z, x0.w, px), f8_bf16(w0.z, w0.w, pw), acc[j], 0, 0, 0);
                    acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f8_bf16(x1.x, x1.y, px), f8_bf16(w1.x, w1.y, pw), acc[j], 0, 0, 0);
                    acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f8_bf16(x1.z, x1.w, px), f8_bf16(w1.z, w1.w, pw), acc[j], 0, 0, 0);
                }
            }
            // the queue moves up by one
#pragma unroll
            for (int i = 0; i + 1 < AHEAD; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    q[i][j][0] = q[i + 1][j][0];
                    q[i][j][1] = q[i + 1][j][1];
                    sw[i][j] = sw[i + 1][j];
                }
            load(AHEAD - 1);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) s_sum[parity][wave * PART + (j * 4 + i) * 64 + lane] = acc[j][i];
        __syncthreads();                                                  // the other half of s_sum is free by the next one
        for (int id = threadIdx.x; id < WN * PART; id += THREADS) {
            const int part = id / PART, e = id % PART;
            float sum = 0.0f;
#pragma unroll
            for (int o = 0; o < WK; ++o) sum += s_sum[parity][(part * WK + o) * PART + e];
            const int n = tile * ROWS + (part * NT + e / 256) * 16 + (e & 15), tok = 4 * (e >> 4 & 3) + (e >> 6 & 3);
            if (n < w.rows && tok < t) w4_store1<BF16>(y, int64_t(tok) * y_stride + n, sum);
        }
    }
}

}  // namespace lpmm
