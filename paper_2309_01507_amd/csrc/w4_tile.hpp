// The product with 4-bit weights and its gradients for many tokens: tiles through LDS and the 32x32x16 matrix instructions.
#pragma once

#include "tile.hpp"
#include "w4.hpp"

namespace lpmm {

// ---- staging: octets of rows, from global memory into registers and from there into LDS ------------------------------------------

// Elements as they come from memory: 8 of them
template <bool BF16> struct RawOctet;
template <> struct RawOctet<true> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const void* p, int64_t i, int64_t end) {
        if (i + 8 <= end) {
            const Vec16 q = *reinterpret_cast<const Vec16*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = q.v[e];
        } else {
            const uint16_t* x = static_cast<const uint16_t*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = i + 2 * e < end ? x[i + 2 * e] : 0, hi = i + 2 * e + 1 < end ? x[i + 2 * e + 1] : 0;
                w[e] = lo | hi << 16;
            }
        }
    }
    __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
    __device__ __forceinline__ void terms(uint4 out[]) const { out[0] = make_uint4(w[0], w[1], w[2], w[3]); }
};
template <> struct RawOctet<false> {
    f32x4 lo, hi;
    __device__ __forceinline__ void load(const void* p, int64_t i, int64_t end) {
        const float* x = static_cast<const float*>(p) + i;
        if (i + 8 <= end) {
            lo = *reinterpret_cast<const f32x4u*>(x);
            hi = *reinterpret_cast<const f32x4u*>(x + 4);
        } else {
            const int64_t left = end - i;
            lo = f32x4{left > 0 ? x[0] : 0.0f, left > 1 ? x[1] : 0.0f, left > 2 ? x[2] : 0.0f, left > 3 ? x[3] : 0.0f};
            hi = f32x4{left > 4 ? x[4] : 0.0f, left > 5 ? x[5] : 0.0f, left > 6 ? x[6] : 0.0f, 0.0f};
        }
    }
    __device__ __forceinline__ void zero() { lo = hi = f32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void terms(uint4 out[]) const {
        const float x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        uint32_t w[3][4];
        split3_8(x, w);
#pragma unroll
        for (int j = 0; j < 3; ++j) out[j] = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
    }
};

// ROWS rows of 2^LOG octets, staged by THREADS threads: the octets of a thread are THREADS apart
template <bool BF16, int ROWS, int LOG, int THREADS>
struct Stage {
    static constexpr int kPieces = ROWS << LOG, kOwn = kPieces / THREADS, kTerms = kW4Terms<BF16>;
    static_assert(kPieces % THREADS == 0, "whole octets per thread");
    RawOctet<BF16> raw[kOwn];
    // rows row0 .. of a matrix of `rows` rows; columns col0 .. ; what lies outside is 0
    __device__ __forceinline__ void load(const void* p, int64_t stride, int row0, int rows, int col0, int cols) {
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            const int id = threadIdx.x + j * THREADS, r = row0 + (id >> LOG), c = col0 + (id & ((1 << LOG) - 1)) * 8;
            if (r < rows && c < cols) raw[j].load(p, int64_t(r) * stride + c, int64_t(r) * stride + cols);
            else raw[j].zero();
        }
    }
    __device__ __forceinline__ void store(uint4* lds) const {
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            const int id = threadIdx.x + j * THREADS;
            uint4 t[kTerms];
            raw[j].terms(t);
#pragma unroll
            for (int k = 0; k < kTerms; ++k) lds[k * kPieces + lds_piece<LOG>(id >> LOG, id & ((1 << LOG) - 1))] = t[k];
        }
    }
};

// ---- y = x W^T --------------------------------------------------------------------------------------------------------------------
//
// A workgroup of WN x WT waves takes WN NT 32 rows of W and WT TT 32 tokens.  x goes through LDS in runs of 128; codes
// go from memory into the registers of the waves that use them and are converted there.  Each group's products are summed from 0 and
// join the total with one multiply-add by the scale.  For fp32 and for bf16 off 16-byte boundaries: x passes through registers, so that its rows may
// start and end anywhere.  Bound by the matrix unit, for fp32, whose products cost three each, and the taking apart beside it (77 x 50257 x 1024, groups
// of 32: 51 to 54 us, 150 TFLOP/s, 450 of bf16; 4096 x 11008 x 4096, groups of 128: 945 to 990 us, 380); by conversions and waits for bf16 (that: 469 us, 790 TFLOP/s; groups
// of 64 spill 4 registers).
template <bool BF16, int GROUP, int WN, int WT, int NT, int TT>
__global__ __launch_bounds__(64 * WN * WT, 2) void w4_linear_tile_kernel(W4Mat m, const void* x, int t, int64_t x_stride, void* y,
                                                                      int64_t y_stride, int n_tiles, int t_tiles) {
    constexpr int TERMS = kW4Terms<BF16>, THREADS = 64 * WN * WT, BN = WN * NT * 32, BT = WT * TT * 32;
    typedef Stage<BF16, BT, 4, THREADS> StageX;
    __shared__ uint4 s_x[2][TERMS * StageX::kPieces];
    int n_tile, t_tile;
    if (!tile_of(blockIdx.x, n_tiles, t_tiles, n_tile, t_tile)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int n0 = n_tile * BN + (wave % WN) * NT * 32, t0 = t_tile * BT, tw = (wave / WN) * TT * 32;
    const uint32_t* codes[NT];
    const float* scales[NT];
#pragma unroll
    for (int b = 0; b < NT; ++b) {
        const int n = min(n0 + b * 32 + col, m.n - 1);
        codes[b] = m.codes + int64_t(n) * m.words + half * 4;
        scales[b] = m.scales + int64_t(n) * m.groups;
    }
    constexpr int GROUPS = kW4Chunk / GROUP;             // of a run
    uint4 q[NT][2];
    float sc[NT][GROUPS];
    auto load_w = [&](int run) {
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            q[b][0] = *reinterpret_cast<const uint4*>(codes[b] + run * 16);
            q[b][1] = *reinterpret_cast<const uint4*>(codes[b] + run * 16 + 8);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const int at = run * GROUPS + g;
                sc[b][g] = at < m.groups ? scales[b][at] : 0.0f;
            }
        }
    };
    f32x16 acc[TT][NT] = {};
    StageX stage;
    const int runs = m.words / 16;
    stage.load(x, x_stride, t0, t, 0, m.k);
    load_w(0);
    stage.store(s_x[0]);
    __syncthreads();
    for (int run = 0; run < runs; ++run) {
        uint32_t w[NT][8];
        float s_now[NT][GROUPS];
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            // step s uses piece s % 2 (logical word 2 s + half), word s / 2
            w[b][0] = q[b][0].x; w[b][1] = q[b][1].x; w[b][2] = q[b][0].y; w[b][3] = q[b][1].y;
            w[b][4] = q[b][0].z; w[b][5] = q[b][1].z; w[b][6] = q[b][0].w; w[b][7] = q[b][1].w;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) s_now[b][g] = sc[b][g];
        }
        const bool more = run + 1 < runs;
        if (more) {
            stage.load(x, x_stride, t0, t, (run + 1) * kW4Chunk, m.k);
            load_w(run + 1);
        }
        const uint4* lds = s_x[run & 1];
        f32x16 part[TT][NT];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            if (s * 16 % GROUP == 0) {
#pragma unroll
                for (int a = 0; a < TT; ++a)
#pragma unroll
                    for (int b = 0; b < NT; ++b) part[a][b] = f32x16{};
            }
            bf16x8 bw[NT];
#pragma unroll
            for (int b = 0; b < NT; ++b) bw[b] = w4_codes_bf16(w[b][s]);
#pragma unroll
            for (int a = 0; a < TT; ++a)
#pragma unroll
                for (int j = 0; j < TERMS; ++j) {
                    const bf16x8 ax = as_operand(lds[j * StageX::kPieces + lds_piece<4>(tw + a * 32 + col, 2 * s + half)]);
#pragma unroll
                    for (int b = 0; b < NT; ++b) part[a][b] = mfma32(ax, bw[b], part[a][b]);
                }
            if ((s + 1) * 16 % GROUP == 0) {
#pragma unroll
                for (int a = 0; a < TT; ++a)
#pragma unroll
                    for (int b = 0; b < NT; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float sum = __builtin_fmaf(s_now[b][s * 16 / GROUP], part[a][b][i], acc[a][b][i]);
                            if (GROUPS > 1) asm volatile("" : "+v"(sum));      // here: further down the sums of all groups would be held
                            acc[a][b][i] = sum;
                        }
            }
        }
        if (more) stage.store(s_x[(run + 1) & 1]);
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < TT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const int n = n0 + b * 32 + col;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int tok = t0 + tw + a * 32 + mfma32_row(i, half);
                if (n < m.n && tok < t) w4_store1<BF16>(y, int64_t(tok) * y_stride + n, acc[a][b][i]);
            }
        }
}

// The same for fewer tokens than fill the GPU with such tiles: 32 tokens by NT 32 rows of W per workgroup, whose 4 or 8 waves share the runs and join
// their sums at the end.  Tokens and codes go from memory into the registers of the lanes that multiply them, a run ahead; nothing is staged.
// Bound by latency and the taking apart of fp32 (each workgroup repeats it): 100 x 4096 x 4096, groups of 64, fp32: 31 us (4 waves 37, tiles above 70); with
// 64 rows of W 5 to 11 registers spill.
template <bool BF16, int GROUP, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void w4_linear_share_kernel(W4Mat m, const void* x, int t, int64_t x_stride, void* y, int64_t y_stride,
                                                              int n_tiles, int t_tiles) {
    constexpr int TERMS = kW4Terms<BF16>, GROUPS = kW4Chunk / GROUP;
    __shared__ float s_sum[WAVES][NT * 16 * 64];
    int n_tile, t_tile;
    if (!tile_of(blockIdx.x, n_tiles, t_tiles, n_tile, t_tile)) return;
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, half = lane >> 5;
    const int n0 = n_tile * NT * 32, t0 = t_tile * 32;
    const int64_t row = int64_t(min(t0 + col, t - 1)) * x_stride;
    const uint32_t* codes[NT];
    const float* scales[NT];
#pragma unroll
    for (int b = 0; b < NT; ++b) {
        const int n = min(n0 + b * 32 + col, m.n - 1);
        codes[b] = m.codes + int64_t(n) * m.words + half * 4;
        scales[b] = m.scales + int64_t(n) * m.groups;
    }
    RawOctet<BF16> raw[8];
    uint4 q[NT][2];
    float sc[NT][GROUPS];
    auto load = [&](int run) {
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int k = run * kW4Chunk + s * 16 + half * 8;
            if (k < m.k) raw[s].load(x, row + k, row + m.k);
            else raw[s].zero();
        }
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            q[b][0] = *reinterpret_cast<const uint4*>(codes[b] + run * 16);
            q[b][1] = *reinterpret_cast<const uint4*>(codes[b] + run * 16 + 8);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const int at = run * GROUPS + g;
                sc[b][g] = at < m.groups ? scales[b][at] : 0.0f;
            }
        }
    };
    f32x16 acc[NT] = {};
    const int runs = m.words / 16;
    if (wave < runs) load(wave);
    for (int run = wave; run < runs; run += WAVES) {
        RawOctet<BF16> now[8];
        uint32_t w[NT][8];
        float s_now[NT][GROUPS];
#pragma unroll
        for (int s = 0; s < 8; ++s) now[s] = raw[s];
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            // step s uses piece s % 2 (logical word 2 s + half), word s / 2
            w[b][0] = q[b][0].x; w[b][1] = q[b][1].x; w[b][2] = q[b][0].y; w[b][3] = q[b][1].y;
            w[b][4] = q[b][0].z; w[b][5] = q[b][1].z; w[b][6] = q[b][0].w; w[b][7] = q[b][1].w;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) s_now[b][g] = sc[b][g];
        }
        if (run + WAVES < runs) load(run + WAVES);
        f32x16 part[NT];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            if (s * 16 % GROUP == 0) {
#pragma unroll
                for (int b = 0; b < NT; ++b) part[b] = f32x16{};
            }
            uint4 ax[TERMS];
            now[s].terms(ax);
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const bf16x8 bw = w4_codes_bf16(w[b][s]);
#pragma unroll
                for (int j = 0; j < TERMS; ++j) part[b] = mfma32(as_operand(ax[j]), bw, part[b]);
            }
            if ((s + 1) * 16 % GROUP == 0) {
#pragma unroll
                for (int b = 0; b < NT; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float sum = __builtin_fmaf(s_now[b][s * 16 / GROUP], part[b][i], acc[b][i]);
                        if (GROUPS > 1) asm volatile("" : "+v"(sum));      // here: further down the sums of all groups would be held
                        acc[b][i] = sum;
                    }
            }
        }
    }
#pragma unroll
    for (int b = 0; b < NT; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s_sum[wave][(b * 16 + i) * 64 + lane] = acc[b][i];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NT * 16 / WAVES; ++j) {
        const int id = wave * (NT * 16 / WAVES) + j, i = id & 15, b = id >> 4;
        float v = s_sum[0][id * 64 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s_sum[w][id * 64 + lane];
        const int n = n0 + b * 32 + col, tok = t0 + mfma32_row(i, half);
        if (n < m.n && tok < t) w4_store1<BF16>(y, int64_t(tok) * y_stride + n, v);
    }
}

// An operand whose reduction runs down the rows of an array in LDS (2^LOG pieces a row, staged with TR): rows `row` + 8 half .. + 7, column
// cols + lane % 32.  A transposed read gives each of 16 lanes a column of 4 rows by 16 columns that their addresses make up.
typedef short s16x4 __attribute__((ext_vector_type(4)));
template <int LOG>
__device__ __forceinline__ bf16x8 operand_tr(const uint4* lds, int row, int cols) {
    const int lane = threadIdx.x & 63, half = lane >> 5, sub = lane & 15;
    union { s16x4 q[2]; bf16x8 v; } u;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int r = row + 8 * half + 4 * j + (sub >> 2), piece = (cols >> 3) + 2 * ((lane >> 4) & 1) + ((sub >> 1) & 1);
        const char* at = reinterpret_cast<const char*>(lds + lds_piece_tr(LOG, r, piece)) + (sub & 1) * 8;
#ifdef __HIP_DEVICE_COMPILE__
        u.q[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at));
#endif
    }
    return u.v;
}

// The same product for bf16 tokens on 16-byte boundaries (CUT: rows that end within a run).  Tokens and codes are loaded straight into LDS, a run
// ahead; a lane loads the scales of four groups at a time.  Two workgroups of 4 waves share a CU, so that one computes while the other waits at
// its barrier.  Bound by the matrix unit, beside which the conversion of the codes and the multiply-adds by the scales take issue slots:
// 4096 x 11008 x 4096, groups of 128: 331 us, 1117 TFLOP/s (a library's bf16 product of that size, without the weights' expansion: 360 to
// 429 us); groups of 64 359, of 32 424.  8 waves with one workgroup a CU and three buffers: 365 to 391; tokens through registers: 461.
template <int GROUP, int WN, int WT, int NT, int TT, bool CUT>
__global__ __launch_bounds__(64 * WN * WT, 2) void w4_linear_direct_kernel(W4Mat m, const void* x, int t, int64_t x_stride, void* y,
                                                                        int64_t y_stride, int n_tiles, int t_tiles) {
    constexpr int BN = WN * NT * 32, BT = WT * TT * 32, GROUPS = kW4Chunk / GROUP, WAVES = WN * WT;
    constexpr int QUAD = GROUP / 32;                           // runs that four groups make
    typedef StageDirect<BT, 4, WAVES> StageX;
    typedef StageDirect<BN, 2, WAVES> StageW;
    __shared__ uint4 s_x0[StageX::kPieces], s_x1[StageX::kPieces];       // objects of their own: what is loaded into one is no reason to wait in
    __shared__ uint4 s_w0[StageW::kPieces], s_w1[StageW::kPieces];       // front of reading another
    int n_tile, t_tile;
    if (!tile_of(blockIdx.x, n_tiles, t_tiles, n_tile, t_tile)) return;
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, half = lane >> 5;
    const int n0 = n_tile * BN, nw = (wave % WN) * NT * 32, t0 = t_tile * BT, tw = (wave / WN) * TT * 32;
    StageX stage_x;
    StageW stage_w;
    stage_x.setup(static_cast<const char*>(x) + int64_t(t0) * x_stride * 2, x_stride * 2, t - t0, wave);
    stage_w.setup(m.codes + int64_t(n0) * m.words, int64_t(m.words) * 4, m.n - n0, wave);
    const float* scales[NT];
#pragma unroll
    for (int b = 0; b < NT; ++b) scales[b] = m.scales + int64_t(min(n0 + nw + b * 32 + col, m.n - 1)) * m.groups;
    f32x4 sc[NT], sc_next[NT];
    auto load_scales = [&](int g) {
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            if (g + 4 <= m.groups) {
                sc_next[b] = *reinterpret_cast<const f32x4u*>(scales[b] + g);
            } else {
                sc_next[b].x = scales[b][g];
                sc_next[b].y = g + 1 < m.groups ? scales[b][g + 1] : 0.0f;
                sc_next[b].z = g + 2 < m.groups ? scales[b][g + 2] : 0.0f;
                sc_next[b].w = 0.0f;
            }
        }
    };
    auto load_x = [&](int run, uint4* lds) {
        if constexpr (CUT) stage_x.load_cut(run * (kW4Chunk * 2), m.k * 2, lds, wave);
        else stage_x.load(run * (kW4Chunk * 2), lds, wave);
    };
    f32x16 acc[TT][NT] = {};
    const f32x16 zero = opaque_zero();
    const int runs = m.words / 16;
    auto step = [&](bool more, int run, const uint4* now_x, const uint4* now_w, uint4* next_x, uint4* next_w) {
        if (run % QUAD == 0) {
#pragma unroll
            for (int b = 0; b < NT; ++b) sc[b] = sc_next[b];
        }
        if (more) {
            load_x(run + 1, next_x);
            stage_w.load((run + 1) * (kW4Chunk / 2), next_w, wave);
            if ((run + 1) % QUAD == 0) load_scales((run + 1) * GROUPS);
        }
        uint4 q[NT][2];
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            q[b][0] = now_w[lds_piece<2>(nw + b * 32 + col, half)];
            q[b][1] = now_w[lds_piece<2>(nw + b * 32 + col, half + 2)];
        }
        f32x16 part[TT][NT];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            bf16x8 bw[NT];
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const uint4 v = q[b][s & 1];                   // logical word 2 s + half
                bw[b] = w4_codes_bf16(s < 2 ? v.x : s < 4 ? v.y : s < 6 ? v.z : v.w);
            }
#pragma unroll
            for (int a = 0; a < TT; ++a) {
                const bf16x8 ax = as_operand(now_x[lds_piece<4>(tw + a * 32 + col, 2 * s + half)]);
#pragma unroll
                for (int b = 0; b < NT; ++b) part[a][b] = mfma32(ax, bw[b], s * 16 % GROUP == 0 ? zero : part[a][b]);
            }
            if ((s + 1) * 16 % GROUP == 0) {
                const int at = run % QUAD * GROUPS + s * 16 / GROUP;     // of the four; the same in all lanes
#pragma unroll
                for (int b = 0; b < NT; ++b) {
                    const float scale = at < 2 ? (at < 1 ? sc[b].x : sc[b].y) : (at < 3 ? sc[b].z : sc[b].w);
#pragma unroll
                    for (int a = 0; a < TT; ++a)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float sum = __builtin_fmaf(scale, part[a][b][i], acc[a][b][i]);
                            if (GROUPS > 1) asm volatile("" : "+v"(sum));      // here: further down the sums of all groups would be held
                            acc[a][b][i] = sum;
                        }
                }
            }
        }
        __syncthreads();
    };
    load_x(0, s_x0);
    stage_w.load(0, s_w0, wave);
    load_scales(0);
    __syncthreads();
    int run = 0;
    for (; run + 2 < runs; run += 2) {
        step(true, run, s_x0, s_w0, s_x1, s_w1);
        step(true, run + 1, s_x1, s_w1, s_x0, s_w0);
    }
    step(run + 1 < runs, run, s_x0, s_w0, s_x1, s_w1);
    if (run + 1 < runs) step(false, run + 1, s_x1, s_w1, s_x0, s_w0);
#pragma unroll
    for (int a = 0; a < TT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const int n = n0 + nw + b * 32 + col;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int tok = t0 + tw + a * 32 + mfma32_row(i, half);
                if (n < m.n && tok < t) w4_store1<true>(y, int64_t(tok) * y_stride + n, acc[a][b][i]);
            }
        }
}

// The same for fewer tokens than fill the GPU with such tiles: a tile of NT 32 rows of W and TT 32 tokens per workgroup, whose 4 waves share the
// runs.  Each wave stages its own runs in its own part of LDS, one ahead, and waits for nobody until the sums are joined.  Bound by the latency of
// a wave's runs: 64 x 4096 x 4096, groups of 128: 6.1 us, 1.6 TB/s; 256 tokens 13.6 us, 630 TFLOP/s, with one
// wave a SIMD, beside whose conversions and waits nothing runs.
template <int GROUP, int NT, int TT, bool CUT>
__global__ __launch_bounds__(256, 1) void w4_linear_split_kernel(W4Mat m, const void* x, int t, int64_t x_stride, void* y, int64_t y_stride,
                                                              int n_tiles, int t_tiles) {
    constexpr int BN = NT * 32, BT = TT * 32, GROUPS = kW4Chunk / GROUP, WAVES = 4;
    typedef StageDirect<BT, 4, 1> StageX;
    typedef StageDirect<BN, 2, 1> StageW;
    constexpr int PIECES = StageX::kPieces + StageW::kPieces;
    static_assert(PIECES * 16 >= NT * TT * 16 * 64 * 4, "room for a wave's sums");
    __shared__ uint4 s_a[WAVES][PIECES];
    __shared__ uint4 s_b[WAVES][PIECES];
    int n_tile, t_tile;
    if (!tile_of(blockIdx.x, n_tiles, t_tiles, n_tile, t_tile)) return;
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, half = lane >> 5;
    const int n0 = n_tile * BN, t0 = t_tile * BT;
    StageX stage_x;
    StageW stage_w;
    stage_x.setup(static_cast<const char*>(x) + int64_t(t0) * x_stride * 2, x_stride * 2, t - t0, 0);
    stage_w.setup(m.codes + int64_t(n0) * m.words, int64_t(m.words) * 4, m.n - n0, 0);
    const float* scales[NT];
#pragma unroll
    for (int b = 0; b < NT; ++b) scales[b] = m.scales + int64_t(min(n0 + b * 32 + col, m.n - 1)) * m.groups;
    float sc[NT][GROUPS];
    f32x16 acc[TT][NT] = {};
    const f32x16 zero = opaque_zero();
    const int runs = m.words / 16;
    auto load = [&](int run, uint4* lds) {
        if constexpr (CUT) stage_x.load_cut(run * (kW4Chunk * 2), m.k * 2, lds, 0);
        else stage_x.load(run * (kW4Chunk * 2), lds, 0);
        stage_w.load(run * (kW4Chunk / 2), lds + StageX::kPieces, 0);
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) sc[b][g] = scales[b][CUT ? min(run * GROUPS + g, m.groups - 1) : run * GROUPS + g];
    };
    auto step = [&](bool more, int run, const uint4* now, uint4* next) {
        // No barrier here: this run's loads have landed and the last one's reads are done, before the next one's loads go out.  Nothing crosses.
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070);                    // vmcnt(0), lgkmcnt(0)
        __builtin_amdgcn_sched_barrier(0);
        float scale[NT][GROUPS];
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) scale[b][g] = CUT && run * GROUPS + g >= m.groups ? 0.0f : sc[b][g];     // no group: the sum is 0, the scale another's
        if (more) load(run + WAVES, next);
        __builtin_amdgcn_sched_barrier(0);
        const uint4* now_w = now + StageX::kPieces;
        uint4 q[NT][2];
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            q[b][0] = now_w[lds_piece<2>(b * 32 + col, half)];
            q[b][1] = now_w[lds_piece<2>(b * 32 + col, half + 2)];
        }
        f32x16 part[TT][NT];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            bf16x8 bw[NT];
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const uint4 v = q[b][s & 1];                   // logical word 2 s + half
                bw[b] = w4_codes_bf16(s < 2 ? v.x : s < 4 ? v.y : s < 6 ? v.z : v.w);
            }
#pragma unroll
            for (int a = 0; a < TT; ++a) {
                const bf16x8 ax = as_operand(now[lds_piece<4>(a * 32 + col, 2 * s + half)]);
#pragma unroll
                for (int b = 0; b < NT; ++b) part[a][b] = mfma32(ax, bw[b], s * 16 % GROUP == 0 ? zero : part[a][b]);
            }
            if ((s + 1) * 16 % GROUP == 0) {
#pragma unroll
                for (int b = 0; b < NT; ++b)
#pragma unroll
                    for (int a = 0; a < TT; ++a)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float sum = __builtin_fmaf(scale[b][s * 16 / GROUP], part[a][b][i], acc[a][b][i]);
                            if (GROUPS > 1) asm volatile("" : "+v"(sum));      // here: further down the sums of all groups would be held
                            acc[a][b][i] = sum;
                        }
            }
        }
    };
    if (wave < runs) {
        load(wave, s_a[wave]);
        int run = wave;
        for (; run + 2 * WAVES < runs; run += 2 * WAVES) {     // no conditions here: a load that may not have been made is waited for with all others
            step(true, run, s_a[wave], s_b[wave]);
            step(true, run + WAVES, s_b[wave], s_a[wave]);
        }
        step(run + WAVES < runs, run, s_a[wave], s_b[wave]);
        if (run + WAVES < runs) step(false, run + WAVES, s_b[wave], s_a[wave]);
    }
    // sums through LDS: the wave's part of s_a is free, but loads into it may still be on their way
    __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);              // vmcnt(0)
    float* mine = reinterpret_cast<float*>(s_a[wave]);
#pragma unroll
    for (int a = 0; a < TT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) mine[((a * NT + b) * 16 + i) * 64 + lane] = acc[a][b][i];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NT * TT * 16 / WAVES; ++j) {
        const int id = wave * (NT * TT * 16 / WAVES) + j, i = id & 15, b = (id >> 4) % NT, a = (id >> 4) / NT;
        float v = reinterpret_cast<const float*>(s_a[0])[id * 64 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += reinterpret_cast<const float*>(s_a[w])[id * 64 + lane];
        const int n = n0 + b * 32 + col, tok = t0 + a * 32 + mfma32_row(i, half);
        if (n < m.n && tok < t) w4_store1<true>(y, int64_t(tok) * y_stride + n, v);
    }
}

// Sum over the 32 columns of a result tile: lane l of a half gets that of element l % 16.  Each step hands half of a lane's values to its partner
// and takes the partner's share of the others: 45 operations, where summing up each value in all lanes takes 80 and 16 exchanges through LDS.
__device__ __forceinline__ float sum_columns(f32x16 v) {
    const int lane = threadIdx.x & 63;
    float a[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) a[e] = v[e];
    const bool b3 = lane & 8, b2 = lane & 4, b1 = lane & 2, b0 = lane & 1;
#define LPMM_FOLD(BIT, HALF, CTRL) \
    for (int e = 0; e < HALF; ++e) { \
        const float keep = BIT ? a[e + HALF] : a[e], send = BIT ? a[e] : a[e + HALF]; \
        a[e] = keep + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(send), CTRL, 0xF, 0xF, false)); \
    }
#pragma unroll
    LPMM_FOLD(b3, 8, 0x140)                                    // with lane 15 - i of 16
#pragma unroll
    LPMM_FOLD(b2, 4, 0x141)                                    // with lane 7 - i of 8
#pragma unroll
    LPMM_FOLD(b1, 2, 0x4E)                                     // with lane i ^ 2
#pragma unroll
    LPMM_FOLD(b0, 1, 0xB1)                                     // with lane i ^ 1
#undef LPMM_FOLD
    return a[0] + __shfl_xor(a[0], 16);
}

// ---- gradient of the scales ---------------------------------------------------------------------------------------------------------
//
// dscales[n][g] = sum_t dy[t][n] P[t][n][g] with P the product's sum over the group before its scale: the same matrix products, and no
// weight gradient of n x k is ever formed.  A workgroup takes WN NT 32 rows of W and a run of 128 and walks over the tokens
// (those of split blockIdx.y); the run's codes stay converted in registers.  Here W is the A operand, so that a lane holds one token and
// for it 4 consecutive rows of W at a time, as dy has them; the sum over the lanes' tokens waits until the end.  Bound by LDS for
// many tokens, which delivers one fragment of x for each matrix instruction (fp32 4096 x 11008 x 4096, groups of 128: 1310 us, 281 TFLOP/s, 843 of bf16; bf16
// off 16-byte boundaries 758 us, groups of 64 with 2 registers spilled), by one tile's latency for few (fp32 333 x 2304 x 768, groups of 64: 12.5 us with the join).
template <bool BF16, int GROUP, int WN, int WT, int NT, int TT>
__global__ __launch_bounds__(64 * WN * WT, 2) void w4_dscale_tile_kernel(W4Mat m, const void* x, const void* dy, int t, int64_t x_stride,
                                                                      int64_t dy_stride, int n_tiles, int t_per_split, float* out,
                                                                      int64_t out_split) {
    constexpr int TERMS = kW4Terms<BF16>, THREADS = 64 * WN * WT, BN = WN * NT * 32, BT = WT * TT * 32;
    constexpr int GROUPS = kW4Chunk / GROUP, LOGD = BN == 256 ? 5 : 4;      // octets of dy a row
    static_assert(BN == 8 << LOGD, "rows of W of a tile");
    constexpr int DPIECE = BF16 ? 1 : 2;                                    // 16-byte pieces of an octet of dy
    typedef Stage<BF16, BT, 4, THREADS> StageX;
    typedef Stage<BF16, BT, LOGD, THREADS> StageD;                          // its raw octets only
    __shared__ uint4 s_x[2][TERMS * StageX::kPieces];
    __shared__ uint4 s_d[2][DPIECE * StageD::kPieces];
    __shared__ float s_sum[WT][GROUPS][BN];
    int n_tile, run;
    if (!tile_of(blockIdx.x, n_tiles, m.words / 16, n_tile, run)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int nw = (wave % WN) * NT * 32, n0 = n_tile * BN, tw = (wave / WN) * TT * 32;
    bf16x8 aw[NT][8];
#pragma unroll
    for (int b = 0; b < NT; ++b) {
        const int n = min(n0 + nw + b * 32 + col, m.n - 1);
        const uint32_t* c = m.codes + int64_t(n) * m.words + run * 16 + half * 4;
        const uint4 q0 = *reinterpret_cast<const uint4*>(c), q1 = *reinterpret_cast<const uint4*>(c + 8);
        const uint32_t w[8] = {q0.x, q1.x, q0.y, q1.y, q0.z, q1.z, q0.w, q1.w};
#pragma unroll
        for (int s = 0; s < 8; ++s) aw[b][s] = w4_codes_bf16(w[s]);
    }
    f32x16 sum[GROUPS][NT] = {};
    const int first = blockIdx.y * t_per_split, last = min(t, first + t_per_split);
    StageX sx;
    StageD sd;
    auto load = [&](int tok) {
        sx.load(x, x_stride, tok, last, run * kW4Chunk, m.k);
        sd.load(dy, dy_stride, tok, last, n0, m.n);
    };
    auto store = [&](int at) {
        sx.store(s_x[at]);
#pragma unroll
        for (int j = 0; j < StageD::kOwn; ++j) {
            const int id = threadIdx.x + j * THREADS, r = id >> LOGD, o = id & ((1 << LOGD) - 1);
            if constexpr (BF16) {
                s_d[at][lds_piece<LOGD>(r, o)] = make_uint4(sd.raw[j].w[0], sd.raw[j].w[1], sd.raw[j].w[2], sd.raw[j].w[3]);
            } else {
                s_d[at][lds_piece<LOGD + 1>(r, 2 * o)] = __builtin_bit_cast(uint4, sd.raw[j].lo);
                s_d[at][lds_piece<LOGD + 1>(r, 2 * o + 1)] = __builtin_bit_cast(uint4, sd.raw[j].hi);
            }
        }
    };
    if (first < last) {
        load(first);
        store(0);
    }
    __syncthreads();
    for (int tok = first, at = 0; tok < last; tok += BT, at ^= 1) {
        const bool more = tok + BT < last;
        if (more) load(tok + BT);
#pragma unroll
        for (int a = 0; a < TT; ++a) {
            const int r = tw + a * 32 + col;
            f32x16 d[NT];
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int o = (nw + b * 32) / 8 + i;                    // rows of W 8 o + 4 half .. + 3
                    if constexpr (BF16) {
                        const uint2 v = reinterpret_cast<const uint2*>(&s_d[at][lds_piece<LOGD>(r, o)])[half];
                        d[b][4 * i] = __uint_as_float(v.x << 16);
                        d[b][4 * i + 1] = __uint_as_float(v.x & 0xFFFF0000u);
                        d[b][4 * i + 2] = __uint_as_float(v.y << 16);
                        d[b][4 * i + 3] = __uint_as_float(v.y & 0xFFFF0000u);
                    } else {
                        const uint4 v = s_d[at][lds_piece<LOGD + 1>(r, 2 * o + half)];
                        d[b][4 * i] = __uint_as_float(v.x);
                        d[b][4 * i + 1] = __uint_as_float(v.y);
                        d[b][4 * i + 2] = __uint_as_float(v.z);
                        d[b][4 * i + 3] = __uint_as_float(v.w);
                    }
                }
            f32x16 part[NT];
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                if (s * 16 % GROUP == 0) {
#pragma unroll
                    for (int b = 0; b < NT; ++b) part[b] = f32x16{};
                }
#pragma unroll
                for (int j = 0; j < TERMS; ++j) {
                    const bf16x8 bx = as_operand(s_x[at][j * StageX::kPieces + lds_piece<4>(r, 2 * s + half)]);
#pragma unroll
                    for (int b = 0; b < NT; ++b) part[b] = mfma32(aw[b][s], bx, part[b]);
                }
                if ((s + 1) * 16 % GROUP == 0) {
#pragma unroll
                    for (int b = 0; b < NT; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float total = __builtin_fmaf(part[b][i], d[b][i], sum[s * 16 / GROUP][b][i]);
                            if (GROUPS > 1) asm volatile("" : "+v"(total));
                            sum[s * 16 / GROUP][b][i] = total;
                        }
                }
            }
        }
        if (more) store(at ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const float v = sum_columns(sum[g][b]);
            if (col < 16) s_sum[wave / WN][g][nw + b * 32 + mfma32_row(col, half)] = v;
        }
    __syncthreads();
    for (int id = threadIdx.x; id < GROUPS * BN; id += THREADS) {
        const int g = id % GROUPS, n = id / GROUPS, at = run * GROUPS + g;
        if (n0 + n >= m.n || at >= m.groups) continue;
        float v = s_sum[0][g][n];
#pragma unroll
        for (int w = 1; w < WT; ++w) v += s_sum[w][g][n];
        out[int64_t(blockIdx.y) * out_split + int64_t(n0 + n) * m.groups + at] = v;
    }
}

// The same for bf16 on 16-byte boundaries, the other way round: dy^T x is summed over the tokens by the matrix unit alone, in tiles of 256 rows of
// W by a run of 128 that are never written, and at the end multiplied by the codes and added up over the groups.  (With the product over the
// inputs first, 4096 tokens and 11008 x 4096 took 603 us: a multiply-add a product and token, and dy's conversion.)  Both operands'
// reduction runs down the rows of their arrays, hence the transposed reads.  Bound by the matrix unit and the reads that feed it: 4096 x 11008 x 4096,
// groups of 128: 319 us, 1160 TFLOP/s; 333 x 2304 x 768 10.0 us with the join, a third of it the end, where columns are summed up.
template <int GROUP>
__global__ __launch_bounds__(256, 2) void w4_dscale_direct_kernel(W4Mat m, const void* x, const void* dy, int t, int64_t x_stride,
                                                               int64_t dy_stride, int n_tiles, int t_per_split, float* out,
                                                               int64_t out_split) {
    constexpr int STEP = 32, NT = 4, KT = 2;                   // tokens of a step; tiles of a wave: 128 rows of W by 64 inputs
    typedef StageDirect<STEP, 5, 4, true> StageD;              // 256 rows of W
    typedef StageDirect<STEP, 4, 4, true> StageX;              // 128 inputs
    __shared__ uint4 s_d0[StageD::kPieces], s_d1[StageD::kPieces], s_x0[StageX::kPieces], s_x1[StageX::kPieces];
    __shared__ float s_sum[2][256];
    int n_tile, run;
    if (!tile_of(blockIdx.x, n_tiles, m.words / 16, n_tile, run)) return;
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, half = lane >> 5;
    const int n0 = n_tile * 256, nw = (wave & 1) * 128, k0 = run * kW4Chunk, kw = (wave >> 1) * 64;
    const int first = blockIdx.y * t_per_split, last = min(t, first + t_per_split);
    const char* from_d = static_cast<const char*>(dy) + (int64_t(first) * dy_stride + n0) * 2;
    const char* from_x = static_cast<const char*>(x) + (int64_t(first) * x_stride + k0) * 2;
    // a descriptor ends with the 32-bit word of the last row's last element (words are checked as a whole)
    const int64_t cut_d = int64_t(dy_stride - (m.n - n0)) * 2 & ~int64_t(3), cut_x = int64_t(x_stride - (m.k - k0)) * 2 & ~int64_t(3);
    StageD stage_d;
    StageX stage_x;
    stage_d.setup(from_d, dy_stride * 2, last - first, wave);
    stage_x.setup(from_x, x_stride * 2, last - first, wave);
    auto load = [&](int tok, uint4* lds_d, uint4* lds_x) {
        const int64_t left = last - tok;
        stage_d.buffer.set(from_d + int64_t(tok - first) * dy_stride * 2, min(left, int64_t(STEP)) * dy_stride * 2 - cut_d);
        stage_x.buffer.set(from_x + int64_t(tok - first) * x_stride * 2, min(left, int64_t(STEP)) * x_stride * 2 - cut_x);
        stage_d.load(0, lds_d, wave);
        stage_x.load(0, lds_x, wave);
    };
    f32x16 acc[NT][KT] = {};
    auto step = [&](bool more, int tok, const uint4* now_d, const uint4* now_x, uint4* next_d, uint4* next_x) {
        if (more) load(tok + STEP, next_d, next_x);
        __builtin_amdgcn_sched_barrier(0);                     // requested here, not at the step's end
#pragma unroll
        for (int s = 0; s < STEP / 16; ++s) {
            bf16x8 a[NT], b[KT];
#pragma unroll
            for (int i = 0; i < NT; ++i) a[i] = operand_tr<5>(now_d, s * 16, nw + i * 32);
#pragma unroll
            for (int j = 0; j < KT; ++j) b[j] = operand_tr<4>(now_x, s * 16, kw + j * 32);
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < KT; ++j) acc[i][j] = mfma32(a[i], b[j], acc[i][j]);
        }
        __syncthreads();
    };
    if (first < last) {
        load(first, s_d0, s_x0);
        __syncthreads();
        int tok = first;
        for (; tok + 2 * STEP < last; tok += 2 * STEP) {
            step(true, tok, s_d0, s_x0, s_d1, s_x1);
            step(true, tok + STEP, s_d1, s_x1, s_d0, s_x0);
        }
        step(tok + STEP < last, tok, s_d0, s_x0, s_d1, s_x1);
        if (tok + STEP < last) step(false, tok + STEP, s_d1, s_x1, s_d0, s_x0);
    }
    // times the codes, summed over the group: within the wave's two tiles, its 32 lanes, and for groups of 128 the two waves
    StageDirect<256, 2, 4> stage_w;
    static_assert(StageDirect<256, 2, 4>::kPieces <= StageD::kPieces, "room for the codes");
    stage_w.setup(m.codes + int64_t(n0) * m.words + run * 16, int64_t(m.words) * 4, m.n - n0, wave);
    stage_w.buffer.set(stage_w.buffer.start, int64_t(min(m.n - n0, 256) - 1) * m.words * 4 + kW4Chunk / 2);
    stage_w.load(0, s_d0, wave);
    __syncthreads();
    const int shift = (col & 7) * 4;
    uint32_t in[KT];                                           // mask: inputs beyond the row's end
    int place[KT];
#pragma unroll
    for (int j = 0; j < KT; ++j) {
        in[j] = k0 + kw + j * 32 + col < m.k ? 0xFFFFFFFFu : 0u;
        place[j] = w4_place((kw + j * 32 + col) >> 3);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        f32x16 v[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = nw + i * 32 + mfma32_row(e, half);
                const uint32_t word = reinterpret_cast<const uint32_t*>(s_d0 + lds_piece<2>(row, place[j] >> 2))[place[j] & 3];
                const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word >> shift, 1.0f, 0);
                v[j][e] = __uint_as_float(__float_as_uint(acc[i][j][e] * c.x) & in[j]);
            }
        if constexpr (GROUP > 32) {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[0][e] += v[1][e];
        }
        const int row = nw + i * 32 + mfma32_row(col & 15, half), n = n0 + row;
#pragma unroll
        for (int j = 0; j < (GROUP > 32 ? 1 : KT); ++j) {
            const float sum = sum_columns(v[j]);
            if (GROUP == 128) {
                if (col < 16) s_sum[wave >> 1][row] = sum;
            } else {
                const int at = (k0 + kw + j * 32) / GROUP;
                if (col < 16 && n < m.n && at < m.groups) out[int64_t(blockIdx.y) * out_split + int64_t(n) * m.groups + at] = sum;
            }
        }
    }
    if constexpr (GROUP == 128) {
        __syncthreads();
        const int n = n0 + int(threadIdx.x);
        if (n < m.n) out[int64_t(blockIdx.y) * out_split + int64_t(n) * m.groups + run] = s_sum[0][threadIdx.x] + s_sum[1][threadIdx.x];
    }
}

// Sum of `splits` floats, `apart` from one to the next, in their order; 4 are on their way at a time
__device__ __forceinline__ float sum_parts(const float* p, int splits, int64_t apart) {
    float v = *p;
    int s = 1;
    for (; s + 4 <= splits; s += 4) {
        const float a = p[s * apart], b = p[(s + 1) * apart], c = p[(s + 2) * apart], d = p[(s + 3) * apart];
        v = v + a + b + c + d;
    }
    for (; s < splits; ++s) v += p[s * apart];
    return v;
}

// The splits' parts added up.  Bound by latency (27648 sums of 6: 2 to 4 us).
__global__ __launch_bounds__(256) void w4_join_kernel(const float* parts, int splits, int64_t count, float* out) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i < count) out[i] = sum_parts(parts + i, splits, count);
}

// ---- dx = dy W -------------------------------------------------------------------------------------------------------------------------
//
// The reduction runs along W's rows, whose scales differ: value * scale is formed once per workgroup, as two bf16 terms for bf16 tokens (right to
// 2^-13; a single one would round each weight as coarsely as the result) or as three for fp32, and goes to LDS as it stands in W, a
// lane a word at a time; the transposition is the reads'.  fp32 takes the six products of terms that reach 2^-24 of the largest; there
// infinity must not meet a term of 0 of a number that is not, which would make NaN of it.  A dy that is not finite meets W's first term only, and a fourth array,
// dy's first terms with 2^-126 in its place, the other two; an infinite weight stands in W's third term, which meets that array only, and has 2^-126 in the first.  dy goes through registers, so that rows may start and end anywhere.  Bound by the matrix unit for many tokens (fp32
// 4096 x 11008 x 4096: 2425 us, 152 TFLOP/s, 914 of bf16; bf16 705 us, 524, 1050 of bf16), by the steps' latency for few (fp32 333 x 2304 x 768, groups of
// 64: 25 us with the join).

// A scale as a + b: a has 6 significant bits, so that a code's value times a is exact in bf16, and value * b is rounded to bf16, 2^-13 of the weight.
// b is taken 2^-20 of the scale too large, so that both have its sign and neither is 0: an infinite dy then meets no 0 and no infinity of the other sign.
__device__ __forceinline__ void split_scale(float s, float& a, float& b) {
    const bool finite = fabsf(s) < __builtin_inff();
    a = finite ? __uint_as_float(__float_as_uint(s) & 0xFFFC0000u) : s;
    b = finite ? __builtin_fmaf(s, 0x1p-20f, s - a) : __builtin_copysignf(1.0f, s);
}
// A word's weights as two terms
__device__ __forceinline__ void w4_weights8(uint32_t word, float scale, uint4& a, uint4& b) {
    float v[8], sa, sb;
    w4_values8(word, v);
    split_scale(scale, sa, sb);
    a = make_uint4(pack_bf16(v[0] * sa, v[1] * sa), pack_bf16(v[2] * sa, v[3] * sa), pack_bf16(v[4] * sa, v[5] * sa), pack_bf16(v[6] * sa, v[7] * sa));
    b = make_uint4(pack_bf16(v[0] * sb, v[1] * sb), pack_bf16(v[2] * sb, v[3] * sb), pack_bf16(v[4] * sb, v[5] * sb), pack_bf16(v[6] * sb, v[7] * sb));
}
// Three terms of 8 weights where some are infinite: those stand in the third term, and the first keeps their sign
__device__ __forceinline__ void split3_infinite(const float v[8], uint32_t w[3][4]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (fabsf(v[e]) != __builtin_inff()) continue;
        const int at = e / 2, shift = 16 * (e & 1);
        const uint32_t others = ~(0xFFFFu << shift), sign = (__float_as_uint(v[e]) >> 31) << (15 + shift);
        w[0][at] = (w[0][at] & others) | sign | 0x0080u << shift;
        w[2][at] = (w[2][at] & others) | sign | 0x7F80u << shift;
    }
}

template <bool BF16, int WT, int TT>
__global__ __launch_bounds__(128 * WT, 2) void w4_dx_tile_kernel(W4Mat m, const void* dy, int t, int64_t dy_stride, void* dx,
                                                              int64_t dx_stride, int t_tiles, int k_tiles, int n_per_split,
                                                              float* parts, int group_shift) {
    constexpr int TERMS = BF16 ? 2 : 3, DTERMS = BF16 ? 1 : 4, WK = 2, KT = 2, THREADS = 64 * WT * WK, BT = WT * TT * 32, STEP = 32;
    constexpr int WPIECES = STEP << 4, OWN = WPIECES / THREADS, ROWS = STEP / OWN;            // of 128 inputs; a word makes a piece
    typedef Stage<BF16, BT, 2, THREADS> StageD;
    __shared__ uint4 s_d[2][DTERMS * StageD::kPieces];
    __shared__ uint4 s_w[2][TERMS * WPIECES];
    int t_tile, k_tile;
    if (!tile_of(blockIdx.x, t_tiles, k_tiles, t_tile, k_tile)) return;
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, half = lane >> 5;
    const int t0 = t_tile * BT, tw = (wave % WT) * TT * 32, kw = (wave / WT) * KT * 32;
    const int first = blockIdx.y * n_per_split, last = min(m.n, first + n_per_split);
    const int d = threadIdx.x & 15, r = threadIdx.x >> 4, at = k_tile * kW4Chunk + d * 8;
    const uint32_t* codes = m.codes + k_tile * 16 + w4_place(d);
    const float* scales = m.scales + min(at >> group_shift, m.groups - 1);                    // beyond the last group all codes are 0
    StageD stage;
    uint32_t word[OWN];
    float sc[OWN];
    auto load = [&](int n) {
        stage.load(dy, dy_stride, t0, t, n, last);
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int row = n + r + j * ROWS;
            word[j] = row < last ? codes[int64_t(row) * m.words] : 0u;
            sc[j] = row < last ? scales[int64_t(row) * m.groups] : 0.0f;
        }
    };
    auto store = [&](uint4* lds_d, uint4* lds_w) {
        stage.store(lds_d);
        if constexpr (!BF16) {
#pragma unroll
            for (int j = 0; j < StageD::kOwn; ++j) {
                const int id = threadIdx.x + j * THREADS;
                uint4 f[3];
                stage.raw[j].terms(f);
                uint32_t w[4] = {f[0].x, f[0].y, f[0].z, f[0].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if ((w[e] & 0x7F80u) == 0x7F80u) w[e] = (w[e] & 0xFFFF8000u) | 0x0080u;
                    if ((w[e] & 0x7F800000u) == 0x7F800000u) w[e] = (w[e] & 0x8000FFFFu) | 0x00800000u;
                }
                lds_d[3 * StageD::kPieces + lds_piece<2>(id >> 2, id & 3)] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int to = lds_piece_tr(4, r + j * ROWS, d);
            if constexpr (BF16) {
                w4_weights8(word[j], sc[j], lds_w[to], lds_w[WPIECES + to]);
            } else {
                float v[8];
                w4_values8(word[j], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= sc[j];
                uint32_t w[3][4];
                split3_8(v, w);
                if (!(fabsf(sc[j]) < 0x1p125f)) split3_infinite(v, w);
#pragma unroll
                for (int k = 0; k < TERMS; ++k) lds_w[k * WPIECES + to] = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
            }
        }
    };
    f32x16 acc[TT][KT] = {};
    if (first < last) {
        load(first);
        store(s_d[0], s_w[0]);
    }
    __syncthreads();
    for (int n = first, now = 0; n < last; n += STEP, now ^= 1) {
        const bool more = n + STEP < last;
        if (more) load(n + STEP);
#pragma unroll
        for (int s = 0; s < STEP / 16; ++s) {
            bf16x8 bw[KT][TERMS];
#pragma unroll
            for (int b = 0; b < KT; ++b)
#pragma unroll
                for (int j = 0; j < TERMS; ++j) bw[b][j] = operand_tr<4>(s_w[now] + j * WPIECES, s * 16, kw + b * 32);
#pragma unroll
            for (int a = 0; a < TT; ++a)
#pragma unroll
                for (int j = 0; j < DTERMS; ++j) {
                    const bf16x8 ad = as_operand(s_d[now][j * StageD::kPieces + lds_piece<2>(tw + a * 32 + col, 2 * s + half)]);
                    // fp32: dy's terms 0, 1, 2 meet W's first 1, 2, 1 terms, the finite ones of term 0 its other two
                    constexpr int from[4] = {0, 0, 0, 1}, to[4] = {BF16 ? 2 : 1, 2, 1, 3};
#pragma unroll
                    for (int b = 0; b < KT; ++b)
#pragma unroll
                        for (int i = from[j]; i < to[j]; ++i) acc[a][b] = mfma32(ad, bw[b][i], acc[a][b]);
                }
        }
        if (more) store(s_d[now ^ 1], s_w[now ^ 1]);
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < TT; ++a)
#pragma unroll
        for (int b = 0; b < KT; ++b) {
            const int k = k_tile * kW4Chunk + kw + b * 32 + col;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int tok = t0 + tw + a * 32 + mfma32_row(i, half);
                if (k < m.k && tok < t) {
                    if (parts) parts[(int64_t(blockIdx.y) * t + tok) * m.k + k] = acc[a][b][i];
                    else w4_store1<BF16>(dx, int64_t(tok) * dx_stride + k, acc[a][b][i]);
                }
            }
        }
}

// The same for bf16 tokens on 16-byte boundaries and rows of W in whole steps of 32: dy straight into LDS, value * scale as it stands in W, so that
// a lane converts a word at a time; the transposition is the reads'.  Bound by the matrix unit, which takes two products for one: 4096 x 11008 x 4096
// 573 to 610 us, 605 to 645 TFLOP/s, twice that of bf16.  (With value * scale rounded to one bf16 number 362 us; the error against 64 bits was then 1.4 times that of rounding dx.)
template <bool PARTS, int TT>
__global__ __launch_bounds__(256, 2) void w4_dx_direct_kernel(W4Mat m, const void* dy, int t, int64_t dy_stride, void* dx, int64_t dx_stride,
                                                           int t_tiles, int k_tiles, int n_per_split, float* parts, int group_shift) {
    constexpr int STEP = 32, KT = 2;                           // rows of W of a step; tiles of a wave: 32 TT tokens by 64 inputs
    typedef StageDirect<64 * TT, 2, 4> StageD;                 // tokens by 32 rows of W
    constexpr int WPIECES = STEP << 4;                         // of 128 inputs
    __shared__ uint4 s_d0[StageD::kPieces], s_d1[StageD::kPieces], s_w0[2 * WPIECES], s_w1[2 * WPIECES];
    int t_tile, k_tile;
    if (!tile_of(blockIdx.x, t_tiles, k_tiles, t_tile, k_tile)) return;
    const int lane = threadIdx.x & 63, wave = wave_number(), col = lane & 31, half = lane >> 5;
    const int t0 = t_tile * (64 * TT), tw = (wave & 1) * (32 * TT), kw = (wave >> 1) * 64;
    const int first = blockIdx.y * n_per_split, last = min(m.n, first + n_per_split);
    StageD stage_d;
    stage_d.setup(static_cast<const char*>(dy) + int64_t(t0) * dy_stride * 2, dy_stride * 2, t - t0, wave);
    // a thread converts two words of a step: rows r and r + 16, word d
    const int d = threadIdx.x & 15, r = threadIdx.x >> 4, at = k_tile * kW4Chunk + d * 8;
    const uint32_t* codes = m.codes + int64_t(r) * m.words + k_tile * 16 + w4_place(d);
    const float* scales = m.scales + int64_t(r) * m.groups + min(at >> group_shift, m.groups - 1);     // beyond the last group all codes are 0
    uint32_t word[2];
    float sc[2];
    auto load = [&](int n, uint4* lds) {
        stage_d.load(n * 2, lds, wave);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            word[j] = codes[int64_t(n + 16 * j) * m.words];
            sc[j] = scales[int64_t(n + 16 * j) * m.groups];
        }
    };
    auto convert = [&](uint4* lds) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int to = lds_piece_tr(4, r + 16 * j, d);
            w4_weights8(word[j], sc[j], lds[to], lds[WPIECES + to]);
        }
    };
    f32x16 acc[TT][KT] = {};
    auto step = [&](bool more, int n, const uint4* now_d, const uint4* now_w, uint4* next_d, uint4* next_w) {
        if (more) load(n + STEP, next_d);
        __builtin_amdgcn_sched_barrier(0);                     // requested here, not at the step's end
#pragma unroll
        for (int s = 0; s < STEP / 16; ++s) {
            bf16x8 a[TT];
#pragma unroll
            for (int i = 0; i < TT; ++i) a[i] = as_operand(now_d[lds_piece<2>(tw + i * 32 + col, 2 * s + half)]);
#pragma unroll
            for (int term = 0; term < 2; ++term) {
                bf16x8 b[KT];
#pragma unroll
                for (int j = 0; j < KT; ++j) b[j] = operand_tr<4>(now_w + term * WPIECES, s * 16, kw + j * 32);
#pragma unroll
                for (int i = 0; i < TT; ++i)
#pragma unroll
                    for (int j = 0; j < KT; ++j) acc[i][j] = mfma32(a[i], b[j], acc[i][j]);
            }
        }
        if (more) convert(next_w);
        __syncthreads();
    };
    if (first < last) {
        load(first, s_d0);
        convert(s_w0);
        __syncthreads();
        int n = first;
        for (; n + 2 * STEP < last; n += 2 * STEP) {
            step(true, n, s_d0, s_w0, s_d1, s_w1);
            step(true, n + STEP, s_d1, s_w1, s_d0, s_w0);
        }
        step(n + STEP < last, n, s_d0, s_w0, s_d1, s_w1);
        if (n + STEP < last) step(false, n + STEP, s_d1, s_w1, s_d0, s_w0);
    }
#pragma unroll
    for (int i = 0; i < TT; ++i)
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            const int k = k_tile * kW4Chunk + kw + j * 32 + col;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int tok = t0 + tw + i * 32 + mfma32_row(e, half);
                if (k < m.k && tok < t) {
                    if constexpr (PARTS) parts[(int64_t(blockIdx.y) * t + tok) * m.k + k] = acc[i][j][e];
                    else w4_store1<true>(dx, int64_t(tok) * dx_stride + k, acc[i][j][e]);
                }
            }
        }
}

// The splits' parts (t x k each) added up
template <bool BF16>
__global__ __launch_bounds__(256) void w4_dx_join_kernel(const float* parts, int splits, int t, int k, void* dx, int64_t dx_stride) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x, count = uint32_t(t) * uint32_t(k);     // below 2^25: larger ones are not split
    if (i >= count) return;
    w4_store1<BF16>(dx, int64_t(i / uint32_t(k)) * dx_stride + i % uint32_t(k), sum_parts(parts + i, splits, count));
}

}  // namespace lpmm
