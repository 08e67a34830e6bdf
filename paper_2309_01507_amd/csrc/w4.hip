// C ABI of the 4-bit weights and of distillation (declared in include/lpmm4.h): argument checks and launches.  The arithmetic is
// in w4.hpp and distill.hpp.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "host_util.hpp"
#include "w4_tile.hpp"
#include "distill.hpp"

namespace {

using namespace lpmm;

constexpr int64_t kMaxDim = int64_t(1) << 30;
// A launch has fewer than 2^32 threads
constexpr int64_t kMaxTokens = (int64_t(1) << 24) - 1, kMaxWeights = int64_t(1) << 34, kMaxBlocks = (int64_t(1) << 23) - 1;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
int group_shift(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }
int elem_size(int dtype) { return dtype == LPMM_BF16 ? 2 : 4; }

int check_w4(const int64_t* shape, int group, W4Mat* m) {
    if (!shape || (group != 32 && group != 64 && group != 128)) return LPMM_EINVAL;
    if (shape[0] < 1 || shape[1] < 1 || shape[0] > kMaxDim || shape[1] > kMaxDim) return LPMM_EINVAL;
    const int64_t kp = div_up(shape[1], kW4Chunk) * kW4Chunk;
    if (shape[0] > kMaxWeights / kp) return LPMM_EINVAL;
    m->n = int(shape[0]);
    m->k = int(shape[1]);
    m->words = int(kp / 8);
    m->groups = int(div_up(shape[1], group));
    return LPMM_OK;
}

// `rows` rows of `len` elements, `stride` apart
int check_rows(const void* p, int dtype, int64_t rows, int64_t len, int64_t stride) {
    if (dtype != LPMM_F32 && dtype != LPMM_BF16) return LPMM_EINVAL;
    if (rows < 0 || rows > kMaxDim || stride < len || stride > (int64_t(1) << 40)) return LPMM_EINVAL;
    if (rows > 0 && (!p || !aligned(p, elem_size(dtype)))) return LPMM_EINVAL;
    return LPMM_OK;
}

int check_codes(const uint8_t* codes) { return codes && aligned(codes, 16) ? LPMM_OK : LPMM_EINVAL; }
int check_floats(const float* p) { return p && aligned(p, 4) ? LPMM_OK : LPMM_EINVAL; }

int check_workspace(const void* p, size_t have, size_t need) {
    if (need == 0) return LPMM_OK;
    if (!p || !aligned(p, 16)) return LPMM_EINVAL;
    return have < need ? LPMM_EWORKSPACE : LPMM_OK;
}

#define LPMM_TRY(call) do { const int rc_ = (call); if (rc_) return rc_; } while (0)

int check_distill(const void* z, int z_dtype, int64_t t, int64_t v, int64_t z_stride, const float* top,
                  const int64_t* index, int slots, float tau, DistillArgs* a) {
    if (t > kMaxTokens || v < 1 || v > kMaxDim || slots < 1 || slots > LPMM_DISTILL_MAX_SLOTS) return LPMM_EINVAL;
    // what the kernels multiply by: log2(e) / tau and tau^2
    if (!(tau > 0.0f) || !std::isfinite(kLog2e / tau) || !std::isfinite(tau * tau)) return LPMM_EINVAL;
    LPMM_TRY(check_rows(z, z_dtype, t, v, z_stride));
    if (t > 0 && (check_floats(top) || !index || !aligned(index, 8))) return LPMM_EINVAL;
    a->z = z;
    a->z_stride = z_stride;
    a->t = t;
    a->v = int(v);
    a->slots = slots;
    a->top = top;
    a->index = index;
    a->tau = tau;
    a->inv_tau = 1.0f / tau;
    a->c = kLog2e / tau;
    return LPMM_OK;
}

// Few rows that are long: the workgroups that share a row's sum; 1: one does it all
constexpr int kSpanBytes = 32768;
int distill_spans(int64_t t, int64_t v, int esize) {
    if (t >= 128 || v * esize < 8 * kSpanBytes) return 1;
    return int(std::min(div_up(v * esize, kSpanBytes), div_up(1024, t)));
}

int launch_loss(const DistillArgs& a, bool bf16, void* workspace, hipStream_t s) {
    const int spans = distill_spans(a.t, a.v, bf16 ? 2 : 4);
    if (spans > 1) {
        float2* parts = static_cast<float2*>(workspace);
        const int span = int(div_up(a.v, spans));
        const dim3 grid(unsigned(spans), unsigned(a.t)), rows(unsigned(a.t));      // spans * span >= v > (spans - 1) * span
        if (bf16) {
            hipLaunchKernelGGL(distill_part_kernel<true>, grid, dim3(kDistillThreads), 0, s, a, span, parts);
            LPMM_HIP(hipGetLastError());
            hipLaunchKernelGGL(distill_finish_kernel<true>, rows, dim3(64), distill_lds(a.slots), s, a, parts, spans);
        } else {
            hipLaunchKernelGGL(distill_part_kernel<false>, grid, dim3(kDistillThreads), 0, s, a, span, parts);
            LPMM_HIP(hipGetLastError());
            hipLaunchKernelGGL(distill_finish_kernel<false>, rows, dim3(64), distill_lds(a.slots), s, a, parts, spans);
        }
        LPMM_HIP(hipGetLastError());
        return LPMM_OK;
    }
    const dim3 rows(unsigned(a.t));
    const int64_t bytes = int64_t(a.v) * (bf16 ? 2 : 4);
#define LPMM_LOSS(B, N) hipLaunchKernelGGL((distill_loss_kernel<B, N>), rows, dim3(N), distill_lds(a.slots), s, a)
    if (bytes <= 16384) { if (bf16) LPMM_LOSS(true, 64); else LPMM_LOSS(false, 64); }
    else if (bytes <= 131072) { if (bf16) LPMM_LOSS(true, 256); else LPMM_LOSS(false, 256); }
    else { if (bf16) LPMM_LOSS(true, 1024); else LPMM_LOSS(false, 1024); }
#undef LPMM_LOSS
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

int launch_grad(const DistillArgs& a, bool bf16, hipStream_t s) {
    constexpr int64_t kRows = 32768;                     // of a launch: grid.y
    const bool narrow = int64_t(a.v) * (bf16 ? 2 : 4) <= 16384;      // short rows: a wave each
    for (int64_t r = 0; r < a.t; r += kRows) {
        DistillArgs b = a;
        b.z = static_cast<const char*>(a.z) + r * a.z_stride * (bf16 ? 2 : 4);
        b.dz = static_cast<char*>(a.dz) + r * a.dz_stride * (bf16 ? 2 : 4);
        b.top += r * a.slots;
        b.index += r * a.slots;
        b.grad += r;
        b.lse += r;
#define LPMM_GRAD(B, N) hipLaunchKernelGGL((distill_grad_kernel<B, N>), dim3(unsigned(div_up(a.v, kGradSpan<B, N>)), \
                                           unsigned(std::min(kRows, a.t - r))), dim3(N), distill_lds(a.slots), s, b)
        if (narrow) { if (bf16) LPMM_GRAD(true, 64); else LPMM_GRAD(false, 64); }
        else { if (bf16) LPMM_GRAD(true, 256); else LPMM_GRAD(false, 256); }
#undef LPMM_GRAD
        LPMM_HIP(hipGetLastError());
    }
    return LPMM_OK;
}

// Loss and gradient with a row in a workgroup's registers: the smallest shape that holds it.  Rows share a CU three or four at a time
// but for the longest: while one is summed up, others are read and written.  False: no shape holds it.
bool launch_both(const DistillArgs& a, bool bf16, hipStream_t s) {
    const int64_t pieces = div_up(a.v, bf16 ? kPiece<true> : kPiece<false>);
    const dim3 rows(unsigned(a.t));
#define LPMM_BOTH_OF(B, N, I, W) { hipLaunchKernelGGL((distill_both_kernel<B, N, I, W>), rows, dim3(N), distill_lds(a.slots), s, a); return true; }
#define LPMM_BOTH(N, I, W) if (pieces <= (N) * (I)) { if (bf16) LPMM_BOTH_OF(true, N, I, W) else LPMM_BOTH_OF(false, N, I, W) }
    LPMM_BOTH(64, 4, 8)
    LPMM_BOTH(64, 8, 4)
    LPMM_BOTH(256, 4, 8)
    LPMM_BOTH(256, 8, 4)
    LPMM_BOTH(256, 16, 3)
    // 25 pieces a thread, of which a few registers spill, pay for bf16 rows by the thousand (us with 256 and with 512 threads: 33000 logits, 2500 rows 67 and 64, 3500 rows 89
    // and 85, 4096 106 and 116, 8000 203 and 219; 40000: 71 and 71, 103 and 115, 125 and 130, 233 and 245; 50257: 100 and 101, 160 and 176, 190 and 205, 364 and 396;
    // 51200: 102 and 100, 141 and 139, 164 and 160, 317 and 303; 300 rows of 50257 22 and 19), for fp32 rows never (4096 rows of 17000, 20001, 25600: 113 and 107,
    // 143 and 132, 168 and 154)
    if (bf16 && a.t >= 3500 && pieces <= 256 * 25) LPMM_BOTH_OF(true, 256, 25, 3)
    LPMM_BOTH(512, 13, 4)
    LPMM_BOTH(512, 16, 4)
    LPMM_BOTH(1024, 13, 4)
    LPMM_BOTH(1024, 16, 4)
#undef LPMM_BOTH
#undef LPMM_BOTH_OF
    return false;
}

// Splits of a reduction over `steps` pieces for a launch of `blocks` workgroups: as many as bring it to `want` of them.
int splits_for(int64_t blocks, int64_t steps, int64_t want) {
    return int(std::max<int64_t>(1, std::min(steps, want / std::max<int64_t>(1, blocks))));
}

// The gradient of the scales: rows of W of a tile, tokens of a piece that splits are made of
constexpr int kDscaleRows = 256, kDscaleTokens = 64;
// What a CU holds of the kernel, once for each: two workgroups straight into LDS, one through registers (us, bf16 2000 x 2304 x 768 with 768, 512, 256
// workgroups at most: 21.2, 16.5, 17.6, 4096 x 4096 x 1024 42, 38, 43; fp32 333 x 2304 x 768 15.1, 15.1, 12.8, 2000 x 2304 x 768 43, 37, 36)
int dscale_splits(int64_t t, const W4Mat& m, bool direct) {
    return splits_for(div_up(m.n, kDscaleRows) * (m.words / 16), div_up(t, kDscaleTokens), direct ? 512 : 256);
}

// The gradient of the input: tiles of 128 inputs by 256, 128 or 64 tokens, the largest that still fill the GPU, since W is converted once for a
// tile (us with each: bf16 4096 x 11008 x 4096 609, 752, -; 1500 x 4096 x 4032 115, 115, -; 512 x 4096 x 4096 66, 54, -; off 16-byte boundaries 711, 885, 1041; 138,
// 141, 155; 79, 62, 69; 333 x 2304 x 768 30, 21, 17; fp32 2048 x 4096 x 4096 -, 456, 508; 512 x 4096 x 4096 -, 123, 137; 333 x 2304 x 2304 -, 43, 47); the
// reduction is split where there are fewer
struct DxPlan {
    bool direct;
    int bt, splits, n_per_split;
};
constexpr int kDxStep = 64;              // rows of W that splits are made of
bool dx_aligned(const void* dy, int dtype, int64_t dy_stride, const W4Mat& m) {
    return dtype == LPMM_BF16 && m.n % 32 == 0 && aligned(dy, 16) && dy_stride % 8 == 0 && dy_stride < (1 << 21);
}
DxPlan dx_plan(int64_t t, const W4Mat& m, bool bf16, bool aligned_rows) {
    DxPlan p{};
    p.direct = aligned_rows && t > 128;
    const int64_t k_tiles = div_up(m.k, kW4Chunk), tiles = div_up(t, 128) * k_tiles;
    p.bt = bf16 && div_up(t, 256) * k_tiles >= 512 ? 256 : p.direct || (bf16 ? tiles >= 128 : t > 64) ? 128 : 64;
    const int64_t steps = div_up(m.n, kDxStep);
    // A step takes a workgroup about 1.3 us (fp32: 3.2; 16 to 100 x 4096 x 4096 without splits: 64 steps, 83 to 88 and 190 to 222 us), each further split the join 0.2 us and
    // the time of writing and reading a part at 3 TB/s.  What that takes and the best of all numbers of splits (us): 1 x 4096 x 4096 bf16 16: 13.2, 20: 12.5; fp32 16: 22,
    // 20: 21.7; 16 x 2304 x 768 12: 10.4, 32: 9.5; 18: 12.8, 20: 12.8; 64 x 4096 x 4096 8: 22.5, 8: 22.4; 13: 34, 16: 31; 333 x 2304 x 768 6: 17.5, 10: 16.7; 9: 25, 9: 25;
    // 512 x 4096 x 4096 3: 55, 4: 50; 2: 124, 2: 124; 1000 x 4096 x 1024 5: 35, 8: 32; 4: 68, 4: 68; 128 x 50272 x 1024 32: 54, 48: 52; 32: 103, 32: 103
    const double step_us = bf16 ? 1.3 : 3.2, split_us = 0.2 + double(t) * m.k * 8 / 3e6;
    const int64_t worth = std::max<int64_t>(1, int64_t(std::sqrt(double(steps) * step_us / split_us)));
    const int splits = splits_for(div_up(t, p.bt) * k_tiles, std::min(div_up(steps, 2), worth), bf16 || p.bt == 64 ? 512 : 256);     // one workgroup of 8 waves a CU
    p.n_per_split = int(div_up(steps, splits)) * kDxStep;
    p.splits = int(div_up(m.n, p.n_per_split));
    return p;
}
size_t dx_bytes(int64_t t, const W4Mat& m, const DxPlan& p) { return p.splits > 1 ? size_t(p.splits) * size_t(t) * size_t(m.k) * 4 : 0; }

}  // namespace

extern "C" {

int lpmm_w4_sizes(const int64_t shape[2], int group, size_t sizes[2]) {
    W4Mat m{};
    if (!sizes) return LPMM_EINVAL;
    LPMM_TRY(check_w4(shape, group, &m));
    sizes[0] = size_t(m.n) * m.words * 4;
    sizes[1] = size_t(m.n) * m.groups * 4;
    return LPMM_OK;
}

int lpmm_w4_quant(const void* w, int dtype, int64_t w_stride, const int64_t shape[2], int group, uint8_t* codes,
                  float* scales, void* stream) {
    W4Mat m{};
    LPMM_TRY(check_w4(shape, group, &m));
    LPMM_TRY(check_rows(w, dtype, m.n, m.k, w_stride));
    LPMM_TRY(check_codes(codes));
    LPMM_TRY(check_floats(scales));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int runs = m.words / 16;
    const dim3 grid(unsigned(div_up(int64_t(m.n) * runs, 16)));
#define LPMM_QUANT(B, G) hipLaunchKernelGGL((w4_quant_kernel<B, G>), grid, dim3(256), 0, s, w, w_stride, m.n, m.k, runs, m.groups, \
                                            reinterpret_cast<uint32_t*>(codes), scales)
    if (dtype == LPMM_BF16) {
        if (group == 32) LPMM_QUANT(true, 32); else if (group == 64) LPMM_QUANT(true, 64); else LPMM_QUANT(true, 128);
    } else {
        if (group == 32) LPMM_QUANT(false, 32); else if (group == 64) LPMM_QUANT(false, 64); else LPMM_QUANT(false, 128);
    }
#undef LPMM_QUANT
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

int lpmm_w4_dequant(const uint8_t* codes, const float* scales, const int64_t shape[2], int group, void* w, int dtype,
                    int64_t w_stride, void* stream) {
    W4Mat m{};
    LPMM_TRY(check_w4(shape, group, &m));
    LPMM_TRY(check_rows(w, dtype, m.n, m.k, w_stride));
    LPMM_TRY(check_codes(codes));
    LPMM_TRY(check_floats(scales));
    m.codes = reinterpret_cast<const uint32_t*>(codes);
    m.scales = scales;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int runs = m.words / 16;
    const dim3 grid(unsigned(div_up(int64_t(m.n) * runs, 16)));
    if (dtype == LPMM_BF16) hipLaunchKernelGGL(w4_dequant_kernel<true>, grid, dim3(256), 0, s, m, runs, group_shift(group), w, w_stride);
    else hipLaunchKernelGGL(w4_dequant_kernel<false>, grid, dim3(256), 0, s, m, runs, group_shift(group), w, w_stride);
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

int lpmm_w4_linear(const void* x, int dtype, int64_t t, int64_t x_stride, const uint8_t* codes, const float* scales,
                   const int64_t shape[2], int group, void* y, int64_t y_stride, void* stream) {
    W4Mat m{};
    LPMM_TRY(check_w4(shape, group, &m));
    if (t > kMaxTokens) return LPMM_EINVAL;
    LPMM_TRY(check_rows(x, dtype, t, m.k, x_stride));
    LPMM_TRY(check_rows(y, dtype, t, m.n, y_stride));
    LPMM_TRY(check_codes(codes));
    LPMM_TRY(check_floats(scales));
    if (t == 0) return LPMM_OK;
    m.codes = reinterpret_cast<const uint32_t*>(codes);
    m.scales = scales;
    hipStream_t s = static_cast<hipStream_t>(stream);
    // 16-byte boundaries, whole octets, offsets within a tile below 2^31
    constexpr int kFew = 16;                             // tokens
    const bool direct = dtype == LPMM_BF16 && m.k % 8 == 0 && aligned(x, 16) && x_stride % 8 == 0 && x_stride < (1 << 22) && m.k < (1 << 22);
    // The runs split among a workgroup's waves while tiles of 64 x 64 are no more than two for each CU; smaller tiles while they leave CUs idle
    // (4096 x 4096, us, tiles of 128 x 128, 64 x 64, 64 rows x 32 tokens, 32 x 32: 64 tokens 32, 14, 8.8, 6.7; 100 33, 14, 9.2, 11;
    // 256 33, 15, 17, 19; 512 36, 27, 33, 37; 768 36, 42)
    const bool cut = m.k % kW4Chunk != 0;
    const auto tiles_of = [&](int rows, int tokens) { return div_up(m.n, rows) * div_up(t, tokens); };
    if (t > kFew && direct && tiles_of(64, 64) <= 512) {
        const bool n32 = tiles_of(32, 32) <= 256, t32 = tiles_of(64, 32) <= 256;
        const int64_t n_tiles = div_up(m.n, n32 ? 32 : 64), t_tiles = div_up(t, t32 ? 32 : 64), blocks = div_up(n_tiles * t_tiles, 8) * 8;
#define LPMM_SPLIT(G, NT, TT, C) hipLaunchKernelGGL((w4_linear_split_kernel<G, NT, TT, C>), dim3(unsigned(blocks)), dim3(256), 0, s, m, x, int(t), x_stride, \
                                                 y, y_stride, int(n_tiles), int(t_tiles))
#define LPMM_SPLIT_C(NT, TT, C) { if (group == 32) LPMM_SPLIT(32, NT, TT, C); else if (group == 64) LPMM_SPLIT(64, NT, TT, C); else LPMM_SPLIT(128, NT, TT, C); }
#define LPMM_SPLIT_G(NT, TT) { if (cut) LPMM_SPLIT_C(NT, TT, true) else LPMM_SPLIT_C(NT, TT, false) }
        if (n32) LPMM_SPLIT_G(1, 1) else if (t32) LPMM_SPLIT_G(2, 1) else LPMM_SPLIT_G(2, 2)
#undef LPMM_SPLIT_G
#undef LPMM_SPLIT_C
#undef LPMM_SPLIT
        LPMM_HIP(hipGetLastError());
        return LPMM_OK;
    }
    if (t > kFew && direct) {
        const int64_t n_tiles = div_up(m.n, 128), t_tiles = div_up(t, 128);
        const int64_t blocks = div_up(n_tiles * t_tiles, 8) * 8;
        if (blocks > kMaxBlocks) return LPMM_EINVAL;
#define LPMM_DIRECT(G, C) hipLaunchKernelGGL((w4_linear_direct_kernel<G, 2, 2, 2, 2, C>), dim3(unsigned(blocks)), dim3(256), 0, s, m, x, \
                                             int(t), x_stride, y, y_stride, int(n_tiles), int(t_tiles))
#define LPMM_DIRECT_G(C) { if (group == 32) LPMM_DIRECT(32, C); else if (group == 64) LPMM_DIRECT(64, C); else LPMM_DIRECT(128, C); }
        if (cut) LPMM_DIRECT_G(true) else LPMM_DIRECT_G(false)
#undef LPMM_DIRECT_G
#undef LPMM_DIRECT
        LPMM_HIP(hipGetLastError());
        return LPMM_OK;
    }
    const bool bf16 = dtype == LPMM_BF16;
    // Elsewhere (us, fp32 with groups of 32; the few tokens' kernel, runs shared by waves with 32 and 64 rows of W, tiles of 256 rows by 32 tokens): 32 x 4096 x 4096
    // 19, 26, 35; 32 x 32000 x 4096 140, 78, 57; 64 x 4096 x 4096 37, 27, 36; 64 x 11008 x 4096 -, 61, 54, 82; 256 x 4096 x 4096 -, 75, 57, 83;
    // 300 x 4000 x 4096 -, -, 99, 83; 64 x 50257 x 1024 -, -, 62, 38.  bf16 off 16-byte boundaries, the last two: 256 x 4096 x 4096 59, 80; 512 x 4096 x 4096 105, 82
    const bool many = t > 32 || t > kFew && tiles_of(64, 32) > 128;
    if (many && tiles_of(64, 32) <= 512) {
        const bool n32 = tiles_of(32, 32) <= 256;
        const int64_t n_tiles = div_up(m.n, n32 ? 32 : 64), t_tiles = div_up(t, 32), blocks = div_up(n_tiles * t_tiles, 8) * 8;
#define LPMM_SHARE(B, G, NT, W) hipLaunchKernelGGL((w4_linear_share_kernel<B, G, NT, W>), dim3(unsigned(blocks)), dim3(64 * W), 0, s, m, x, int(t), x_stride, \
                                                y, y_stride, int(n_tiles), int(t_tiles))
#define LPMM_SHARE_G(B, NT, W) { if (group == 32) LPMM_SHARE(B, 32, NT, W); else if (group == 64) LPMM_SHARE(B, 64, NT, W); else LPMM_SHARE(B, 128, NT, W); }
        // 8 waves where CUs have one workgroup, 4 where they have two (fp32, groups of 32, 4 and 8: 64 x 4096 x 4096 26, 22; 100 x 4096 x 4096 36, 30;
        // 256 x 4096 x 4096 56, 61; 32 x 32000 x 4096 58, 63)
        const bool one = blocks <= 256;
        if (bf16) { if (n32) LPMM_SHARE_G(true, 1, 8) else if (one) LPMM_SHARE_G(true, 2, 8) else LPMM_SHARE_G(true, 2, 4) }
        else { if (n32) LPMM_SHARE_G(false, 1, 8) else if (one) LPMM_SHARE_G(false, 2, 8) else LPMM_SHARE_G(false, 2, 4) }
#undef LPMM_SHARE_G
#undef LPMM_SHARE
        LPMM_HIP(hipGetLastError());
        return LPMM_OK;
    }
    if (many) {
        // 256 rows of W by 64 tokens, fp32, whose terms take three times the room, by 32; 4 waves, two workgroups a CU.  (1000 x 4096 x 4096 bf16 off 16-byte
        // boundaries, groups of 128: 54 us, with 8 waves and 128 tokens 88, with 128 by 128 114; fp32 105, 128 rows by 64 tokens 122, 256 by 64 and 8 waves 112)
        const int64_t n_tiles = div_up(m.n, 256), t_tiles = div_up(t, bf16 ? 64 : 32);
        const int64_t blocks = div_up(n_tiles * t_tiles, 8) * 8;
        if (blocks > kMaxBlocks) return LPMM_EINVAL;
#define LPMM_TILE(B, G, TT) hipLaunchKernelGGL((w4_linear_tile_kernel<B, G, 4, 1, 2, TT>), dim3(unsigned(blocks)), dim3(256), 0, s, m, x, int(t), x_stride, y, \
                                               y_stride, int(n_tiles), int(t_tiles))
        if (bf16) {
            if (group == 32) LPMM_TILE(true, 32, 2); else if (group == 64) LPMM_TILE(true, 64, 2); else LPMM_TILE(true, 128, 2);
        } else {
            if (group == 32) LPMM_TILE(false, 32, 1); else if (group == 64) LPMM_TILE(false, 64, 1); else LPMM_TILE(false, 128, 1);
        }
#undef LPMM_TILE
        LPMM_HIP(hipGetLastError());
        return LPMM_OK;
    }
    // At most 32 tokens: 16 or 32 a workgroup; as many runs a wave as cover a row with 8 or 16 waves, up to what registers hold
    // (S waves a SIMD; E: the next tile's codes ahead of this one's products)
    const int mt = t <= 16 ? 1 : 2, runs = m.words / 16;
    const int64_t tiles = div_up(m.n, 16);
#define LPMM_FEW(B, G, MT, W, A, S, E) hipLaunchKernelGGL((w4_linear_kernel<B, G, MT, W, A, S, E>), dim3(unsigned(std::min<int64_t>(tiles, 256 * 4 * S / W))), \
                                                          dim3(64 * W), 0, s, m, x, int(t), x_stride, y, y_stride)
#define LPMM_FEW_G(B, MT, W, A, S, E) { if (group == 32) LPMM_FEW(B, 32, MT, W, A, S, E); else if (group == 64) LPMM_FEW(B, 64, MT, W, A, S, E); else LPMM_FEW(B, 128, MT, W, A, S, E); }
    if (bf16) {
        if (mt == 1) {
            if (runs <= 8) LPMM_FEW_G(true, 1, 8, 1, 4, true)
            else if (runs <= 16) LPMM_FEW_G(true, 1, 8, 2, 4, true)
            else LPMM_FEW_G(true, 1, 16, 2, 4, true)
        } else if (runs <= 8) {
            LPMM_FEW_G(true, 2, 8, 1, 4, true)
        } else {
            LPMM_FEW_G(true, 2, 16, 1, 4, true)
        }
    } else if (mt == 1) {
        if (runs <= 8) LPMM_FEW_G(false, 1, 8, 1, 4, true)
        // x of a whole row in registers, some of which spill (238 in groups of 64, 16 in groups of 128), pays for many rows that 8 waves cover at once (us, with it and
        // with (16, 1, 4); 7 x 32000 x 4096 groups of 64 55 and 67, of 128 34 and 66; 1 x 16384 x 4096 32 and 32, 22 and 31; 16 x 32000 x 4096 60 and 104, 37 and 104; longer
        // rows 7 x 32000 x 8192 221 and 126, 187 and 126; groups of 32, with 594 spilled, 93 and 68 for 7 x 32000 x 4096)
        else if (runs > 16 && runs <= 32 && tiles >= 1024 && group == 64) LPMM_FEW(false, 64, 1, 8, 4, 2, false);
        else if (runs > 16 && runs <= 32 && tiles >= 1024 && group == 128) LPMM_FEW(false, 128, 1, 8, 4, 2, false);
        else LPMM_FEW_G(false, 1, 16, 1, 4, true)                                      // 1 x 4096 x 4096: 9 us, with (16, 2, 4) 17
    } else {
        LPMM_FEW_G(false, 2, 8, 1, 2, true)
    }
#undef LPMM_FEW_G
#undef LPMM_FEW
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

size_t lpmm_w4_linear_dx_workspace_bytes(int64_t t, const int64_t shape[2], int dtype) {
    W4Mat m{};
    if (check_w4(shape, 32, &m) || t < 1 || t > kMaxTokens || (dtype != LPMM_F32 && dtype != LPMM_BF16)) return 0;
    const bool bf16 = dtype == LPMM_BF16;
    return std::max(dx_bytes(t, m, dx_plan(t, m, bf16, false)), dx_bytes(t, m, dx_plan(t, m, bf16, bf16)));
}

int lpmm_w4_linear_dx(const void* dy, int dtype, int64_t t, int64_t dy_stride, const uint8_t* codes,
                      const float* scales, const int64_t shape[2], int group, void* dx, int64_t dx_stride, void* workspace,
                      size_t workspace_bytes, void* stream) {
    W4Mat m{};
    LPMM_TRY(check_w4(shape, group, &m));
    if (t > kMaxTokens) return LPMM_EINVAL;
    LPMM_TRY(check_rows(dy, dtype, t, m.n, dy_stride));
    LPMM_TRY(check_rows(dx, dtype, t, m.k, dx_stride));
    LPMM_TRY(check_codes(codes));
    LPMM_TRY(check_floats(scales));
    if (t == 0) return LPMM_OK;
    const bool bf16 = dtype == LPMM_BF16;
    const DxPlan p = dx_plan(t, m, bf16, dx_aligned(dy, dtype, dy_stride, m));
    LPMM_TRY(check_workspace(workspace, workspace_bytes, dx_bytes(t, m, p)));
    m.codes = reinterpret_cast<const uint32_t*>(codes);
    m.scales = scales;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t t_tiles = div_up(t, p.bt), k_tiles = div_up(m.k, kW4Chunk), blocks = div_up(t_tiles * k_tiles, 8) * 8;
    if (blocks > kMaxBlocks) return LPMM_EINVAL;
    float* parts = p.splits > 1 ? static_cast<float*>(workspace) : nullptr;
    const dim3 grid(unsigned(blocks), unsigned(p.splits));
#define LPMM_DX(B, WT, TT) hipLaunchKernelGGL((w4_dx_tile_kernel<B, WT, TT>), grid, dim3(128 * WT), 0, s, m, dy, \
                                                            int(t), dy_stride, dx, dx_stride, int(t_tiles), int(k_tiles), p.n_per_split, \
                                                            parts, group_shift(group))
#define LPMM_DX_DIRECT(P, TT) hipLaunchKernelGGL((w4_dx_direct_kernel<P, TT>), grid, dim3(256), 0, s, m, dy, int(t), dy_stride, dx, dx_stride, int(t_tiles), \
                                             int(k_tiles), p.n_per_split, parts, group_shift(group))
    if (p.direct && p.bt == 256) LPMM_DX_DIRECT(false, 4);          // as many tiles need no splits
    else if (p.direct) { if (parts) LPMM_DX_DIRECT(true, 2); else LPMM_DX_DIRECT(false, 2); }
    else if (bf16 && p.bt == 256) LPMM_DX(true, 2, 4);
    else if (bf16 && p.bt == 128) LPMM_DX(true, 2, 2);
    else if (bf16) LPMM_DX(true, 2, 1);
    else if (p.bt == 128) LPMM_DX(false, 4, 1);
    else LPMM_DX(false, 2, 1);
#undef LPMM_DX_DIRECT
#undef LPMM_DX
    LPMM_HIP(hipGetLastError());
    if (parts) {
        const dim3 join(unsigned(div_up(t * m.k, 256)));
        if (bf16) hipLaunchKernelGGL(w4_dx_join_kernel<true>, join, dim3(256), 0, s, parts, p.splits, int(t), m.k, dx, dx_stride);
        else hipLaunchKernelGGL(w4_dx_join_kernel<false>, join, dim3(256), 0, s, parts, p.splits, int(t), m.k, dx, dx_stride);
        LPMM_HIP(hipGetLastError());
    }
    return LPMM_OK;
}

size_t lpmm_w4_linear_dscale_workspace_bytes(int64_t t, const int64_t shape[2], int group) {
    W4Mat m{};
    if (check_w4(shape, group, &m) || t < 1 || t > kMaxTokens) return 0;
    const int splits = dscale_splits(t, m, true);            // no fewer than the others take
    return splits > 1 ? size_t(splits) * m.n * m.groups * 4 : 0;
}

int lpmm_w4_linear_dscale(const void* x, const void* dy, int dtype, int64_t t, int64_t x_stride, int64_t dy_stride,
                          const uint8_t* codes, const int64_t shape[2], int group, float* dscales, void* workspace,
                          size_t workspace_bytes, void* stream) {
    W4Mat m{};
    LPMM_TRY(check_w4(shape, group, &m));
    if (t > kMaxTokens) return LPMM_EINVAL;
    LPMM_TRY(check_rows(x, dtype, t, m.k, x_stride));
    LPMM_TRY(check_rows(dy, dtype, t, m.n, dy_stride));
    LPMM_TRY(check_codes(codes));
    LPMM_TRY(check_floats(dscales));
    LPMM_TRY(check_workspace(workspace, workspace_bytes, lpmm_w4_linear_dscale_workspace_bytes(t, shape, group)));
    m.codes = reinterpret_cast<const uint32_t*>(codes);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t n_tiles = div_up(m.n, kDscaleRows), blocks = div_up(n_tiles * (m.words / 16), 8) * 8;
    if (blocks > kMaxBlocks) return LPMM_EINVAL;
    const bool direct = dtype == LPMM_BF16 && aligned(x, 16) && aligned(dy, 16) && x_stride % 8 == 0 && dy_stride % 8 == 0 &&
                        x_stride < (1 << 24) && dy_stride < (1 << 24) && m.k < (1 << 23);
    int splits = dscale_splits(t, m, direct);
    const int per = int(div_up(div_up(t, kDscaleTokens), splits)) * kDscaleTokens;
    splits = std::max(1, int(div_up(t, std::max(per, 1))));
    const int64_t count = int64_t(m.n) * m.groups;
    float* out = splits > 1 ? static_cast<float*>(workspace) : dscales;
    const dim3 grid = dim3(unsigned(blocks), unsigned(splits));
    if (direct) {
#define LPMM_DSCALE_DIRECT(G) hipLaunchKernelGGL(w4_dscale_direct_kernel<G>, grid, dim3(256), 0, s, m, x, dy, int(t), x_stride, dy_stride, int(n_tiles), \
                                                 per, out, count)
        if (group == 32) LPMM_DSCALE_DIRECT(32); else if (group == 64) LPMM_DSCALE_DIRECT(64); else LPMM_DSCALE_DIRECT(128);
#undef LPMM_DSCALE_DIRECT
    } else
#define LPMM_DSCALE(B, G, WN, WT, NT, TT) hipLaunchKernelGGL((w4_dscale_tile_kernel<B, G, WN, WT, NT, TT>), grid, dim3(512), 0, s, m, x, dy, int(t), \
                                                             x_stride, dy_stride, int(n_tiles), per, out, count)
    if (dtype == LPMM_BF16) {
        if (group == 32) LPMM_DSCALE(true, 32, 8, 1, 1, 2);
        else if (group == 64) LPMM_DSCALE(true, 64, 4, 2, 2, 1);
        else LPMM_DSCALE(true, 128, 4, 2, 2, 1);
    } else {
        if (group == 32) LPMM_DSCALE(false, 32, 8, 1, 1, 1);
        else if (group == 64) LPMM_DSCALE(false, 64, 8, 1, 1, 1);
        else LPMM_DSCALE(false, 128, 8, 1, 1, 1);
    }
#undef LPMM_DSCALE
    LPMM_HIP(hipGetLastError());
    if (splits > 1) {
        hipLaunchKernelGGL(w4_join_kernel, dim3(unsigned(div_up(count, 256))), dim3(256), 0, s, out, splits, count, dscales);
        LPMM_HIP(hipGetLastError());
    }
    return LPMM_OK;
}

size_t lpmm_distill_workspace_bytes(int64_t t, int64_t v) {
    if (t < 1 || t > kMaxTokens || v < 1 || v > kMaxDim) return 0;
    const int spans = std::max(distill_spans(t, v, 2), distill_spans(t, v, 4));
    return spans > 1 ? size_t(t) * spans * sizeof(float2) : 0;
}

int lpmm_distill_loss(const void* z, int z_dtype, int64_t t, int64_t v, int64_t z_stride, const float* top,
                      const int64_t* index, int slots, float tau, float* loss, float* lse, void* workspace,
                      size_t workspace_bytes, void* stream) {
    DistillArgs a{};
    LPMM_TRY(check_distill(z, z_dtype, t, v, z_stride, top, index, slots, tau, &a));
    if (t == 0) return LPMM_OK;
    LPMM_TRY(check_floats(loss));
    LPMM_TRY(check_floats(lse));
    LPMM_TRY(check_workspace(workspace, workspace_bytes, lpmm_distill_workspace_bytes(t, v)));
    a.loss = loss;
    a.lse = lse;
    return launch_loss(a, z_dtype == LPMM_BF16, workspace, static_cast<hipStream_t>(stream));
}

int lpmm_distill_grad(const void* z, int z_dtype, int64_t t, int64_t v, int64_t z_stride, const float* top,
                      const int64_t* index, int slots, float tau, const float* lse, const float* grad, void* dz,
                      int64_t dz_stride, void* stream) {
    DistillArgs a{};
    LPMM_TRY(check_distill(z, z_dtype, t, v, z_stride, top, index, slots, tau, &a));
    LPMM_TRY(check_rows(dz, z_dtype, t, v, dz_stride));
    if (t == 0) return LPMM_OK;
    if (dz == z && dz_stride != z_stride) return LPMM_EINVAL;
    LPMM_TRY(check_floats(lse));
    LPMM_TRY(check_floats(grad));
    a.lse = const_cast<float*>(lse);
    a.grad = grad;
    a.dz = dz;
    a.dz_stride = dz_stride;
    return launch_grad(a, z_dtype == LPMM_BF16, static_cast<hipStream_t>(stream));
}

int lpmm_distill_loss_grad(const void* z, int z_dtype, int64_t t, int64_t v, int64_t z_stride, const float* top,
                           const int64_t* index, int slots, float tau, const float* grad, float* loss, float* lse,
                           void* dz, int64_t dz_stride, void* workspace, size_t workspace_bytes, void* stream) {
    DistillArgs a{};
    LPMM_TRY(check_distill(z, z_dtype, t, v, z_stride, top, index, slots, tau, &a));
    LPMM_TRY(check_rows(dz, z_dtype, t, v, dz_stride));
    if (t == 0) return LPMM_OK;
    if (dz == z && dz_stride != z_stride) return LPMM_EINVAL;
    LPMM_TRY(check_floats(loss));
    LPMM_TRY(check_floats(lse));
    LPMM_TRY(check_floats(grad));
    LPMM_TRY(check_workspace(workspace, workspace_bytes, lpmm_distill_workspace_bytes(t, v)));
    a.loss = loss;
    a.lse = lse;
    a.grad = grad;
    a.dz = dz;
    a.dz_stride = dz_stride;
    const bool bf16 = z_dtype == LPMM_BF16;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (launch_both(a, bf16, s)) {
        LPMM_HIP(hipGetLastError());
        return LPMM_OK;
    }
    LPMM_TRY(launch_loss(a, bf16, workspace, s));
    return launch_grad(a, bf16, s);
}

}  // extern "C"
