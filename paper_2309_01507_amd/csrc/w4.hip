// C ABI of the 4-bit weights and of distillation (declared in include/lpmm4.h): argument checks and launches.  The arithmetic is
// in w4.hpp and distill.hpp.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "host_util.hpp"
#include "w4.hpp"
#include "distill.hpp"

namespace {

using namespace lpmm;

constexpr int64_t kMaxDim = (int64_t(1) << 31) - 1 - 2 * kW4Chunk;
constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 1;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
int group_shift(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }
int elem_size(int dtype) { return dtype == LPMM_BF16 ? 2 : 4; }

int check_w4(const int64_t* shape, int group, W4Mat* m) {
    if (!shape || (group != 32 && group != 64 && group != 128)) return LPMM_EINVAL;
    if (shape[0] < 1 || shape[1] < 1 || shape[0] > kMaxDim || shape[1] > kMaxDim) return LPMM_EINVAL;
    const int64_t kp = div_up(shape[1], kW4Chunk) * kW4Chunk;
    if (shape[0] > (int64_t(1) << 37) / kp) return LPMM_EINVAL;
    m->n = int(shape[0]);
    m->k = int(shape[1]);
    m->words = int(kp / 8);
    m->groups = int(div_up(shape[1], group));
    return LPMM_OK;
}

// `rows` rows of `len` elements, `stride` apart
int check_rows(const void* p, int dtype, int64_t rows, int64_t len, int64_t stride) {
    if (dtype != LPMM_F32 && dtype != LPMM_BF16) return LPMM_EINVAL;
    if (rows < 0 || rows > kMaxTokens || stride < len || stride > (int64_t(1) << 40)) return LPMM_EINVAL;
    if (rows > 0 && (!p || !aligned(p, elem_size(dtype)))) return LPMM_EINVAL;
    return LPMM_OK;
}

int check_codes(const uint8_t* codes) { return codes && aligned(codes, 16) ? LPMM_OK : LPMM_EINVAL; }
int check_floats(const float* p) { return p && aligned(p, 4) ? LPMM_OK : LPMM_EINVAL; }

#define LPMM_TRY(call) do { const int rc_ = (call); if (rc_) return rc_; } while (0)

int check_distill(const void* z, int z_dtype, int64_t t, int64_t v, int64_t z_stride, const float* top,
                  const int64_t* index, int slots, float tau, DistillArgs* a) {
    if (v < 1 || v > kMaxDim || slots < 1 || slots > LPMM_DISTILL_MAX_SLOTS) return LPMM_EINVAL;
    if (!std::isfinite(tau) || !(tau > 0.0f) || !std::isfinite(1.0f / tau)) return LPMM_EINVAL;
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
    return LPMM_OK;
}

int launch_loss(const DistillArgs& a, bool bf16, hipStream_t s) {
    if (bf16) hipLaunchKernelGGL((distill_loss_kernel<true, 1024>), dim3(unsigned(a.t)), dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((distill_loss_kernel<false, 1024>), dim3(unsigned(a.t)), dim3(1024), 0, s, a);
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

int launch_grad(const DistillArgs& a, bool bf16, hipStream_t s) {
    const int span = 8192;
    constexpr int64_t kRows = 32768;                     // of a launch: grid.y
    for (int64_t r = 0; r < a.t; r += kRows) {
        DistillArgs b = a;
        b.z = static_cast<const char*>(a.z) + r * a.z_stride * (bf16 ? 2 : 4);
        b.dz = static_cast<char*>(a.dz) + r * a.dz_stride * (bf16 ? 2 : 4);
        b.top += r * a.slots;
        b.index += r * a.slots;
        b.grad += r;
        b.lse += r;
        const dim3 grid(unsigned(div_up(a.v, span)), unsigned(std::min(kRows, a.t - r)));
        if (bf16) hipLaunchKernelGGL(distill_grad_kernel<true>, grid, dim3(kDistillThreads), 0, s, b, span);
        else hipLaunchKernelGGL(distill_grad_kernel<false>, grid, dim3(kDistillThreads), 0, s, b, span);
        LPMM_HIP(hipGetLastError());
    }
    return LPMM_OK;
}

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
    LPMM_TRY(check_rows(x, dtype, t, m.k, x_stride));
    LPMM_TRY(check_rows(y, dtype, t, m.n, y_stride));
    LPMM_TRY(check_codes(codes));
    LPMM_TRY(check_floats(scales));
    if (t == 0) return LPMM_OK;
    m.codes = reinterpret_cast<const uint32_t*>(codes);
    m.scales = scales;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int esize = elem_size(dtype);
    constexpr int64_t kTokens = 16 * 32768;              // of a launch: grid.y
    for (int64_t at = 0; at < t; at += kTokens) {
        const int part = int(std::min(kTokens, t - at));
        const void* xp = static_cast<const char*>(x) + at * x_stride * esize;
        void* yp = static_cast<char*>(y) + at * y_stride * esize;
        const dim3 grid(unsigned(div_up(m.n, 16)), unsigned(div_up(part, 16)));
#define LPMM_LINEAR(B, G) hipLaunchKernelGGL((w4_linear_kernel<B, G, 4>), grid, dim3(256), 0, s, m, xp, part, x_stride, yp, y_stride)
        if (dtype == LPMM_BF16) {
            if (group == 32) LPMM_LINEAR(true, 32); else if (group == 64) LPMM_LINEAR(true, 64); else LPMM_LINEAR(true, 128);
        } else {
            if (group == 32) LPMM_LINEAR(false, 32); else if (group == 64) LPMM_LINEAR(false, 64); else LPMM_LINEAR(false, 128);
        }
#undef LPMM_LINEAR
        LPMM_HIP(hipGetLastError());
    }
    return LPMM_OK;
}

int lpmm_w4_linear_dx(const void* dy, int dtype, int64_t t, int64_t dy_stride, const uint8_t* codes,
                      const float* scales, const int64_t shape[2], int group, void* dx, int64_t dx_stride,
                      void* stream) {
    W4Mat m{};
    LPMM_TRY(check_w4(shape, group, &m));
    LPMM_TRY(check_rows(dy, dtype, t, m.n, dy_stride));
    LPMM_TRY(check_rows(dx, dtype, t, m.k, dx_stride));
    LPMM_TRY(check_codes(codes));
    LPMM_TRY(check_floats(scales));
    if (t == 0) return LPMM_OK;
    m.codes = reinterpret_cast<const uint32_t*>(codes);
    m.scales = scales;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int esize = elem_size(dtype);
    constexpr int64_t kTokens = 32768;                   // of a launch: grid.y
    for (int64_t at = 0; at < t; at += kTokens) {
        const int part = int(std::min(kTokens, t - at));
        const void* dyp = static_cast<const char*>(dy) + at * dy_stride * esize;
        void* dxp = static_cast<char*>(dx) + at * dx_stride * esize;
        const dim3 grid(unsigned(div_up(m.words, 256)), unsigned(part));
        if (dtype == LPMM_BF16) hipLaunchKernelGGL(w4_dx_kernel<true>, grid, dim3(256), 0, s, m, dyp, part, dy_stride, dxp, dx_stride, group_shift(group));
        else hipLaunchKernelGGL(w4_dx_kernel<false>, grid, dim3(256), 0, s, m, dyp, part, dy_stride, dxp, dx_stride, group_shift(group));
        LPMM_HIP(hipGetLastError());
    }
    return LPMM_OK;
}

size_t lpmm_w4_linear_dscale_workspace_bytes(int64_t t, const int64_t shape[2], int group) {
    (void)t; (void)shape; (void)group;
    return 0;
}

int lpmm_w4_linear_dscale(const void* x, const void* dy, int dtype, int64_t t, int64_t x_stride, int64_t dy_stride,
                          const uint8_t* codes, const int64_t shape[2], int group, float* dscales, void* workspace,
                          size_t workspace_bytes, void* stream) {
    W4Mat m{};
    LPMM_TRY(check_w4(shape, group, &m));
    LPMM_TRY(check_rows(x, dtype, t, m.k, x_stride));
    LPMM_TRY(check_rows(dy, dtype, t, m.n, dy_stride));
    LPMM_TRY(check_codes(codes));
    LPMM_TRY(check_floats(dscales));
    (void)workspace; (void)workspace_bytes;
    m.codes = reinterpret_cast<const uint32_t*>(codes);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t blocks = div_up(int64_t(m.n) * m.groups, 4);
    if (blocks > 0x7FFFFFFF) return LPMM_EINVAL;
    if (dtype == LPMM_BF16) hipLaunchKernelGGL(w4_dscale_kernel<true>, dim3(unsigned(blocks)), dim3(256), 0, s, m, x, dy, int(t), x_stride, dy_stride, group_shift(group), dscales);
    else hipLaunchKernelGGL(w4_dscale_kernel<false>, dim3(unsigned(blocks)), dim3(256), 0, s, m, x, dy, int(t), x_stride, dy_stride, group_shift(group), dscales);
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

size_t lpmm_distill_workspace_bytes(int64_t t, int64_t v) {
    (void)t; (void)v;
    return 0;
}

int lpmm_distill_loss(const void* z, int z_dtype, int64_t t, int64_t v, int64_t z_stride, const float* top,
                      const int64_t* index, int slots, float tau, float* loss, float* lse, void* workspace,
                      size_t workspace_bytes, void* stream) {
    DistillArgs a{};
    LPMM_TRY(check_distill(z, z_dtype, t, v, z_stride, top, index, slots, tau, &a));
    if (t == 0) return LPMM_OK;
    LPMM_TRY(check_floats(loss));
    LPMM_TRY(check_floats(lse));
    (void)workspace; (void)workspace_bytes;
    a.loss = loss;
    a.lse = lse;
    return launch_loss(a, z_dtype == LPMM_BF16, static_cast<hipStream_t>(stream));
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
    (void)workspace; (void)workspace_bytes;
    a.loss = loss;
    a.lse = lse;
    a.grad = grad;
    a.dz = dz;
    a.dz_stride = dz_stride;
    const bool bf16 = z_dtype == LPMM_BF16;
    hipStream_t s = static_cast<hipStream_t>(stream);
    LPMM_TRY(launch_loss(a, bf16, s));
    return launch_grad(a, bf16, s);
}

}  // extern "C"
