// C ABI of matrices in 8 bits and of their products (declared in include/lpmm4.h): argument checks and launches.  The arithmetic is in
// f8.hpp and f8_tile.hpp.

#include <hip/hip_runtime.h>

#include <algorithm>

#include "host_util.hpp"
#include "f8_tile.hpp"

namespace {

using namespace lpmm;

constexpr int64_t kMaxF8Row = int64_t(1) << 22, kMaxF8Codes = int64_t(1) << 33;

int64_t code_bytes(int64_t cols) { return div_up(cols, kF8Block) * kF8Block; }
int64_t scale_bytes(int64_t cols) { return div_up(div_up(cols, kF8Block), 4) * 4; }

int check_f8(int64_t rows, int64_t cols, int tile, F8Mat* m) {
    if ((tile != 1 && tile != 128) || rows < 0 || cols < 1 || rows > kMaxDim || cols > kMaxF8Row) return LPMM_EINVAL;
    if (rows > kMaxF8Codes / code_bytes(cols)) return LPMM_EINVAL;
    m->rows = int(rows);
    m->bytes = int(code_bytes(cols));
    m->scale_bytes = int(scale_bytes(cols));
    m->shift = tile == 1 ? 0 : 7;
    return LPMM_OK;
}

int check_f8(const lpmm_f8* f, F8Mat* m) {
    if (!f) return LPMM_EINVAL;
    LPMM_TRY(check_f8(f->rows, f->cols, f->tile, m));
    if (m->rows > 0 && (check_codes(f->codes) || !f->scales || !aligned(f->scales, 4))) return LPMM_EINVAL;
    m->codes = f->codes;
    m->scales = f->scales;
    return LPMM_OK;
}

int launch_quant(const void* x, int dtype, int64_t stride, const F8Mat& m, int64_t cols, uint8_t* codes, uint8_t* scales, hipStream_t s) {
    const int blocks = m.bytes / kF8Block;
    const int64_t groups = div_up(int64_t(m.rows) * blocks, 16);
    if (groups > kMaxBlocks) return LPMM_EINVAL;
    const dim3 grid{unsigned(groups)};
    if (dtype == LPMM_BF16)
        hipLaunchKernelGGL(f8_quant_kernel<true>, grid, dim3(256), 0, s, x, stride, m.rows, int(cols), blocks, codes, scales, m.scale_bytes);
    else
        hipLaunchKernelGGL(f8_quant_kernel<false>, grid, dim3(256), 0, s, x, stride, m.rows, int(cols), blocks, codes, scales, m.scale_bytes);
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

// Tiles down the rows go in launches of at most 2^15
int launch_quant_tile(const void* x, int dtype, int64_t stride, int64_t rows, int64_t cols, int tile, const F8Mat& m, const F8Mat& mt, uint8_t* codes,
                      uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, hipStream_t s) {
    const int64_t across = div_up(cols, kF8Block), down = div_up(rows, kF8Block);
    if (down > 65535) return LPMM_EINVAL;
    const dim3 grid{unsigned(across), unsigned(down)};
#define LPMM_F8_TILE(B, T) hipLaunchKernelGGL((f8_quant_tile_kernel<B, T>), grid, dim3(256), 0, s, x, stride, int(rows), int(cols), codes, scales, m.bytes, \
                                              m.scale_bytes, codes_t, scales_t, mt.bytes, mt.scale_bytes)
    if (dtype == LPMM_BF16) { if (tile == 1) LPMM_F8_TILE(true, 1); else LPMM_F8_TILE(true, 128); }
    else { if (tile == 1) LPMM_F8_TILE(false, 1); else LPMM_F8_TILE(false, 128); }
#undef LPMM_F8_TILE
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

int check_out(const lpmm_f8* f, int64_t rows, int64_t cols, int tile, F8Mat* m) {
    LPMM_TRY(check_f8(f, m));
    return f->rows == rows && f->cols == cols && f->tile == tile ? LPMM_OK : LPMM_EINVAL;
}

// Parts of the reduction: as many as fill the GPU once
struct ProductPlan {
    int splits, per;
};
ProductPlan product_plan(int64_t m, int64_t n, int64_t blocks) {
    const int64_t tiles = div_up(m, 128) * div_up(n, 128);
    const int64_t want = std::max<int64_t>(1, std::min(blocks / 2, 512 / std::max<int64_t>(1, tiles)));
    ProductPlan p{};
    p.per = int(div_up(blocks, want));
    p.splits = int(div_up(blocks, p.per));
    return p;
}
size_t product_bytes(int64_t m, int64_t n, const ProductPlan& p) { return p.splits > 1 ? size_t(p.splits) * size_t(m) * size_t(n) * 4 : 0; }

int launch_product(const F8Mat& a, const F8Mat& b, void* c, int dtype, int64_t stride, void* workspace, hipStream_t s) {
    if (a.rows == 0 || b.rows == 0) return LPMM_OK;
    const ProductPlan p = product_plan(a.rows, b.rows, a.bytes / kF8Block);
    const int64_t m_tiles = div_up(a.rows, 128), n_tiles = div_up(b.rows, 128), blocks = div_up(m_tiles * n_tiles, 8) * 8;
    if (blocks > kMaxBlocks) return LPMM_EINVAL;
    float* parts = p.splits > 1 ? static_cast<float*>(workspace) : nullptr;
    const dim3 grid(unsigned(blocks), unsigned(p.splits));
    if (dtype == LPMM_BF16) hipLaunchKernelGGL((f8_tile_kernel<true, true, 2, 2, 2, 2>), grid, dim3(256), 0, s, a, b, c, stride, int(m_tiles), int(n_tiles), p.per, parts);
    else hipLaunchKernelGGL((f8_tile_kernel<false, false, 2, 2, 2, 2>), grid, dim3(256), 0, s, a, b, c, stride, int(m_tiles), int(n_tiles), p.per, parts);
    LPMM_HIP(hipGetLastError());
    if (parts) {
        const int64_t groups = div_up(int64_t(a.rows) * b.rows, 256);
        if (groups > kMaxBlocks) return LPMM_EINVAL;
        if (dtype == LPMM_BF16) hipLaunchKernelGGL(f8_join_kernel<true>, dim3(unsigned(groups)), dim3(256), 0, s, parts, p.splits, a.rows, b.rows, c, stride);
        else hipLaunchKernelGGL(f8_join_kernel<false>, dim3(unsigned(groups)), dim3(256), 0, s, parts, p.splits, a.rows, b.rows, c, stride);
        LPMM_HIP(hipGetLastError());
    }
    return LPMM_OK;
}

constexpr int kF8Few = 16;               // tokens that a wave's operand holds

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

}  // namespace

extern "C" {

int lpmm_f8_sizes(int64_t rows, int64_t cols, int tile, size_t sizes[2]) {
    F8Mat m{};
    if (!sizes) return LPMM_EINVAL;
    LPMM_TRY(check_f8(rows, cols, tile, &m));
    sizes[0] = size_t(m.rows) * m.bytes;
    sizes[1] = size_t(div_up(rows, tile)) * m.scale_bytes;
    return LPMM_OK;
}

int lpmm_f8_quant(const void* x, int dtype, int64_t stride, const lpmm_f8* out, void* stream) {
    F8Mat m{};
    LPMM_TRY(check_f8(out, &m));
    LPMM_TRY(check_rows(x, dtype, out->rows, out->cols, stride));
    if (m.rows == 0) return LPMM_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (out->tile == 1) return launch_quant(x, dtype, stride, m, out->cols, out->codes, out->scales, s);
    return launch_quant_tile(x, dtype, stride, out->rows, out->cols, 128, m, F8Mat{}, out->codes, out->scales, nullptr, nullptr, s);
}

int lpmm_f8_quant_both(const void* x, int dtype, int64_t stride, const lpmm_f8* out, const lpmm_f8* out_t, void* stream) {
    F8Mat m{}, mt{};
    LPMM_TRY(check_f8(out, &m));
    if (out->rows < 1) return LPMM_EINVAL;                       // a transpose has columns
    LPMM_TRY(check_out(out_t, out->cols, out->rows, out->tile, &mt));
    LPMM_TRY(check_rows(x, dtype, out->rows, out->cols, stride));
    return launch_quant_tile(x, dtype, stride, out->rows, out->cols, out->tile, m, mt, out->codes, out->scales, out_t->codes, out_t->scales,
                             static_cast<hipStream_t>(stream));
}

int lpmm_f8_dequant(const lpmm_f8* f, void* out, int dtype, int64_t stride, void* stream) {
    F8Mat m{};
    LPMM_TRY(check_f8(f, &m));
    LPMM_TRY(check_rows(out, dtype, f->rows, f->cols, stride));
    if (m.rows == 0) return LPMM_OK;
    const int blocks = m.bytes / kF8Block;
    const int64_t groups = div_up(int64_t(m.rows) * blocks, 16);
    if (groups > kMaxBlocks) return LPMM_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == LPMM_BF16) hipLaunchKernelGGL(f8_dequant_kernel<true>, dim3(unsigned(groups)), dim3(256), 0, s, m, int(f->cols), blocks, out, stride);
    else hipLaunchKernelGGL(f8_dequant_kernel<false>, dim3(unsigned(groups)), dim3(256), 0, s, m, int(f->cols), blocks, out, stride);
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

size_t lpmm_f8_matmul_workspace_bytes(int64_t a_rows, int64_t b_rows, int64_t cols) {
    F8Mat a{}, b{};
    if (check_f8(a_rows, cols, 1, &a) || check_f8(b_rows, cols, 1, &b) || a_rows < 1 || b_rows < 1) return 0;
    return product_bytes(a_rows, b_rows, product_plan(a_rows, b_rows, a.bytes / kF8Block));
}

int lpmm_f8_matmul(const lpmm_f8* a, const lpmm_f8* b, void* c, int dtype, int64_t stride, void* workspace, size_t workspace_bytes, void* stream) {
    F8Mat ma{}, mb{};
    LPMM_TRY(check_f8(a, &ma));
    LPMM_TRY(check_f8(b, &mb));
    if (a->cols != b->cols) return LPMM_EINVAL;
    LPMM_TRY(check_rows(c, dtype, b->rows ? a->rows : 0, b->rows, stride));          // without columns there is nothing to point at
    LPMM_TRY(check_workspace(workspace, workspace_bytes, lpmm_f8_matmul_workspace_bytes(a->rows, b->rows, a->cols)));
    return launch_product(ma, mb, c, dtype, stride, workspace, static_cast<hipStream_t>(stream));
}

size_t lpmm_f8_linear_workspace_bytes(int64_t t, int64_t n, int64_t k) {
    F8Mat x{}, w{};
    if (t <= kF8Few || t > kMaxTokens || check_f8(t, k, 1, &x) || check_f8(n, k, 128, &w) || n < 1) return 0;
    return up16(size_t(t) * x.bytes) + up16(size_t(t) * x.scale_bytes) + lpmm_f8_matmul_workspace_bytes(t, n, k);
}

int lpmm_f8_linear(const void* x, int dtype, int64_t t, int64_t x_stride, const lpmm_f8* w, void* y, int64_t y_stride, void* workspace,
                   size_t workspace_bytes, void* stream) {
    F8Mat mw{}, mx{};
    LPMM_TRY(check_f8(w, &mw));
    if (t > kMaxTokens) return LPMM_EINVAL;
    LPMM_TRY(check_rows(x, dtype, t, w->cols, x_stride));
    LPMM_TRY(check_rows(y, dtype, w->rows ? t : 0, w->rows, y_stride));
    if (t == 0 || mw.rows == 0) return LPMM_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (t <= kF8Few) {
        const dim3 grid{unsigned(div_up(mw.rows, 16))};
        if (dtype == LPMM_BF16) hipLaunchKernelGGL((f8_few_kernel<true, 1, 8>), grid, dim3(512), 0, s, mw, x, int(t), int(w->cols), x_stride, y, y_stride);
        else hipLaunchKernelGGL((f8_few_kernel<false, 1, 8>), grid, dim3(512), 0, s, mw, x, int(t), int(w->cols), x_stride, y, y_stride);
        LPMM_HIP(hipGetLastError());
        return LPMM_OK;
    }
    LPMM_TRY(check_f8(t, w->cols, 1, &mx));
    LPMM_TRY(check_workspace(workspace, workspace_bytes, lpmm_f8_linear_workspace_bytes(t, w->rows, w->cols)));
    uint8_t* codes = static_cast<uint8_t*>(workspace);
    uint8_t* scales = codes + up16(size_t(t) * mx.bytes);
    mx.codes = codes;
    mx.scales = scales;
    LPMM_TRY(launch_quant(x, dtype, x_stride, mx, w->cols, codes, scales, s));
    return launch_product(mx, mw, y, dtype, y_stride, scales + up16(size_t(t) * mx.scale_bytes), s);
}

}  // extern "C"
