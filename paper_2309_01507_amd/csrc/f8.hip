// C ABI of matrices in 8 bits and of their products (declared in include/lpmm4.h): argument checks and launches.  The arithmetic is in
// f8.hpp and f8_tile.hpp.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "host_util.hpp"
#include "f8_tile.hpp"

namespace {

using namespace lpmm;

constexpr int64_t kMaxF8Row = int64_t(1) << 22, kMaxF8Codes = int64_t(1) << 33;

int64_t code_bytes(int64_t cols) { return div_up(cols, kF8Block) * kF8Block; }
int64_t scale_bytes(int64_t rows, int64_t cols, int tile) { return div_up(tile == 1 ? rows : div_up(cols, kF8Block), 4) * 4; }

int64_t scale_rows(const F8Mat& m) { return m.shift == 0 ? m.bytes / kF8Block : div_up(m.rows, kF8Block); }

int check_f8(int64_t rows, int64_t cols, int tile, F8Mat* m) {
    if ((tile != 1 && tile != 128) || rows < 0 || cols < 1 || rows > kMaxDim || cols > kMaxF8Row) return LPMM_EINVAL;
    if (rows > kMaxF8Codes / code_bytes(cols)) return LPMM_EINVAL;
    m->rows = int(rows);
    m->bytes = int(code_bytes(cols));
    m->scale_bytes = int(scale_bytes(rows, cols, tile));
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
    const dim3 grid{unsigned(std::min(div_up(m.rows, 4) * div_up(blocks, 4), kMaxBlocks))};          // of at most 2^24: 2^33 codes
    if (dtype == LPMM_BF16)
        hipLaunchKernelGGL(f8_quant_kernel<true>, grid, dim3(256), 0, s, x, stride, m.rows, int(cols), blocks, codes, scales, m.scale_bytes);
    else
        hipLaunchKernelGGL(f8_quant_kernel<false>, grid, dim3(256), 0, s, x, stride, m.rows, int(cols), blocks, codes, scales, m.scale_bytes);
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

int launch_quant_tile(const void* x, int dtype, int64_t stride, int64_t rows, int64_t cols, int tile, const F8Mat& m, const F8Mat& mt, uint8_t* codes,
                      uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, hipStream_t s) {
    const int64_t across = div_up(cols, kF8Block), tiles = across * div_up(rows, kF8Block);
    if (tiles > kMaxBlocks) return LPMM_EINVAL;
    const dim3 grid{unsigned(tiles)};
#define LPMM_F8_TILE(B, T) hipLaunchKernelGGL((f8_quant_tile_kernel<B, T>), grid, dim3(256), 0, s, x, stride, int(rows), int(cols), int(across), codes, scales, m.bytes, \
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

// Tiles of 256 x 256 (8 waves, one workgroup a CU), 128 x 128, 64 x 128 or 64 x 64 (4 waves, two to four workgroups a CU), and the parts of the reduction.
// us of each, b's rows x columns with a's rows: bf16 4096 x 4096: 64 -, 15.3, 12.4, 11.5; 333 27, 23, 16.5, 15.7; 1024 42, 29, 26, 31; 4096 63, 70, -, -;
// 11008 x 4096: 333 41, 30, 33, 40; 1024 53, 58, 64, 74; 2000 103, 94, -, -; 4096 166, 188, -, -; 50257 x 1024: 64 20, 15, 13.4, 14.5; 128 21, 16, 19.5, 19; 512 37, 46, 43, 51;
// fp32 4096 x 4096: 512 40, 32, 28, 29; 4096 110, 121, -, -; 11008 x 4096: 512 69, 56, 51, 61; 1024 99, 95, 96, 107; 50257 x 1024: 128 33, 23, 26, 25
enum class Tile { k256, k128, k64x128, k64 };
struct ProductPlan {
    Tile tile;
    int splits, per;
};
ProductPlan product_plan(int64_t m, int64_t n, int64_t blocks, bool fast) {
    const auto tiles = [&](int64_t rows, int64_t cols) { return div_up(m, rows) * div_up(n, cols); };
    // What a round of workgroups costs, the large tiles' as 10: those run alone on a CU, of 128 x 128 two
    const int64_t large = div_up(tiles(256, 256), 256) * 10, middle = div_up(tiles(128, 128), 512) * (fast ? 6 : 5);
    ProductPlan p{Tile::k64, 1, int(blocks)};
    if (tiles(256, 256) >= 160 && large <= middle) p.tile = Tile::k256;
    else if (tiles(128, 128) >= 250 && (fast || m <= 128)) p.tile = Tile::k128;       // fp32 gains by these, with few rows alone
    else if (tiles(64, 128) >= 280) p.tile = Tile::k64x128;
    const int64_t small = tiles(64, 64);
    // A block takes a tile of 64 x 64 some 0.28 us (fp32 0.45), the join 2.5 us and 0.2 more for each part: parts pay where CUs have less than two workgroups, and two parts
    // for long sums where they have no more than two (us without parts and with, bf16: 17 x 8192 x 4096 20.3, 13.5; 17 x 8192 x 8192 35, 18; 17 x 11008 x 4096 20.9, 16.6; 64 x
    // 16384 x 4096 23.0, 20.9; 128 x 4096 x 11008 47, 24; 200 x 4096 x 4096 20.7, 21.2; 333 x 4096 x 11008 50, 39; with three where two are taken 128 x 4096 x 4096 17.8, 19.7)
    const double whole = double(blocks) * (fast ? 0.28 : 0.45);
    if (p.tile == Tile::k64 && small <= 512 && whole >= 6.0) {
        const int64_t want = std::min<int64_t>(std::max<int64_t>(512 / small, whole >= 20.0 ? 2 : 1), int64_t(std::sqrt(whole / 0.2)));
        p.per = int(div_up(blocks, std::max<int64_t>(1, want)));
        p.splits = int(div_up(blocks, p.per));
    }
    return p;
}
size_t product_bytes(int64_t m, int64_t n, const ProductPlan& p) { return p.splits > 1 ? size_t(p.splits) * size_t(m) * size_t(n) * 4 : 0; }

int launch_product(const F8Mat& a, const F8Mat& b, void* c, int dtype, int64_t stride, void* workspace, hipStream_t s) {
    if (a.rows == 0 || b.rows == 0) return LPMM_OK;
    const bool fast = dtype == LPMM_BF16;
    const ProductPlan p = product_plan(a.rows, b.rows, a.bytes / kF8Block, fast);
    const int64_t bm = p.tile == Tile::k256 ? 256 : p.tile == Tile::k128 ? 128 : 64, bn = p.tile == Tile::k256 ? 256 : p.tile == Tile::k64 ? 64 : 128;
    const int64_t m_tiles = div_up(a.rows, bm), n_tiles = div_up(b.rows, bn), blocks = div_up(m_tiles * n_tiles, 8) * 8;
    if (blocks > kMaxBlocks) return LPMM_EINVAL;
    float* parts = p.splits > 1 ? static_cast<float*>(workspace) : nullptr;
    const dim3 grid(unsigned(blocks), unsigned(p.splits));
#define LPMM_TILE(WM, WN, MT, NT) { \
        if (fast) hipLaunchKernelGGL((f8_tile_kernel<true, WM, WN, MT, NT>), grid, dim3(64 * WM * WN), 0, s, a, b, c, stride, int(m_tiles), int(n_tiles), p.per, parts); \
        else hipLaunchKernelGGL((f8_tile_kernel<false, WM, WN, MT, NT>), grid, dim3(64 * WM * WN), 0, s, a, b, c, stride, int(m_tiles), int(n_tiles), p.per, parts); }
    if (p.tile == Tile::k256) LPMM_TILE(4, 2, 2, 4)
    else if (p.tile == Tile::k128) LPMM_TILE(2, 2, 2, 2)
    else if (p.tile == Tile::k64x128) LPMM_TILE(2, 2, 1, 2)
    else LPMM_TILE(2, 2, 1, 1)
#undef LPMM_TILE
    LPMM_HIP(hipGetLastError());
    if (parts) {
        const dim3 groups{unsigned(div_up(int64_t(a.rows) * b.rows, 256))};        // at most 512 tiles of 64 x 64
        if (fast) hipLaunchKernelGGL(f8_join_kernel<true>, groups, dim3(256), 0, s, parts, p.splits, a.rows, b.rows, c, stride);
        else hipLaunchKernelGGL(f8_join_kernel<false>, groups, dim3(256), 0, s, parts, p.splits, a.rows, b.rows, c, stride);
        LPMM_HIP(hipGetLastError());
    }
    return LPMM_OK;
}

// Up to 16 tokens whose codes LDS holds have a kernel of their own
bool few(int64_t t, int64_t bytes) { return t <= kF8FewTokens && t * bytes <= kF8FewBytes; }
// but not for results in bf16 where every workgroup brings so much to 8 bits that one is all a CU has room for, and W has many rows, up to 2^28 codes (us, that kernel and the
// tiles, bf16: 16 tokens 24576 x 4096 24.9, 21.5; 28672 x 4096 27.3, 22.0; 32000 x 4096 29.3, 27.5; 50257 x 4096 40.8, 34.3; 65536 x 4096 48.4, 44.2; 50257 x 2560
// 29.3, 24.1; 12 tokens 24576 x 4096 23.5, 21.5; 32000 x 4096 27.9, 27.4; 36864 x 4096 29.0, 29.4; 50257 x 5120 45.4, 44.8; where it stays 8 tokens 32000 x 4096 26.5, 27.3; 16 tokens
// 16384 x 2560 13.3, 15.3; 20000 x 4096 22.1, 21.1; 100000 x 4096 80.5, 86.2; 32000 x 2048 15.5, 17.6; fp32 16 tokens 32000 x 4096 30.0, 35.9)
bool few_by_tiles(int64_t t, int64_t rows, int64_t bytes) { return t >= 12 && t * bytes > 32768 && rows >= 24576 && rows * bytes <= int64_t(1) << 28; }

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// A matrix laid out in a caller's memory from `at` on, which moves behind it
F8Mat carve(char*& at, int64_t rows, int64_t cols, int tile) {
    F8Mat m{};
    check_f8(rows, cols, tile, &m);                              // the caller has checked them
    m.codes = reinterpret_cast<uint8_t*>(at);
    at += up16(size_t(m.rows) * m.bytes);
    m.scales = reinterpret_cast<uint8_t*>(at);
    at += up16(size_t(scale_rows(m)) * m.scale_bytes);
    return m;
}
size_t carved(int64_t rows, int64_t cols, int tile) {
    char* at = nullptr;
    carve(at, rows, cols, tile);
    return size_t(at - static_cast<char*>(nullptr));
}

int check_train(int64_t t, int64_t n, int64_t k, int grads) {
    F8Mat m{};
    if (t < 1 || t > kMaxTokens || t > kMaxF8Row || n < 1 || n > kMaxF8Row || grads < 0 || grads > 3) return LPMM_EINVAL;
    LPMM_TRY(check_f8(t, k, 1, &m));
    LPMM_TRY(check_f8(k, t, 1, &m));
    LPMM_TRY(check_f8(t, n, 1, &m));
    LPMM_TRY(check_f8(n, t, 1, &m));
    LPMM_TRY(check_f8(k, n, 128, &m));
    return check_f8(n, k, 128, &m);
}

uint8_t* writable(const uint8_t* p) { return const_cast<uint8_t*>(p); }

int quant_into(const void* x, int dtype, int64_t stride, int64_t rows, int64_t cols, int tile, const F8Mat& m, const F8Mat& mt, hipStream_t s) {
    if (tile == 1 && !mt.codes) return launch_quant(x, dtype, stride, m, cols, writable(m.codes), writable(m.scales), s);
    return launch_quant_tile(x, dtype, stride, rows, cols, tile, m, mt, writable(m.codes), writable(m.scales), writable(mt.codes), writable(mt.scales), s);
}

}  // namespace

extern "C" {

int lpmm_f8_sizes(int64_t rows, int64_t cols, int tile, size_t sizes[2]) {
    F8Mat m{};
    if (!sizes) return LPMM_EINVAL;
    LPMM_TRY(check_f8(rows, cols, tile, &m));
    sizes[0] = size_t(m.rows) * m.bytes;
    sizes[1] = size_t(scale_rows(m)) * m.scale_bytes;
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
    const int64_t blocks = a.bytes / kF8Block;
    return std::max(product_bytes(a_rows, b_rows, product_plan(a_rows, b_rows, blocks, false)), product_bytes(a_rows, b_rows, product_plan(a_rows, b_rows, blocks, true)));
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
    if (t < 1 || t > kMaxTokens || check_f8(t, k, 1, &x) || check_f8(n, k, 128, &w) || n < 1 || (few(t, x.bytes) && !few_by_tiles(t, n, x.bytes))) return 0;
    return up16(size_t(t) * x.bytes) + up16(size_t(scale_rows(x)) * x.scale_bytes) + lpmm_f8_matmul_workspace_bytes(t, n, k);
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
    if (few(t, mw.bytes) && !(dtype == LPMM_BF16 && few_by_tiles(t, mw.rows, mw.bytes))) {
        const size_t lds = up16(size_t(t) * (mw.bytes + mw.bytes / kF8Block));
        // 16 waves share the blocks of 16 rows; of rows of about 4096 two share those of 32 where tiles of 128 rows are one a CU, nearly (us, 1 token bf16, each: 4096 x 4096 5.3, 18;
        // 16384 x 4096 13.0, 18.2; 24576 x 4096 20.3, 18.5; 28672 x 4096 22.5, 19.9; 32000 x 4096 24.7, 21.7, 8 tokens 26.5, 25.9, 16 tokens 29.3, 30.2; 36864 x 4096 25.6, 34.4; 50257 x
        // 4096 34.6, 35.3; 32000 x 5120 25.0, 26.3; 32000 x 2048 11.9, 13.7; 50257 x 1024 10.6, 11.5).  Two workgroups a CU while x leaves room for them (16 tokens 11008 x 4096 one 16.1, two 24)
        const int64_t most = lds <= 32768 ? 512 : 256;
        const int blocks = mw.bytes / kF8Block;
        const bool wide = t <= 8 && blocks >= 32 && blocks < 40 && mw.rows >= 24576 && mw.rows <= 32768;
#define LPMM_FEW(B, K, N, T) hipLaunchKernelGGL((f8_few_kernel<B, K, N, T, 2>), dim3(unsigned(std::min<int64_t>(most, div_up(mw.rows, 16 * T * N)))), dim3(64 * K * N), lds, \
                                                s, mw, x, int(t), int(w->cols), x_stride, y, y_stride)
        if (wide) { if (dtype == LPMM_BF16) LPMM_FEW(true, 2, 4, 2); else LPMM_FEW(false, 2, 4, 2); }
        else { if (dtype == LPMM_BF16) LPMM_FEW(true, 16, 1, 1); else LPMM_FEW(false, 16, 1, 1); }
#undef LPMM_FEW
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
    return launch_product(mx, mw, y, dtype, y_stride, scales + up16(size_t(scale_rows(mx)) * mx.scale_bytes), s);
}

size_t lpmm_f8_train_kept_bytes(int64_t t, int64_t n, int64_t k, int grads) {
    if (check_train(t, n, k, grads)) return 0;
    return (grads & LPMM_F8_DX ? carved(k, n, 128) : 0) + (grads & LPMM_F8_DW ? carved(k, t, 1) : 0);
}

size_t lpmm_f8_train_workspace_bytes(int64_t t, int64_t n, int64_t k) {
    if (check_train(t, n, k, 0)) return 0;
    const size_t forward = carved(t, k, 1) + carved(n, k, 128) + lpmm_f8_matmul_workspace_bytes(t, n, k);
    const size_t backward = carved(t, n, 1) + carved(n, t, 1) + std::max(lpmm_f8_matmul_workspace_bytes(t, k, n), lpmm_f8_matmul_workspace_bytes(n, k, t));
    return std::max(forward, backward);
}

int lpmm_f8_train_forward(const void* x, int dtype, int64_t t, int64_t x_stride, const void* w, int w_dtype, int64_t n, int64_t k, int64_t w_stride, int grads,
                          void* y, int64_t y_stride, void* kept, size_t kept_bytes, void* workspace, size_t workspace_bytes, void* stream) {
    LPMM_TRY(check_train(t, n, k, grads));
    LPMM_TRY(check_rows(x, dtype, t, k, x_stride));
    LPMM_TRY(check_rows(w, w_dtype, n, k, w_stride));
    LPMM_TRY(check_rows(y, dtype, t, n, y_stride));
    LPMM_TRY(check_workspace(kept, kept_bytes, lpmm_f8_train_kept_bytes(t, n, k, grads)));
    LPMM_TRY(check_workspace(workspace, workspace_bytes, lpmm_f8_train_workspace_bytes(t, n, k)));
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* at = static_cast<char*>(workspace);
    const F8Mat qx = carve(at, t, k, 1), qw = carve(at, n, k, 128);
    char* keep = static_cast<char*>(kept);
    const F8Mat qwt = grads & LPMM_F8_DX ? carve(keep, k, n, 128) : F8Mat{}, qxt = grads & LPMM_F8_DW ? carve(keep, k, t, 1) : F8Mat{};
    LPMM_TRY(quant_into(w, w_dtype, w_stride, n, k, 128, qw, qwt, s));
    LPMM_TRY(quant_into(x, dtype, x_stride, t, k, 1, qx, qxt, s));
    return launch_product(qx, qw, y, dtype, y_stride, at, s);
}

int lpmm_f8_train_backward(const void* dy, int dtype, int64_t t, int64_t dy_stride, int64_t n, int64_t k, int grads, const void* kept, size_t kept_bytes, void* dx,
                           int64_t dx_stride, void* dw, int w_dtype, int64_t dw_stride, void* workspace, size_t workspace_bytes, void* stream) {
    LPMM_TRY(check_train(t, n, k, grads));
    const bool want_x = grads & LPMM_F8_DX, want_w = grads & LPMM_F8_DW;
    LPMM_TRY(check_rows(dy, dtype, t, n, dy_stride));
    if (want_x) LPMM_TRY(check_rows(dx, dtype, t, k, dx_stride));
    if (want_w) LPMM_TRY(check_rows(dw, w_dtype, n, k, dw_stride));
    LPMM_TRY(check_workspace(kept, kept_bytes, lpmm_f8_train_kept_bytes(t, n, k, grads)));
    LPMM_TRY(check_workspace(workspace, workspace_bytes, lpmm_f8_train_workspace_bytes(t, n, k)));
    if (!want_x && !want_w) return LPMM_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* at = static_cast<char*>(workspace);
    const F8Mat q = want_x ? carve(at, t, n, 1) : F8Mat{}, qt = want_w ? carve(at, n, t, 1) : F8Mat{};
    char* keep = static_cast<char*>(const_cast<void*>(kept));
    const F8Mat qwt = want_x ? carve(keep, k, n, 128) : F8Mat{}, qxt = want_w ? carve(keep, k, t, 1) : F8Mat{};
    LPMM_TRY(quant_into(dy, dtype, dy_stride, t, n, 1, q, qt, s));
    if (want_x) LPMM_TRY(launch_product(q, qwt, dx, dtype, dx_stride, at, s));
    if (want_w) LPMM_TRY(launch_product(qt, qxt, dw, w_dtype, dw_stride, at, s));
    return LPMM_OK;
}

}  // extern "C"
