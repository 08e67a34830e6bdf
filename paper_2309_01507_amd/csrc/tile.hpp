// What tiled products share: the matrix instruction on bf16, the order of tiles, pieces in LDS, loads straight into it.
//
// Operand layout of v_mfma_f32_32x32x16_bf16: lane l holds, of row (A) or column (B) l % 32, the reduction's elements 8 (l / 32)
// .. + 7; of the result column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4 for i = 0..15.
#pragma once

#include "rows.hpp"

namespace lpmm {

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ int wave_number() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }      // as a scalar
__device__ __forceinline__ int mfma32_row(int i, int half) { return 8 * (i >> 2) + 4 * half + (i & 3); }

// Workgroups go round robin over the 8 XCDs; so that each XCD's L2 serves neighbouring tiles, XCD x takes the x-th eighth of them,
// in an order that walks down `rows` in strips of 4 columns.  False: nothing to do.
__device__ __forceinline__ bool tile_of(int id, int rows, int cols, int& row, int& col) {
    const int total = rows * cols, per = (total + 7) >> 3;
    const int tile = (id & 7) * per + (id >> 3);
    if ((id >> 3) >= per || tile >= total) return false;
    const int strip = tile / (4 * rows), rest = tile - strip * 4 * rows;
    const int width = min(4, cols - strip * 4);
    row = rest / width;
    col = strip * 4 + rest % width;
    return true;
}

// 16-byte pieces in LDS: piece o of row r of an array with 2^LOG pieces a row stands at o ^ (r divided by the rows that make 256 bytes), so
// that lanes that read the same piece of 16 consecutive rows hit all banks.
template <int LOG>
__device__ __forceinline__ int lds_piece(int r, int o) {
    return (r << LOG) + (o ^ ((r >> (LOG < 4 ? 4 - LOG : 0)) & ((1 << LOG) - 1)));
}

// The same for arrays that are read transposed, four rows by 64 bytes at a time: the four rows' pieces hit all banks.
__device__ __forceinline__ int lds_piece_tr(int log, int r, int o) { return (r << log) + (o ^ ((r & 3) << 2)); }

__device__ __forceinline__ bf16x8 as_operand(uint4 v) { return __builtin_bit_cast(bf16x8, v); }

// ---- straight from memory into LDS -------------------------------------------------------------------------------------------------

// Loads go through a buffer descriptor: the lane's part of an address is a 32-bit offset that stays, what moves is a scalar, and what lies
// beyond the end arrives as 0.  Offsets are below 2^31 (the launch sees to it).
struct Buffer {
    const void* start;
    int bytes;
    __device__ __forceinline__ void set(const void* p, int64_t length) {
        start = p;
        bytes = int(length < 0x7FFFFFFF ? length : 0x7FFFFFFF);
    }
    // 16 bytes a lane from lane offset `off` + `at` to lane * 16 bytes behind `to`, which is the same in all lanes.  The
    // descriptor's type exists in device code only.
    __device__ __forceinline__ void to_lds16(uint32_t off, int at, void* to) const {
#ifdef __HIP_DEVICE_COMPILE__
        __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(start), 0, bytes, 0x00020000),
                                                 (__attribute__((address_space(3))) void*)(to), 16, off, at, 0, 0);
#endif
    }
};

// ROWS rows of 2^LOG octets of bf16 (16 bytes), staged by WAVES waves a KiB at a time.  A lane's octet of a row is the one that lds_piece
// puts at the lane's place, so the swizzle costs nothing.
template <int ROWS, int LOG, int WAVES, bool TR = false>
struct StageDirect {
    static constexpr int kPieces = ROWS << LOG, kOwn = kPieces / 64 / WAVES, kRowsAtOnce = 64 >> LOG;
    static_assert(kPieces % (64 * WAVES) == 0, "whole KiB per wave");
    Buffer buffer;
    uint32_t off[kOwn], col[kOwn];                             // bytes
    // stride: bytes from one row to the next; rows: of the matrix from `first` on; those beyond arrive as 0
    // wave: of the WAVES
    __device__ __forceinline__ void setup(const void* first, int64_t stride, int64_t rows, int wave) {
        const int lane = threadIdx.x & 63;
        buffer.set(first, rows < ROWS ? rows * stride : ROWS * stride);
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            const int r = (j * WAVES + wave) * kRowsAtOnce + (lane >> LOG);
            const int o = lane & ((1 << LOG) - 1);
            col[j] = ((TR ? lds_piece_tr(LOG, r, o) : lds_piece<LOG>(r, o)) - (r << LOG)) * 16;                                    // involutions
            off[j] = uint32_t(r) * uint32_t(stride) + col[j];
        }
    }
    // at: bytes from a row's start
    __device__ __forceinline__ void load(int at, uint4* lds, int wave) const {
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
            buffer.to_lds16(off[j], at, lds + (j * WAVES + wave) * 64);
    }
    // the same for rows of `end` bytes: octets beyond arrive as 0
    __device__ __forceinline__ void load_cut(int at, int end, uint4* lds, int wave) const {
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
            buffer.to_lds16(int(col[j]) < end - at ? off[j] : 0x80000000u, at, lds + (j * WAVES + wave) * 64);
    }
};

// 0 in registers that the compiler does not know to be 0: the C operand of a sum's first product, which saves clearing the sum
__device__ __forceinline__ f32x16 opaque_zero() {
    f32x16 z = {};
    asm volatile("" : "+v"(z));
    return z;
}

}  // namespace lpmm
