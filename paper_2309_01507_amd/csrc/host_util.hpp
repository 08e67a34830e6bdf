// What the library's translation units share on the host side: HIP errors, limits and checks of arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/lpmm4.h"

namespace lpmm {

extern thread_local int g_last_hip __attribute__((visibility("hidden")));     // what lpmm_last_hip_error returns; defined in lpmm4.hip

inline int hip_fail(hipError_t e) { g_last_hip = int(e); return LPMM_EHIP; }
#define LPMM_HIP(call) do { hipError_t e_ = (call); if (e_ != hipSuccess) return hip_fail(e_); } while (0)

#define LPMM_TRY(call) do { const int rc_ = (call); if (rc_) return rc_; } while (0)

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMaxDim = int64_t(1) << 30;
// A launch has fewer than 2^32 threads
constexpr int64_t kMaxTokens = (int64_t(1) << 24) - 1, kMaxBlocks = (int64_t(1) << 23) - 1;

inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int elem_size(int dtype) { return dtype == LPMM_BF16 ? 2 : 4; }

// `rows` rows of `len` elements, `stride` apart
inline int check_rows(const void* p, int dtype, int64_t rows, int64_t len, int64_t stride) {
    if (dtype != LPMM_F32 && dtype != LPMM_BF16) return LPMM_EINVAL;
    if (rows < 0 || rows > kMaxDim || stride < len || stride > (int64_t(1) << 40)) return LPMM_EINVAL;
    if (rows > 0 && (!p || !aligned(p, elem_size(dtype)))) return LPMM_EINVAL;
    return LPMM_OK;
}

inline int check_codes(const uint8_t* codes) { return codes && aligned(codes, 16) ? LPMM_OK : LPMM_EINVAL; }
inline int check_floats(const float* p) { return p && aligned(p, 4) ? LPMM_OK : LPMM_EINVAL; }

inline int check_workspace(const void* p, size_t have, size_t need) {
    if (need == 0) return LPMM_OK;
    if (!p || !aligned(p, 16)) return LPMM_EINVAL;
    return have < need ? LPMM_EWORKSPACE : LPMM_OK;
}

}  // namespace lpmm
