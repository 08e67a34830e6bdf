// What the library's two translation units share on the host side: HIP errors and pointer checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/lpmm4.h"

namespace lpmm {

extern thread_local int g_last_hip __attribute__((visibility("hidden")));     // what lpmm_last_hip_error returns; defined in lpmm4.hip

inline int hip_fail(hipError_t e) { g_last_hip = int(e); return LPMM_EHIP; }
#define LPMM_HIP(call) do { hipError_t e_ = (call); if (e_ != hipSuccess) return hip_fail(e_); } while (0)

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace lpmm
