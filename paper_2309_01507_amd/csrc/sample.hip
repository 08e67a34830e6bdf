// C ABI of sampling (declared in include/lpmm4.h): argument checks and launches.  The arithmetic is in sample.hpp.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "host_util.hpp"
#include "sample.hpp"

using namespace lpmm;

extern "C" int lpmm_sample(const void* z, int z_dtype, int64_t t, int64_t v, int64_t z_stride, const float* u, const lpmm_sample_options* options,
                           int64_t* tokens, float* logprob, void* stream) {
    if (!options || t > kMaxTokens || v < 1 || v > kMaxDim) return LPMM_EINVAL;
    LPMM_TRY(check_rows(z, z_dtype, t, v, z_stride));
    const lpmm_sample_options& o = *options;
    if (!(o.temperature >= 0.0f) || o.top_k < 0 || !(o.top_p == o.top_p) || !(o.min_p == o.min_p)) return LPMM_EINVAL;
    if (!aligned(o.temperatures, 4) || !aligned(o.top_ks, 4) || !aligned(o.top_ps, 4) || !aligned(o.min_ps, 4)) return LPMM_EINVAL;
    if (t == 0) return LPMM_OK;
    LPMM_TRY(check_floats(u));
    LPMM_TRY(check_floats(logprob));
    if (!tokens || !aligned(tokens, 8)) return LPMM_EINVAL;
    SampleArgs a{};
    a.z = z;
    a.z_stride = z_stride;
    a.v = int(v);
    a.bits = 46;
    while (a.bits > 32 && (v >> (62 - a.bits)) > 0) --a.bits;             // v weights of 1 add up to less than 2^63
    a.temperature = o.temperature;
    a.top_p = o.top_p;
    a.min_p = o.min_p;
    a.top_k = o.top_k;
    a.temperatures = o.temperatures;
    a.top_ks = o.top_ks;
    a.top_ps = o.top_ps;
    a.min_ps = o.min_ps;
    a.u = u;
    a.tokens = tokens;
    a.logprob = logprob;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 rows{unsigned(t)};
    // Threads of a row: as many as speed up its passes, as few as leave room for other rows (us with 256, 512, 1024: 1 x 1000 12.8, 13.1, 15.4; 1 x 4000 15.4, 13.9, 16.4;
    // 1 x 16000 32, 25, 25; 256 x 32000 66, 46, 42; 300 x 32000 80, 63, 72; 768 x 32000 97, 83, 110; 2048 x 32000 215, 211, 294; 2000 x 16000 105, 111, 185;
    // 2000 x 4000 43, 54, 111)
#define LPMM_SAMPLE(T) { if (z_dtype == LPMM_BF16) hipLaunchKernelGGL((sample_kernel<true, T>), rows, dim3(T), 0, s, a); \
                         else hipLaunchKernelGGL((sample_kernel<false, T>), rows, dim3(T), 0, s, a); }
    if (v <= 2048 || (t > 1024 && v <= 16384)) LPMM_SAMPLE(256)
    else if (t > 256 || v <= 16384) LPMM_SAMPLE(512)
    else LPMM_SAMPLE(1024)
#undef LPMM_SAMPLE
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}
