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
    if (z_dtype == LPMM_BF16) hipLaunchKernelGGL((sample_kernel<true, 256>), rows, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((sample_kernel<false, 256>), rows, dim3(256), 0, s, a);
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}
