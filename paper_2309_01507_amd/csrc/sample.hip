// C ABI of sampling (declared in include/lpmm4.h): argument checks and launches.  The arithmetic is in sample.hpp.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "host_util.hpp"
#include "sample.hpp"

namespace {

using namespace lpmm;

// Workgroups of a row; 1: one does it all.  Sharing costs two launches and the handing over, and takes from the readings of a row.  One workgroup against several, us, bf16, with top_p
// 0.95, and with top_k 50 and top_p 0.9: 1 x 18000 23 and 25, 17 and 24; 1 x 32000 29 and 25, 20 and 24; 1 x 50257 38 and 26, 24 and 24; 1 x 131072 74 and 33, 43 and 27; 16 x 32000
// 30 and 28, 21 and 26; 16 x 50257 40 and 31, 26 and 29; 64 x 50257 45 and 43, 26 and 36; 64 x 131072 80 and 64, 44 and 46; 128 x 131072 81 and 95 (there the workgroups of a row wait for CUs).
// 512 for all rows together: with 256 16 to 64 rows take up to a fourth longer, with 1024 64 x 32000 takes a sixth longer.
int sample_shares(int64_t t, int64_t v) {
    if (t < 1 || t > 64 || v < 24576 + 512 * t || v > int64_t(kSampleBins) * 256) return 1;
    return int(std::min<int64_t>(std::min<int64_t>(kSampleShares, 512 / t), div_up(v, 2048)));
}

}  // namespace

extern "C" {

size_t lpmm_sample_workspace_bytes(int64_t t, int64_t v) {
    return t < 1 || t > kMaxTokens || v < 1 || v > kMaxDim || sample_shares(t, v) == 1 ? 0 : size_t(t) * sizeof(SampleWork);
}

int lpmm_sample(const void* z, int z_dtype, int64_t t, int64_t v, int64_t z_stride, const float* u, const lpmm_sample_options* options,
                int64_t* tokens, float* logprob, void* workspace, size_t workspace_bytes, void* stream) {
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
    LPMM_TRY(check_workspace(workspace, workspace_bytes, lpmm_sample_workspace_bytes(t, v)));
    const int shares = sample_shares(t, v);
    if (shares > 1) {
        const int64_t lines = div_up(v, z_dtype == LPMM_BF16 ? 512 : 256);
        const int per = int(div_up(lines, shares));
        const dim3 grid(unsigned(div_up(lines, per)), unsigned(t)), threads(kSampleShareThreads);
        SampleWork* work = static_cast<SampleWork*>(workspace);
#define LPMM_SHARE(K) { if (z_dtype == LPMM_BF16) hipLaunchKernelGGL(K<true>, grid, threads, 0, s, a, work, per); \
                        else hipLaunchKernelGGL(K<false>, grid, threads, 0, s, a, work, per); LPMM_HIP(hipGetLastError()); }
        LPMM_SHARE(sample_largest_kernel)
        LPMM_SHARE(sample_bins_kernel)
        LPMM_SHARE(sample_finish_kernel)
#undef LPMM_SHARE
        return LPMM_OK;
    }
    const dim3 rows{unsigned(t)};
    // Threads of a row: as many as speed up its passes, as few as leave room for other rows (us with 256, 512, 1024, bf16 with top_p: 1 x 1000 13.0, 14.1, 16.5;
    // 1 x 16000 27, 22, 22; 256 x 32000 43, 34, 32; 128 x 131072 126, 89, 81; 300 x 32000 52, 45, 58; 768 x 32000 69, 64, 92; 2048 x 32000 150, 147, 184;
    // 2000 x 16000 84, 91, 165; 2000 x 4000 39, 51, 117; with top_k too 256 x 32000 32, 22, 22; 300 x 32000 39, 30, 39; 2000 x 4000 33, 37, 92)
#define LPMM_SAMPLE(T) { if (z_dtype == LPMM_BF16) hipLaunchKernelGGL((sample_kernel<true, T>), rows, dim3(T), 0, s, a); \
                         else hipLaunchKernelGGL((sample_kernel<false, T>), rows, dim3(T), 0, s, a); }
    if (v <= 2048 || (t > 1024 && v <= 16384)) LPMM_SAMPLE(256)
    else if (t > 256 || v <= 16384) LPMM_SAMPLE(512)
    else LPMM_SAMPLE(1024)
#undef LPMM_SAMPLE
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

}  // extern "C"
