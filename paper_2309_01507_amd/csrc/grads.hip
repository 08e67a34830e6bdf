// C ABI of the gradients' norm and of clipping (declared in include/lpmm4.h): checks, the plan's tables, launches.  The arithmetic
// is in grads.hpp.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "host_util.hpp"
#include "grads.hpp"

namespace {

using namespace lpmm;

constexpr int64_t kMaxGradTensors = int64_t(1) << 24, kMaxNumel = int64_t(1) << 40, kMaxChunks = (int64_t(1) << 31) - 1;

// Chunks of 64 KiB; of fewer bytes where these would be fewer than the workgroups that the GPU holds at once
int chunk_log(int64_t bytes) {
    int log = 16;
    while (log > 12 && (bytes >> log) < 1024) --log;
    return log;
}

struct Layout {
    int log_bytes;
    int64_t tensors, chunks;
    size_t bytes;
};

int64_t pieces_of(const lpmm_grad_desc& d, int64_t lead) { return ((lead + d.numel) * elem_size(d.dtype) + 15) / 16; }

// The tables' sizes; chunks for the worst alignment, so that they do not depend on addresses
int layout(const lpmm_grad_desc* descs, int64_t n, Layout* l) {
    if (n < 0 || n > kMaxGradTensors || (n > 0 && !descs)) return LPMM_EINVAL;
    int64_t bytes = 0;
    for (int64_t i = 0; i < n; ++i) {
        const lpmm_grad_desc& d = descs[i];
        if ((d.dtype != LPMM_F32 && d.dtype != LPMM_BF16) || d.reserved != 0 || d.numel < 0 || d.numel > kMaxNumel) return LPMM_EINVAL;
        bytes += d.numel * elem_size(d.dtype);
        if (bytes > (int64_t(1) << 46)) return LPMM_EINVAL;
    }
    l->log_bytes = chunk_log(bytes);
    l->tensors = n;
    l->chunks = 0;
    for (int64_t i = 0; i < n; ++i)
        if (descs[i].numel) l->chunks += div_up(pieces_of(descs[i], 16 / elem_size(descs[i].dtype) - 1) * 16, int64_t(1) << l->log_bytes);
    if (l->chunks > kMaxChunks) return LPMM_EINVAL;
    l->bytes = sizeof(GradHead) + size_t(n) * sizeof(GradTensor) + size_t(l->chunks) * sizeof(GradChunk);
    return LPMM_OK;
}

struct Range {
    uintptr_t from, to;
    bool written;
};

// No element is written twice, or written as one tensor's and read as another's
bool apart(std::vector<Range>& ranges) {
    std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t read = 0, written = 0;                 // ends so far
    for (const Range& r : ranges) {
        if (r.from < written || (r.written && r.from < read)) return false;
        (r.written ? written : read) = std::max(r.written ? written : read, r.to);
    }
    return true;
}

int check_plan(const lpmm_grad_plan* plan, GradPlan* p) {
    if (!plan || !plan->device || !aligned(plan->device, 256) || plan->tensors < 0 || plan->chunks < 0 || plan->chunks > kMaxChunks ||
        plan->log_bytes < 12 || plan->log_bytes > 16)
        return LPMM_EINVAL;
    char* at = static_cast<char*>(plan->device);
    p->head = reinterpret_cast<GradHead*>(at);
    p->tensors = reinterpret_cast<const GradTensor*>(at + sizeof(GradHead));
    p->chunks = reinterpret_cast<const GradChunk*>(at + sizeof(GradHead) + size_t(plan->tensors) * sizeof(GradTensor));
    p->count = plan->chunks;
    p->log_bytes = plan->log_bytes;
    return LPMM_OK;
}

// Workgroups: more of them read faster and take longer over their tickets (us with 256, 512, 768 for the norm of 1M fp32 elements 9.8, 11.9, 15.0; 3M 11.5, 12.8, 15.4;
// 25M 28, 24, 26; 355M 437, 258, 226; 3G bf16 2000, 1262, 982)
int launch_norm(const GradPlan& p, int kind, float* norm, hipStream_t s) {
    const int64_t bytes = p.count << p.log_bytes, most = bytes < int64_t(16) << 20 ? 256 : bytes < int64_t(256) << 20 ? 512 : kGradBlocks;
    const dim3 grid(unsigned(std::max<int64_t>(1, std::min(p.count, most))));
    if (kind == LPMM_GRAD_NORM_MAX) hipLaunchKernelGGL(grad_norm_kernel<true>, grid, dim3(kGradThreads), 0, s, p, norm);
    else hipLaunchKernelGGL(grad_norm_kernel<false>, grid, dim3(kGradThreads), 0, s, p, norm);
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

int check_norm(int kind, const float* norm) {
    return (kind == LPMM_GRAD_NORM_L2 || kind == LPMM_GRAD_NORM_MAX) && !check_floats(norm) ? LPMM_OK : LPMM_EINVAL;
}

int check_clip(const lpmm_grad_plan* plan, const float* norm, float limit) {
    return plan->writes && !check_floats(norm) && limit >= 0.0f ? LPMM_OK : LPMM_EINVAL;
}

int launch_clip(const GradPlan& p, const float* norm, float limit, hipStream_t s) {
    if (p.count == 0) return LPMM_OK;
    // us with 256, 512, 768: 3M fp32 elements 11.8, 8.9, 8.7; 355M 440, 522, 540 behind a norm that took 437, 258, 226; 3G bf16 2380, 2254, 2330
    const dim3 grid(unsigned(std::min<int64_t>(p.count, 512)));
    hipLaunchKernelGGL(grad_clip_kernel, grid, dim3(kGradThreads), 0, s, p, norm, limit);
    LPMM_HIP(hipGetLastError());
    return LPMM_OK;
}

}  // namespace

extern "C" {

size_t lpmm_grad_plan_bytes(const lpmm_grad_desc* descs, int64_t n) {
    Layout l{};
    return layout(descs, n, &l) ? 0 : l.bytes;
}

int lpmm_grad_plan_build(const lpmm_grad_desc* descs, int64_t n, void* device, size_t bytes, void* stream, lpmm_grad_plan* plan) {
    Layout l{};
    if (!plan) return LPMM_EINVAL;
    LPMM_TRY(layout(descs, n, &l));
    if (!device || !aligned(device, 256)) return LPMM_EINVAL;
    if (bytes < l.bytes) return LPMM_EWORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
    LPMM_HIP(hipStreamIsCapturing(s, &capturing));
    if (capturing != hipStreamCaptureStatusNone) return LPMM_EINVAL;
    try {
        std::vector<char> host(l.bytes, 0);
        GradTensor* tensors = reinterpret_cast<GradTensor*>(host.data() + sizeof(GradHead));
        GradChunk* chunks = reinterpret_cast<GradChunk*>(tensors + n);
        std::vector<Range> ranges;
        int64_t count = 0;
        bool writes = true;
        for (int64_t i = 0; i < n; ++i) {
            const lpmm_grad_desc& d = descs[i];
            const int e = elem_size(d.dtype);
            tensors[i] = GradTensor{d.grad, d.out, d.numel, d.dtype == LPMM_BF16};
            if (d.numel == 0) continue;
            if (!d.grad || !aligned(d.grad, e) || !aligned(d.out, e)) return LPMM_EINVAL;
            const uintptr_t g = reinterpret_cast<uintptr_t>(d.grad), o = reinterpret_cast<uintptr_t>(d.out);
            if (d.out != d.grad) ranges.push_back(Range{g, g + uintptr_t(d.numel) * e, false});
            if (d.out) ranges.push_back(Range{o, o + uintptr_t(d.numel) * e, true});
            writes = writes && d.out;
            const int64_t own = div_up(pieces_of(d, int64_t(g & 15) / e) * 16, int64_t(1) << l.log_bytes);
            for (int64_t c = 0; c < own; ++c) chunks[count++] = GradChunk{int32_t(i), int32_t(c)};
        }
        if (!apart(ranges)) return LPMM_EINVAL;
        LPMM_HIP(hipMemcpyAsync(device, host.data(), l.bytes, hipMemcpyHostToDevice, s));
        LPMM_HIP(hipStreamSynchronize(s));                     // the tables above end here
        *plan = lpmm_grad_plan{device, n, count, l.log_bytes, writes};
    } catch (const std::bad_alloc&) {
        return LPMM_EWORKSPACE;
    }
    return LPMM_OK;
}

int lpmm_grad_norm(const lpmm_grad_plan* plan, int kind, float* norm, void* stream) {
    GradPlan p{};
    LPMM_TRY(check_plan(plan, &p));
    LPMM_TRY(check_norm(kind, norm));
    return launch_norm(p, kind, norm, static_cast<hipStream_t>(stream));
}

int lpmm_grad_clip(const lpmm_grad_plan* plan, const float* norm, float limit, void* stream) {
    GradPlan p{};
    LPMM_TRY(check_plan(plan, &p));
    LPMM_TRY(check_clip(plan, norm, limit));
    return launch_clip(p, norm, limit, static_cast<hipStream_t>(stream));
}

int lpmm_grad_norm_clip(const lpmm_grad_plan* plan, int kind, float limit, float* norm, void* stream) {
    GradPlan p{};
    LPMM_TRY(check_plan(plan, &p));
    LPMM_TRY(check_norm(kind, norm));
    LPMM_TRY(check_clip(plan, norm, limit));
    LPMM_TRY(launch_norm(p, kind, norm, static_cast<hipStream_t>(stream)));
    return launch_clip(p, norm, limit, static_cast<hipStream_t>(stream));
}

}  // extern "C"
