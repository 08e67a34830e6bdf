// The norm of many gradients as one vector, and their scaling to a limit (formulas: include/lpmm4.h).
//
// A plan cuts every tensor into chunks that begin on 16-byte boundaries; a launch's workgroups walk over the chunks of all tensors.
// Squares are added up in 64 bits: they do not overflow, and beside the loads the wider additions cost nothing.
#pragma once

#include "rows.hpp"

namespace lpmm {

constexpr int kGradThreads = 256, kGradBlocks = 2048;      // workgroups of a launch at most: 8 a CU

struct GradTensor {
    const void* grad;
    void* out;
    int64_t numel;
    int64_t bf16;
};
struct GradChunk {
    int32_t tensor, number;              // chunk `number` of the tensor
};
// Device memory of a plan: this, then the tensors, then the chunks
struct GradHead {
    double parts[kGradBlocks];           // of the workgroups: sum of squares, or the largest magnitude
    uint32_t ticket;                     // workgroups that are done; 0 between launches
    uint32_t pad[63];
};
struct GradPlan {
    GradHead* head;
    const GradTensor* tensors;
    const GradChunk* chunks;
    int64_t count;                       // chunks
    int32_t log_bytes;                   // of a chunk
};

// The 16-byte pieces of a chunk, counted from the boundary at or before the tensor's start
struct GradSpan {
    const char* base;                    // that boundary
    int64_t piece0, piece1;
    int64_t lead;                        // elements between the boundary and the tensor's start
};
template <bool BF16>
__device__ __forceinline__ GradSpan grad_span(const GradTensor& t, int number, int log_bytes) {
    constexpr int E = BF16 ? 2 : 4;
    GradSpan s;
    const uintptr_t at = reinterpret_cast<uintptr_t>(t.grad);
    s.base = reinterpret_cast<const char*>(at & ~uintptr_t(15));
    s.lead = int64_t(at & 15) / E;
    const int64_t pieces = ((s.lead + t.numel) * E + 15) >> 4;
    s.piece0 = int64_t(number) << (log_bytes - 4);
    s.piece1 = min(pieces, s.piece0 + (int64_t(1) << (log_bytes - 4)));
    return s;
}

// Floats of a 16-byte piece; `i0`: the tensor's element that its first one is (negative in front of the tensor).  What lies outside is
// 0 and not read.
template <bool BF16>
__device__ __forceinline__ void grad_piece(const char* base, int64_t piece, int64_t i0, int64_t numel, float x[8]) {
    constexpr int N = BF16 ? 8 : 4;
    const char* at = base + (piece << 4);
    if (i0 >= 0 && i0 + N <= numel) {
        const uint4 q = *reinterpret_cast<const uint4*>(at);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (BF16) {
                x[2 * e] = __uint_as_float(w[e] << 16);
                x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
            } else {
                x[e] = __uint_as_float(w[e]);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = i0 + e >= 0 && i0 + e < numel ? w4_load1<BF16>(at, e) : 0.0f;
    }
}

template <bool MOST>
__device__ __forceinline__ void grad_take(double& sum, uint32_t& most, float x) {
    if constexpr (MOST) {
        const uint32_t a = __float_as_uint(x) & 0x7FFFFFFFu;             // magnitudes order like their bits, NaN above all
        most = a > most ? a : most;
    } else {
        sum = __builtin_fma(double(x), double(x), sum);
    }
}

template <bool BF16, bool MOST>
__device__ __forceinline__ void grad_chunk(const GradTensor& t, int number, int log_bytes, double& sum, uint32_t& most) {
    constexpr int N = BF16 ? 8 : 4;
    const GradSpan s = grad_span<BF16>(t, number, log_bytes);
    for (int64_t p = s.piece0 + threadIdx.x; p < s.piece1; p += kGradThreads) {
        float x[8];
        grad_piece<BF16>(s.base, p, p * N - s.lead, t.numel, x);
#pragma unroll
        for (int e = 0; e < N; ++e) grad_take<MOST>(sum, most, x[e]);
    }
}

// Value of the lane `mask` away
__device__ __forceinline__ double lane_xor(double x, int mask) { return __shfl_xor(x, mask, 64); }

// The workgroup's sum (or maximum) in thread 0, in a fixed order
template <bool MOST>
__device__ __forceinline__ double grad_join(double x, double* lds) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const double y = lane_xor(x, m);
        x = MOST ? fmax(x, y) : x + y;
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < kGradThreads / 64; ++w) x = MOST ? fmax(x, lds[w]) : x + lds[w];
    __syncthreads();
    return x;
}

// The last workgroup to finish joins what all have found, in the order of their numbers: equal inputs give equal bits.  The parts go
// past the L2 caches of the XCDs (agent scope), the ticket orders them.
template <bool MOST>
__global__ __launch_bounds__(kGradThreads) void grad_norm_kernel(GradPlan plan, float* norm) {
    __shared__ double s_join[kGradThreads / 64];
    __shared__ bool s_last;
    double sum = 0.0;
    uint32_t most = 0;
    for (int64_t c = blockIdx.x; c < plan.count; c += gridDim.x) {
        const GradChunk chunk = plan.chunks[c];
        const GradTensor t = plan.tensors[chunk.tensor];
        if (t.bf16) grad_chunk<true, MOST>(t, chunk.number, plan.log_bytes, sum, most);
        else grad_chunk<false, MOST>(t, chunk.number, plan.log_bytes, sum, most);
    }
    // magnitudes' bits as doubles: exact, and NaN, whose bits are the largest, is an ordinary number until the end
    const double mine = grad_join<MOST>(MOST ? double(most) : sum, s_join);
    if (threadIdx.x == 0) {
        __hip_atomic_store(&plan.head->parts[blockIdx.x], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = __hip_atomic_fetch_add(&plan.head->ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    __syncthreads();
    if (!s_last) return;
    double all = 0.0;
    for (int b = threadIdx.x; b < int(gridDim.x); b += kGradThreads) {
        const double part = __hip_atomic_load(&plan.head->parts[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        all = MOST ? fmax(all, part) : all + part;
    }
    all = grad_join<MOST>(all, s_join);
    if (threadIdx.x == 0) {
        norm[0] = MOST ? __uint_as_float(uint32_t(all)) : float(sqrt(all));
        __hip_atomic_store(&plan.head->ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

template <bool BF16>
__device__ __forceinline__ void grad_scale_chunk(const GradTensor& t, int number, int log_bytes, float part) {
    constexpr int N = BF16 ? 8 : 4, E = BF16 ? 2 : 4;
    const GradSpan s = grad_span<BF16>(t, number, log_bytes);
    for (int64_t p = s.piece0 + threadIdx.x; p < s.piece1; p += kGradThreads) {
        const int64_t i0 = p * N - s.lead;
        float x[8];
        grad_piece<BF16>(s.base, p, i0, t.numel, x);
        char* out = static_cast<char*>(t.out) + i0 * E;
        if (i0 >= 0 && i0 + N <= t.numel) {
            if constexpr (BF16) {
                Vec16 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v.v[e] = uint32_t(to_bf16(x[2 * e] * part)) | uint32_t(to_bf16(x[2 * e + 1] * part)) << 16;
                *reinterpret_cast<Vec16*>(out) = v;
            } else {
                Vec16f v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v.v[e] = x[e] * part;
                *reinterpret_cast<Vec16f*>(out) = v;
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (i0 + e >= 0 && i0 + e < t.numel) w4_store1<BF16>(out, e, x[e] * part);
        }
    }
}

// Chunks from the last to the first: what the norm has read last is still in the cache.
__global__ __launch_bounds__(kGradThreads) void grad_clip_kernel(GradPlan plan, const float* norm, float limit) {
    const float part = float(double(limit) / (double(norm[0]) + 1e-6));
    const bool whole = part >= 1.0f || limit == __builtin_inff();        // NaN is not
    for (int64_t i = blockIdx.x; i < plan.count; i += gridDim.x) {
        const GradChunk chunk = plan.chunks[plan.count - 1 - i];
        const GradTensor t = plan.tensors[chunk.tensor];
        if (whole && t.out == t.grad) continue;
        if (t.bf16) grad_scale_chunk<true>(t, chunk.number, plan.log_bytes, whole ? 1.0f : part);
        else grad_scale_chunk<false>(t, chunk.number, plan.log_bytes, whole ? 1.0f : part);
    }
}

}  // namespace lpmm
