// The norm of many gradients as one vector, and their scaling to a limit (formulas: include/lpmm4.h).
//
// A plan cuts every tensor into chunks that begin on 16-byte boundaries; a launch's workgroups walk over the chunks of all tensors.
// Squares are added up in 64 bits: they do not overflow, and beside the loads the wider additions cost nothing.
#pragma once

#include "rows.hpp"

namespace lpmm {

constexpr int kGradThreads = 256, kGradBlocks = 768;       // workgroups of a launch at most: 3 a CU

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

// The 16-byte pieces of a chunk, counted from the boundary at or before the tensor's start: those from `in0` to `in1` lie within the tensor, and there may be one in front
// of them and one behind that lie there in part.
struct GradSpan {
    const char* base;                    // that boundary
    int64_t piece0, in0, in1, piece1;
    int64_t lead;                        // elements between the boundary and the tensor's start
};
template <bool BF16>
__device__ __forceinline__ GradSpan grad_span(const GradTensor& t, int number, int log_bytes) {
    constexpr int N = BF16 ? 8 : 4, E = BF16 ? 2 : 4;
    GradSpan s;
    const uintptr_t at = reinterpret_cast<uintptr_t>(t.grad);
    s.base = reinterpret_cast<const char*>(at & ~uintptr_t(15));
    s.lead = int64_t(at & 15) / E;
    const int64_t end = s.lead + t.numel;
    s.piece0 = int64_t(number) << (log_bytes - 4);
    s.piece1 = min((end + N - 1) / N, s.piece0 + (int64_t(1) << (log_bytes - 4)));
    s.in1 = min(end / N, s.piece1);
    s.in0 = s.piece0 + (s.piece0 == 0 && s.lead > 0);
    if (s.in1 < s.in0) s.in0 = s.in1 = min(s.in0, s.piece1);             // a piece or two, none of them within
    return s;
}

// whole(piece, its 16 bytes), kGradAhead pieces of a thread on their way at once; edge(piece) for those that are not within
constexpr int kGradAhead = 4;
template <typename Whole, typename Edge>
__device__ __forceinline__ void grad_pieces(const GradSpan& s, Whole&& whole, Edge&& edge) {
    for (int64_t p = s.in0 + threadIdx.x; p < s.in1; p += kGradAhead * kGradThreads) {
        uint4 q[kGradAhead];
#pragma unroll
        for (int j = 0; j < kGradAhead; ++j) q[j] = *reinterpret_cast<const uint4*>(s.base + (min(p + j * kGradThreads, s.in1 - 1) << 4));
#pragma unroll
        for (int j = 0; j < kGradAhead; ++j)
            if (p + j * kGradThreads < s.in1) whole(p + j * kGradThreads, q[j]);
    }
    if (threadIdx.x == 0 && s.piece0 < s.in0) edge(s.piece0);
    if (threadIdx.x == 64 && s.in1 < s.piece1) edge(s.in1);
}
template <bool BF16>
__device__ __forceinline__ void grad_floats(const uint4& q, float x[8]) {
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
    grad_pieces(s, [&](int64_t, const uint4& q) {
        float x[8];
        grad_floats<BF16>(q, x);
#pragma unroll
        for (int e = 0; e < N; ++e) grad_take<MOST>(sum, most, x[e]);
    }, [&](int64_t p) {
        const int64_t i0 = p * N - s.lead;
        for (int e = 0; e < N; ++e)
            if (i0 + e >= 0 && i0 + e < t.numel) grad_take<MOST>(sum, most, w4_load1<BF16>(t.grad, i0 + e));
    });
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

// The last workgroup to finish joins what all have found, in the order of their numbers: equal inputs give equal bits.  Parts and ticket go
// past the L2 caches of the XCDs (agent scope), and a workgroup waits for its part to arrive before it takes its ticket: a release would write back an L2 for each workgroup.
// Bound by memory: 6.7G bf16 (13.5 GB) 2110 us, 355M fp32 (1.4 GB) 227 us, 6.3 TB/s; 1M fp32 10 us, a round trip to memory for each of four steps and the tickets, which one address
// takes one after another (2048 workgroups: 25M fp32 35 us, 768 26, 512 24).
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
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");           // for the compiler's order
        __builtin_amdgcn_s_waitcnt(0x0070);                              // the part has arrived behind L2
        s_last = __hip_atomic_fetch_add(&plan.head->ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
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
    grad_pieces(s, [&](int64_t p, const uint4& q) {
        float x[8];
        grad_floats<BF16>(q, x);
        char* out = static_cast<char*>(t.out) + (p * N - s.lead) * E;
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
    }, [&](int64_t p) {
        const int64_t i0 = p * N - s.lead;
        for (int e = 0; e < N; ++e)
            if (i0 + e >= 0 && i0 + e < t.numel) w4_store1<BF16>(t.out, i0 + e, w4_load1<BF16>(t.grad, i0 + e) * part);
    });
}

// Chunks from the last to the first: what the norm has read last is still in the cache.  Bound by memory: 355M fp32 522 us, 5.4 TB/s read and written; stores past the
// caches took as long.
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
