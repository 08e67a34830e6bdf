// Distillation from a teacher's top logits: loss and gradient (formulas: include/lpmm4.h).
//
// One pass over a row of logits keeps a running maximum m and the sum l of exp(z / tau - m), both in fp32 per lane, and joins the
// lanes' pairs at the end; the gradient is exp(z / tau - lse) times a factor everywhere but at the teacher's slots, which
// are written once more behind a barrier.  Bound by reading and writing the logits.
#pragma once

#include "w4.hpp"

namespace lpmm {

constexpr int kDistillSlots = 1024;      // most slots of a row
constexpr float kLog2e = 1.44269504088896340736f;

struct DistillArgs {
    const void* z;
    int64_t z_stride;
    int64_t t;
    int v, slots;
    const float* top;
    const int64_t* index;
    float tau, inv_tau;
    const float* grad;
    float* loss;
    float* lse;
    void* dz;
    int64_t dz_stride;
};

// The teacher's side of a row, in LDS: places (-1 where a slot does not count) and probabilities
struct DistillSlots {
    int at[kDistillSlots];
    float p[kDistillSlots];
};

__device__ __forceinline__ float exp_nat(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// (m, l) of two disjoint sets.  m starts at -FLT_MAX rather than -infinity, so that no difference is infinity - infinity
// as long as the logits hold no +infinity.
__device__ __forceinline__ void join_ml(float& m, float& l, float m2, float l2) {
    const float top = fmaxf(m, m2);
    l = l * exp_nat(m - top) + l2 * exp_nat(m2 - top);
    m = top;
}
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

// One wave reads a row's slots: s.at and s.p of the row, and log p = u - log_total with u = top / tau - top_max in each lane's own
// loop below.  Returns whether any slot counts.
__device__ __forceinline__ bool distill_teacher(const DistillArgs& a, int64_t row, DistillSlots& s, float& u_max,
                                                float& log_total) {
    const int lane = threadIdx.x & 63;
    const float* top = a.top + row * a.slots;
    const int64_t* index = a.index + row * a.slots;
    float m = -__builtin_inff();
    bool any = false;
    for (int j = lane; j < a.slots; j += 64) {
        const int64_t i = index[j];
        const bool ok = i >= 0 && i < a.v;
        const float u = top[j] * a.inv_tau;
        s.at[j] = ok ? int(i) : -1;
        s.p[j] = u;
        if (ok) m = fmaxf(m, u);
        any = any || ok;
    }
    any = __ballot(any) != 0;
    u_max = wave_max(m);
    float sum = 0.0f;
    for (int j = lane; j < a.slots; j += 64) {
        const float e = s.at[j] >= 0 ? exp_nat(s.p[j] - u_max) : 0.0f;
        s.p[j] = e;
        sum += e;
    }
    sum = wave_sum(sum);
    const float inv = 1.0f / sum;
    for (int j = lane; j < a.slots; j += 64) s.p[j] *= inv;
    log_total = logf(sum);
    return any;
}

// One wave: the row's loss from its lse
template <bool BF16>
__device__ __forceinline__ float distill_row_loss(const DistillArgs& a, int64_t row, const DistillSlots& s, float u_max,
                                                  float log_total, float lse) {
    float sum = 0.0f;
    for (int j = threadIdx.x & 63; j < a.slots; j += 64) {
        const int at = s.at[j];
        const float p = s.p[j];
        if (at >= 0 && p != 0.0f) {
            const float log_p = (a.top[row * a.slots + j] * a.inv_tau - u_max) - log_total;
            const float log_q = w4_load1<BF16>(a.z, row * a.z_stride + at) * a.inv_tau - lse;
            sum += p * (log_p - log_q);
        }
    }
    return a.tau * a.tau * wave_sum(sum);
}

// A workgroup takes a row.
template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_loss_kernel(const DistillArgs a) {
    __shared__ DistillSlots s_slots;
    __shared__ float s_m[THREADS / 64], s_l[THREADS / 64];
    __shared__ int s_any;
    const int64_t row = blockIdx.x;
    const int wave = threadIdx.x >> 6;
    float u_max = 0.0f, log_total = 0.0f;
    if (wave == 0) {
        const bool any = distill_teacher(a, row, s_slots, u_max, log_total);
        if (threadIdx.x == 0) s_any = any;
    }
    __syncthreads();
    if (!s_any) {
        if (threadIdx.x == 0) a.loss[row] = a.lse[row] = 0.0f;
        return;
    }
    float m = kLowest, l = 0.0f;
    const int64_t z0 = row * a.z_stride;
    for (int i = threadIdx.x * 8; i < a.v; i += THREADS * 8) {
        float x[8];
        w4_load8<BF16>(a.z, z0 + i, z0 + a.v, x);
        float top = m;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = i + e < a.v ? x[e] * a.inv_tau : -__builtin_inff();
            top = fmaxf(top, x[e]);
        }
        l *= exp_nat(m - top);
        m = top;
#pragma unroll
        for (int e = 0; e < 8; ++e) l += exp_nat(x[e] - m);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const float m2 = __shfl_xor(m, d), l2 = __shfl_xor(l, d);
        join_ml(m, l, m2, l2);
    }
    if ((threadIdx.x & 63) == 0) { s_m[wave] = m; s_l[wave] = l; }
    __syncthreads();
    if (wave == 0) {
        m = s_m[0], l = s_l[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) join_ml(m, l, s_m[w], s_l[w]);
        const float lse = m + logf(l);
        const float loss = distill_row_loss<BF16>(a, row, s_slots, u_max, log_total, lse);
        if (threadIdx.x == 0) { a.loss[row] = loss; a.lse[row] = lse; }
    }
}

// A workgroup takes `span` logits of a row.
constexpr int kDistillThreads = 256;
template <bool BF16>
__global__ __launch_bounds__(kDistillThreads) void distill_grad_kernel(const DistillArgs a, int span) {
    __shared__ DistillSlots s_slots;
    __shared__ int s_any;
    constexpr int kOwn = kDistillSlots / kDistillThreads;
    const int64_t row = blockIdx.y;
    const int first = blockIdx.x * span, last = min(first + span, a.v);
    const float g = a.grad[row] * a.tau;
    const bool masked = a.grad[row] == 0.0f;
    if (threadIdx.x < 64) {
        float u_max, log_total;
        const bool any = distill_teacher(a, row, s_slots, u_max, log_total);
        if (threadIdx.x == 0) s_any = any;
    }
    __syncthreads();
    const int64_t z0 = row * a.z_stride, o0 = row * a.dz_stride;
    if (!s_any || masked) {
        for (int i = first + threadIdx.x; i < last; i += kDistillThreads) w4_store1<BF16>(a.dz, o0 + i, 0.0f);
        return;
    }
    const float lse = a.lse[row];
    // the slots in this span, each place by the first slot that names it; read before anything is written (dz may be z)
    float fixed[kOwn];
    int place[kOwn];
#pragma unroll
    for (int o = 0; o < kOwn; ++o) {
        const int j = threadIdx.x + o * kDistillThreads;
        place[o] = j < a.slots ? s_slots.at[j] : -1;
        if (place[o] < first || place[o] >= last) place[o] = -1;
        fixed[o] = 0.0f;
        if (place[o] >= 0) {
            float p = 0.0f;
            for (int i = 0; i < a.slots; ++i)
                if (s_slots.at[i] == place[o]) {
                    if (i < j) { place[o] = -1; break; }
                    p += s_slots.p[i];
                }
            if (place[o] >= 0) fixed[o] = g * (exp_nat(w4_load1<BF16>(a.z, z0 + place[o]) * a.inv_tau - lse) - p);
        }
    }
    __syncthreads();
    for (int i = first + threadIdx.x; i < last; i += kDistillThreads)
        w4_store1<BF16>(a.dz, o0 + i, g * exp_nat(w4_load1<BF16>(a.z, z0 + i) * a.inv_tau - lse));
    __syncthreads();
#pragma unroll
    for (int o = 0; o < kOwn; ++o)
        if (place[o] >= 0) w4_store1<BF16>(a.dz, o0 + place[o], fixed[o]);
}

}  // namespace lpmm
