// Distillation from a teacher's top logits: loss and gradient (formulas: include/lpmm4.h).
//
// A pass over a row keeps, per lane and in fp32, the largest logit m and the sum l of exp((z - m) / tau), rescaled when m
// rises, and joins the lanes' pairs at the end.  The gradient is a factor times exp((z - m) / tau) everywhere but at the teacher's
// places, which are written once more behind a barrier.  Bound by reading and writing the logits.
//
// A row is taken in pieces of 16 bytes from its first element on, wherever that lies: gfx950 reads and writes them in one piece at any
// alignment of an element, and so the sums' order, and with it the bits, does not depend on where a row stands.
#pragma once

#include "w4.hpp"

namespace lpmm {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;

struct DistillArgs {
    const void* z;
    int64_t z_stride;
    int64_t t;
    int v, slots;
    const float* top;
    const int64_t* index;
    float tau, inv_tau, c;               // c = log2(e) / tau
    const float* grad;
    float* loss;
    float* lse;
    void* dz;
    int64_t dz_stride;
};

// The teacher's side of a row, in LDS: places (-1 where a slot does not count), probabilities and the student's logits there.
// Sized by the launch, so that short lists leave room for many workgroups.
struct DistillSlots {
    int* at;                             // a multiple of 4 of them
    float* p;
    float* z;
    int* later;                          // an earlier slot names the same place
    int* repeats;                        // [0]: some slot is a later one
};
constexpr int distill_room(int slots) { return (slots + 3) / 4 * 4; }
constexpr size_t distill_lds(int slots) { return size_t(distill_room(slots)) * 16 + 16; }
__device__ __forceinline__ DistillSlots distill_slots(int slots) {
    extern __shared__ __align__(16) int distill_memory[];
    const int room = distill_room(slots);
    return DistillSlots{distill_memory, reinterpret_cast<float*>(distill_memory + room), reinterpret_cast<float*>(distill_memory + 2 * room),
                        distill_memory + 3 * room, distill_memory + 4 * room};
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float ln_fast(float x) { return __builtin_amdgcn_logf(x) * kLn2; }     // of sums in [1, v], 0 or not finite

// (m, l) of two disjoint sets.  m starts at -FLT_MAX rather than -infinity, so that no difference is infinity - infinity
// as long as the logits hold no +infinity.
__device__ __forceinline__ void join_ml(float c, float& m, float& l, float m2, float l2) {
    const float top = fmaxf(m, m2);
    l = l * exp2_fast((m - top) * c) + l2 * exp2_fast((m2 - top) * c);
    m = top;
}
__device__ __forceinline__ void wave_join_ml(float c, float& m, float& l) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) join_ml(c, m, l, __shfl_xor(m, d), __shfl_xor(l, d));
}
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

// ---- pieces of 16 bytes ----------------------------------------------------------------------------------------------------

typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));
template <bool BF16> constexpr int kPiece = BF16 ? 8 : 4;          // elements
constexpr uint32_t kMinusInf = 0xFF800000u;

// elements first .. of a row at p[row0 ..]; beyond v: -infinity
template <bool BF16>
__device__ __forceinline__ Vec16 piece_load(const void* p, int64_t row0, int first, int v) {
    if (first + kPiece<BF16> <= v) {
        if constexpr (BF16) return *reinterpret_cast<const Vec16*>(static_cast<const uint16_t*>(p) + row0 + first);
        else return *reinterpret_cast<const Vec16*>(static_cast<const float*>(p) + row0 + first);
    }
    Vec16 r;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if constexpr (BF16) {
            const uint16_t* x = static_cast<const uint16_t*>(p) + row0;
            const int i = first + 2 * w;
            const uint32_t lo = i < v ? x[i] : kMinusInf >> 16, hi = i + 1 < v ? x[i + 1] : kMinusInf >> 16;
            r.v[w] = lo | hi << 16;
        } else {
            const int i = first + w;
            r.v[w] = i < v ? __float_as_uint(static_cast<const float*>(p)[row0 + i]) : kMinusInf;
        }
    }
    return r;
}
template <bool BF16, bool NT>
__device__ __forceinline__ void piece_store(void* p, int64_t row0, int first, int v, const float x[]) {
    if (first + kPiece<BF16> <= v) {
        Vec16 r;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (BF16) {
                const bf16x2 two = {static_cast<__bf16>(x[2 * w]), static_cast<__bf16>(x[2 * w + 1])};
                r.v[w] = __builtin_bit_cast(uint32_t, two);
            } else {
                r.v[w] = __float_as_uint(x[w]);
            }
        }
        u32x4u* to = reinterpret_cast<u32x4u*>(static_cast<char*>(p) + (row0 + first) * (BF16 ? 2 : 4));
        if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(u32x4u, r), to);
        else *to = __builtin_bit_cast(u32x4u, r);
        return;
    }
#pragma unroll
    for (int e = 0; e < kPiece<BF16>; ++e)
        if (first + e < v) w4_store1<BF16>(p, row0 + first + e, x[e]);
}
template <bool BF16>
__device__ __forceinline__ void piece_values(const Vec16& r, float x[]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if constexpr (BF16) {
            x[2 * w] = __uint_as_float(r.v[w] << 16);
            x[2 * w + 1] = __uint_as_float(r.v[w] & 0xFFFF0000u);
        } else {
            x[w] = __uint_as_float(r.v[w]);
        }
    }
}
// (m, l) with a piece's elements in it
template <bool BF16>
__device__ __forceinline__ void piece_ml(const Vec16& r, float c, float& m, float& l) {
    float x[kPiece<BF16>];
    piece_values<BF16>(r, x);
    float top = m;
#pragma unroll
    for (int e = 0; e < kPiece<BF16>; ++e) top = fmaxf(top, x[e]);
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < kPiece<BF16>; ++e) sum += exp2_fast((x[e] - top) * c);
    l = __builtin_fmaf(l, exp2_fast((m - top) * c), sum);
    m = top;
}

// ---- a row's slots -----------------------------------------------------------------------------------------------------------

// Does any slot count?  Every wave finds out by itself, before anything of the row is read.
__device__ __forceinline__ bool distill_any(const DistillArgs& a, int64_t row) {
    bool any = false;
    for (int j = threadIdx.x & 63; j < a.slots; j += 64) {
        const int64_t i = a.index[row * a.slots + j];
        any = any || (i >= 0 && i < a.v);
    }
    return __ballot(any) != 0;
}

// One wave fills s, and the row's largest top / tau and the logarithm of the sum of its exponentials
template <bool BF16>
__device__ __forceinline__ void distill_teacher(const DistillArgs& a, int64_t row, const DistillSlots& s, float& u_max, float& log_total) {
    const int lane = threadIdx.x & 63;
    float m = -__builtin_inff();
    if (lane == 0) s.repeats[0] = 0;
    if (a.slots + lane < distill_room(a.slots)) s.at[a.slots + lane] = -1;           // read four at a time
    for (int j = lane; j < a.slots; j += 64) {
        const int64_t i = a.index[row * a.slots + j];
        const bool ok = i >= 0 && i < a.v;
        s.later[j] = 0;
        const float u = a.top[row * a.slots + j] * a.inv_tau;
        s.at[j] = ok ? int(i) : -1;
        s.p[j] = u;
        s.z[j] = ok ? w4_load1<BF16>(a.z, row * a.z_stride + i) : 0.0f;
        if (ok) m = fmaxf(m, u);
    }
    u_max = wave_max(m);
    float sum = 0.0f;
    for (int j = lane; j < a.slots; j += 64) {
        const float e = s.at[j] >= 0 ? exp2_fast((s.p[j] - u_max) * kLog2e) : 0.0f;
        s.p[j] = e;
        sum += e;
    }
    sum = wave_sum(sum);
    const float inv = 1.0f / sum;
    for (int j = lane; j < a.slots; j += 64) s.p[j] *= inv;
    log_total = ln_fast(sum);
}

// One wave, the one that filled s: the row's loss.  A logit's log-probability is (z - m) / tau - log_l.
__device__ __forceinline__ float distill_row_loss(const DistillArgs& a, int64_t row, const DistillSlots& s, float u_max,
                                                  float log_total, float m, float log_l) {
    float sum = 0.0f;
    for (int j = threadIdx.x & 63; j < a.slots; j += 64) {
        const float p = s.p[j];
        if (s.at[j] >= 0 && p != 0.0f) {
            const float log_p = (a.top[row * a.slots + j] * a.inv_tau - u_max) - log_total;
            const float log_q = (s.z[j] - m) * a.inv_tau - log_l;
            sum += p * (log_p - log_q);
        }
    }
    return a.tau * a.tau * wave_sum(sum);
}

// Marks the slots whose place an earlier one names, by the whole workgroup: a wave holds 64 slots and looks at 4 others at a time.
template <int THREADS>
__device__ __forceinline__ void distill_repeats(const DistillArgs& a, const DistillSlots& s) {
    const int quads = (a.slots + 3) >> 2, pairs = ((a.slots + 63) >> 6) * quads;
    for (int pair = threadIdx.x >> 6; pair < pairs; pair += THREADS / 64) {
        const int block = pair / quads, i = (pair - block * quads) * 4, j = block * 64 + int(threadIdx.x & 63);
        if (i > block * 64 + 63) continue;
        const int at = j < a.slots ? s.at[j] : -1;
        const int4 other = *reinterpret_cast<const int4*>(&s.at[i]);
        const bool later = (other.x == at && i < j) || (other.y == at && i + 1 < j) || (other.z == at && i + 2 < j) ||
                           (other.w == at && i + 3 < j);
        if (at >= 0 && later) {
            s.later[j] = 1;
            s.repeats[0] = 1;
        }
    }
}
// The p of a place: that of slot j, the first to name it, and of all others that do, in their order
__device__ __forceinline__ float distill_place_p(const DistillArgs& a, const DistillSlots& s, int j) {
    float p = s.p[j];
    if (s.repeats[0])
        for (int i = j + 1; i < a.slots; ++i)
            if (s.at[i] == s.at[j]) p += s.p[i];
    return p;
}

// ---- loss ----------------------------------------------------------------------------------------------------------------------

// (m, l) of the logits [first, last) of a row, by one workgroup; in every lane of wave 0
template <bool BF16, int THREADS>
__device__ __forceinline__ void distill_span_ml(const DistillArgs& a, int64_t row, int first, int last, float* s_m, float* s_l,
                                                float& m, float& l) {
    const int64_t row0 = row * a.z_stride + first;
    const int len = last - first;
    m = kLowest;
    l = 0.0f;
    constexpr int kAhead = 4;
    for (int i = threadIdx.x * kPiece<BF16>; i < len; i += kAhead * THREADS * kPiece<BF16>) {
        Vec16 r[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) r[j] = piece_load<BF16>(a.z, row0, i + j * THREADS * kPiece<BF16>, len);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) piece_ml<BF16>(r[j], a.c, m, l);
    }
    wave_join_ml(a.c, m, l);
    if ((threadIdx.x & 63) == 0) { s_m[threadIdx.x >> 6] = m; s_l[threadIdx.x >> 6] = l; }
    __syncthreads();
    if (threadIdx.x < 64) {
        m = s_m[0], l = s_l[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) join_ml(a.c, m, l, s_m[w], s_l[w]);
    }
}

// A workgroup takes a row: 4096 x 32000 bf16 45 us, 5.8 TB/s; 4096 x 50257, whose rows start off 16-byte boundaries, 89 us, 4.6 TB/s;
// 61 x 32000 fp32, one row each for a quarter of the CUs, 8.0 to 8.4 us.
template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_loss_kernel(const DistillArgs a) {
    const DistillSlots s_slots = distill_slots(a.slots);
    __shared__ float s_m[THREADS / 64], s_l[THREADS / 64];
    const int64_t row = blockIdx.x;
    if (!distill_any(a, row)) {
        if (threadIdx.x == 0) a.loss[row] = a.lse[row] = 0.0f;
        return;
    }
    float u_max = 0.0f, log_total = 0.0f, m, l;
    if (threadIdx.x < 64) distill_teacher<BF16>(a, row, s_slots, u_max, log_total);
    distill_span_ml<BF16, THREADS>(a, row, 0, a.v, s_m, s_l, m, l);
    if (threadIdx.x < 64) {
        const float log_l = ln_fast(l), loss = distill_row_loss(a, row, s_slots, u_max, log_total, m, log_l);
        if (threadIdx.x == 0) { a.loss[row] = loss; a.lse[row] = m * a.inv_tau + log_l; }
    }
}

// Few long rows: a workgroup takes `span` logits of a row and leaves its (m, l); a wave per row joins them.  Bound by the latency of two kernels:
// 16 x 131072 fp32 11.8 us, 0.7 TB/s.
constexpr int kDistillThreads = 256;
template <bool BF16>
__global__ __launch_bounds__(kDistillThreads) void distill_part_kernel(const DistillArgs a, int span, float2* parts) {
    __shared__ float s_m[kDistillThreads / 64], s_l[kDistillThreads / 64];
    const int64_t row = blockIdx.y;
    if (!distill_any(a, row)) return;
    float m, l;
    const int first = blockIdx.x * span;
    distill_span_ml<BF16, kDistillThreads>(a, row, first, min(first + span, a.v), s_m, s_l, m, l);
    if (threadIdx.x == 0) parts[row * gridDim.x + blockIdx.x] = make_float2(m, l);
}
template <bool BF16>
__global__ __launch_bounds__(64) void distill_finish_kernel(const DistillArgs a, const float2* parts, int spans) {
    const DistillSlots s_slots = distill_slots(a.slots);
    const int64_t row = blockIdx.x;
    if (!distill_any(a, row)) {
        if (threadIdx.x == 0) a.loss[row] = a.lse[row] = 0.0f;
        return;
    }
    float u_max, log_total, m = kLowest, l = 0.0f;
    distill_teacher<BF16>(a, row, s_slots, u_max, log_total);
    for (int i = threadIdx.x; i < spans; i += 64) {
        const float2 part = parts[row * spans + i];
        join_ml(a.c, m, l, part.x, part.y);
    }
    wave_join_ml(a.c, m, l);
    const float log_l = ln_fast(l), loss = distill_row_loss(a, row, s_slots, u_max, log_total, m, log_l);
    if (threadIdx.x == 0) { a.loss[row] = loss; a.lse[row] = m * a.inv_tau + log_l; }
}

// ---- gradient ----------------------------------------------------------------------------------------------------------------------

template <bool BF16, int THREADS>
__device__ __forceinline__ void distill_zero(const DistillArgs& a, int64_t row0, int len) {
    const float zero[kPiece<BF16>] = {};
    for (int i = threadIdx.x * kPiece<BF16>; i < len; i += THREADS * kPiece<BF16>) piece_store<BF16, false>(a.dz, row0, i, len, zero);
}

// A row whose lse is so large that its rounding would be seen in exp(z / tau - lse), or takes the sum's logarithm with it as where all logits are the type's
// lowest value: one workgroup sums the row up again and writes all of it.  dz may be z: what another workgroup writes is not read.
constexpr float kLseLarge = 1024.0f;     // half a unit in the last place is 2^-14
template <bool BF16, int THREADS>
__device__ __forceinline__ void distill_grad_row(const DistillArgs& a, int64_t row, const DistillSlots& s_slots, float g) {
    __shared__ float s_m[THREADS / 64], s_l[THREADS / 64];
    constexpr int VEC = kPiece<BF16>;
    const int64_t z0 = row * a.z_stride, o0 = row * a.dz_stride;
    float m, l;
    if (threadIdx.x < 64) distill_teacher<BF16>(a, row, s_slots, m, l);
    distill_span_ml<BF16, THREADS>(a, row, 0, a.v, s_m, s_l, m, l);        // behind its barrier everything has been read
    m = s_m[0], l = s_l[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) join_ml(a.c, m, l, s_m[w], s_l[w]);
    const float f = g / l;
    for (int at = threadIdx.x * VEC; at < a.v; at += THREADS * VEC) {
        float x[VEC];
        piece_values<BF16>(piece_load<BF16>(a.z, z0, at, a.v), x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = f * exp2_fast((x[e] - m) * a.c);
        piece_store<BF16, false>(a.dz, o0, at, a.v, x);
    }
    distill_repeats<THREADS>(a, s_slots);
    __syncthreads();
    for (int j = threadIdx.x; j < a.slots; j += THREADS) {
        const int at = s_slots.at[j];
        if (at >= 0 && !s_slots.later[j])
            w4_store1<BF16>(a.dz, o0 + at, g * (exp2_fast((s_slots.z[j] - m) * a.c) / l - distill_place_p(a, s_slots, j)));
    }
}

// A workgroup takes kGradPieces pieces per thread of a row: 4096 x 32000 bf16, 20 slots, 90 us, 5.8 TB/s; 4096 x 50257, 64 slots, 158 us,
// 5.2 TB/s.
constexpr int kGradPieces = 4;
template <bool BF16, int THREADS> constexpr int kGradSpan = THREADS * kGradPieces * kPiece<BF16>;
template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_grad_kernel(const DistillArgs a) {
    const DistillSlots s_slots = distill_slots(a.slots);
    constexpr int VEC = kPiece<BF16>;
    const int64_t row = blockIdx.y;
    const int first = blockIdx.x * kGradSpan<BF16, THREADS>, last = min(first + kGradSpan<BF16, THREADS>, a.v);
    const int64_t z0 = row * a.z_stride, o0 = row * a.dz_stride;
    const float grad = a.grad[row], g = grad * a.tau, lse = a.lse[row];
    const bool any = distill_any(a, row);
    if (!any || grad == 0.0f) {
        distill_zero<BF16, THREADS>(a, o0 + first, last - first);
        return;
    }
    if (fabsf(lse) >= kLseLarge) {
        if (blockIdx.x == 0) distill_grad_row<BF16, THREADS>(a, row, s_slots, g);
        return;
    }
    Vec16 r[kGradPieces];
#pragma unroll
    for (int j = 0; j < kGradPieces; ++j)
        r[j] = piece_load<BF16>(a.z, z0, first + (j * THREADS + int(threadIdx.x)) * VEC, last);
    if (threadIdx.x < 64) {
        float u_max, log_total;
        distill_teacher<BF16>(a, row, s_slots, u_max, log_total);
    }
    __syncthreads();                     // dz may be z: everything has been read (the slots' logits by the first wave)
#pragma unroll
    for (int j = 0; j < kGradPieces; ++j) {
        const int at = first + (j * THREADS + int(threadIdx.x)) * VEC;
        if (at >= last) break;
        float x[VEC];
        piece_values<BF16>(r[j], x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = g * exp2_fast(__builtin_fmaf(x[e], a.inv_tau, -lse) * kLog2e);
        piece_store<BF16, true>(a.dz, o0, at, last, x);
    }
    distill_repeats<THREADS>(a, s_slots);
    __syncthreads();
    for (int j = threadIdx.x; j < a.slots; j += THREADS) {
        const int at = s_slots.at[j];
        if (at >= first && at < last && !s_slots.later[j])
            w4_store1<BF16>(a.dz, o0 + at, g * (exp2_fast(__builtin_fmaf(s_slots.z[j], a.inv_tau, -lse) * kLog2e) -
                                                distill_place_p(a, s_slots, j)));
    }
}

// ---- both ----------------------------------------------------------------------------------------------------------------------------

// A workgroup takes a row and holds it in registers, ITEMS pieces a thread: one read, one write.  Bound by memory: 4096 x 32000 fp32, 20 slots, 183 us,
// 5.7 TB/s, bf16 105 us, 5.0 TB/s; 4096 x 50257 bf16, 64 slots, 196 to 200 us, 4.1 TB/s (50256: 177; loss, then gradient: 248).  dz goes past the caches but for the
// shortest rows (NT; us past them and through them, 64 slots: 4096 x 57344 bf16 185 and 196, 65536 x 2000 bf16 200 and 179, fp32 330 and 303; 8 slots: 174 and 189,
// 107 and 115, 204 and 210).  The largest shapes spill a few registers: 4 with 25 pieces a thread, 3 to 8 with 16 in 1024 threads.
template <bool BF16, int THREADS, int ITEMS, int WAVES>
__global__ __launch_bounds__(THREADS, WAVES) void distill_both_kernel(const DistillArgs a) {
    constexpr bool NT = THREADS > 64 || (BF16 && ITEMS > 4);
    const DistillSlots s_slots = distill_slots(a.slots);
    __shared__ float s_m[THREADS / 64], s_l[THREADS / 64];
    constexpr int VEC = kPiece<BF16>;
    const int64_t row = blockIdx.x;
    const int64_t z0 = row * a.z_stride, o0 = row * a.dz_stride;
    if (!distill_any(a, row)) {
        distill_zero<BF16, THREADS>(a, o0, a.v);
        if (threadIdx.x == 0) a.loss[row] = a.lse[row] = 0.0f;
        return;
    }
    // a wave takes `items` KiB in a row, so that lines which two of its pieces share stay near
    const int items = (a.v + THREADS * VEC - 1) / (THREADS * VEC);
    const int begin = (int(threadIdx.x >> 6) * items * 64 + int(threadIdx.x & 63)) * VEC, end = min(a.v, begin + items * 64 * VEC);
    Vec16 r[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (begin + j * 64 * VEC < end) r[j] = piece_load<BF16>(a.z, z0, begin + j * 64 * VEC, a.v);
    float u_max = 0.0f, log_total = 0.0f;
    if (threadIdx.x < 64) distill_teacher<BF16>(a, row, s_slots, u_max, log_total);
    float m = kLowest, l = 0.0f;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j)
        if (begin + j * 64 * VEC < end) piece_ml<BF16>(r[j], a.c, m, l);
    wave_join_ml(a.c, m, l);
    if ((threadIdx.x & 63) == 0) { s_m[threadIdx.x >> 6] = m; s_l[threadIdx.x >> 6] = l; }
    __syncthreads();                     // and everything of the row has been read: dz may be z
    m = s_m[0], l = s_l[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) join_ml(a.c, m, l, s_m[w], s_l[w]);
    const float grad = a.grad[row], g = grad * a.tau, f = g / l;
    if (grad == 0.0f) {
        distill_zero<BF16, THREADS>(a, o0, a.v);
    } else {
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            const int at = begin + j * 64 * VEC;
            if (at < end) {
                float x[VEC];
                piece_values<BF16>(r[j], x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[e] = f * exp2_fast((x[e] - m) * a.c);
                piece_store<BF16, NT>(a.dz, o0, at, a.v, x);
            }
        }
    }
    distill_repeats<THREADS>(a, s_slots);
    if (threadIdx.x < 64) {
        const float log_l = ln_fast(l), loss = distill_row_loss(a, row, s_slots, u_max, log_total, m, log_l);
        if (threadIdx.x == 0) { a.loss[row] = loss; a.lse[row] = m * a.inv_tau + log_l; }
    }
    __syncthreads();
    if (grad == 0.0f) return;
    for (int j = threadIdx.x; j < a.slots; j += THREADS) {
        const int at = s_slots.at[j];
        if (at >= 0 && !s_slots.later[j])
            w4_store1<BF16>(a.dz, o0 + at, g * (exp2_fast((s_slots.z[j] - m) * a.c) / l - distill_place_p(a, s_slots, j)));
    }
}

}  // namespace lpmm
