// Tokens drawn from rows of logits (formulas: include/lpmm4.h): a workgroup a row.
//
// A logit's weight exp((z - max) / temperature) is computed in 64 bits and held as a whole number of 2^-46 (fewer bits for more than 2^16
// logits): sums of whole numbers are exact in every order, so a histogram filled by atomics gives equal bits every time, and a token
// next to a border falls on the side that 64 bits put it.
//
// The logits that are kept are always the first ones in the order of falling logits, equal ones by their index: what the k largest, the share p and
// the least probability leave is a last (logit, index) each, and the earliest of them counts.
#pragma once

#include "rows.hpp"

namespace lpmm {

typedef unsigned long long u64;

constexpr int kSampleBins = 2048, kSampleList = 1024, kSampleFew = 128, kSampleLines = kSampleBins / 2;

struct SampleArgs {
    const void* z;
    int64_t z_stride;
    int v;
    int bits;                            // fraction bits of a weight
    float temperature, top_p, min_p;     // of all rows, unless the pointers below are there
    int32_t top_k;
    const float* temperatures;
    const int32_t* top_ks;
    const float* top_ps;
    const float* min_ps;
    const float* u;
    int64_t* tokens;
    float* logprob;
};

// floats in an order that unsigned words keep; -0 as +0
__device__ __forceinline__ uint32_t sample_key(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Sums over the lanes up to each one, by moves within the registers: rows of 16 lanes, then their ends into the rows behind
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 scan_step(u64 x) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, int(uint32_t(x)), CTRL, ROWS, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, int(uint32_t(x >> 32)), CTRL, ROWS, 0xF, false);
    return x + (u64(hi) << 32 | lo);
}
__device__ __forceinline__ u64 wave_scan(u64 x) {
    x = scan_step<0x111, 0xF>(x);
    x = scan_step<0x112, 0xF>(x);
    x = scan_step<0x114, 0xF>(x);
    x = scan_step<0x118, 0xF>(x);
    x = scan_step<0x142, 0xA>(x);
    return scan_step<0x143, 0xC>(x);
}
__device__ __forceinline__ u64 last_lane(u64 x) {
    return u64(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(x >> 32)), 63))) << 32 | uint32_t(__builtin_amdgcn_readlane(int(uint32_t(x)), 63));
}
__device__ __forceinline__ u64 wave_sum(u64 x) { return last_lane(wave_scan(x)); }

// What of a row is kept: logits above `z`, and those equal to it up to index `index`
struct SampleEnd {
    float z;
    int index;
    __device__ __forceinline__ bool keeps(float x, int i) const { return x > z || (x == z && i <= index); }
};

// a b + c with c the same in all lanes: one instruction, where the compiler moves c into the result's registers first
__device__ __forceinline__ double fma_by(double a, double b, double c) {
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(c));
    return r;
}

// 2^bits times 2^y for y <= 0, -infinity included, to a whole number, off by some 2^-47 of 1, the rounding to it: y = n + f with |f| <= 1/2, and 2^f = 1 + f q(f), where q, of the 9th power,
// meets (2^f - 1) / f at the ten points cos((2 i + 1) pi / 20) / 2: within 4.4e-16 of 2^f (the first ten powers of the exponential series are 2.2e-13 off).  The sum with 2^52, which is
// returned, rounds to a whole number in its low bits.
__device__ __forceinline__ double sample_rounded(double y, int bits) {
    y = fmax(y, -100.0);
    const double shifted = y + 0x1.8p52, f = y - (shifted - 0x1.8p52);
    const int n = int(uint32_t(u64(__double_as_longlong(shifted))));
    double p = fma_by(f, 7.0709778665081391e-09, 1.0205905413765595e-07);
    p = fma_by(p, f, 1.3215451633221434e-06);
    p = fma_by(p, f, 1.5252672924850737e-05);
    p = fma_by(p, f, 1.5403530424776529e-04);
    p = fma_by(p, f, 1.3333558200794592e-03);
    p = fma_by(p, f, 9.6181291076186653e-03);
    p = fma_by(p, f, 5.5504108664651669e-02);
    p = fma_by(p, f, 2.4022650695910075e-01);
    p = fma_by(p, f, 6.9314718055994617e-01);
    p = __builtin_fma(p, f, 1.0);
    const double power = __hiloint2double((1023 + bits + n) << 20, 0);
    return fma_by(p, power, 0x1p52);
}
__device__ __forceinline__ u64 sample_low_bits(double rounded) { return u64(__double_as_longlong(rounded)) & 0xFFFFFFFFFFFFFull; }

template <bool BF16, int THREADS>
struct SampleRow {
    static constexpr int E = BF16 ? 8 : 4, kWaves = THREADS / 64, LINE = 64 * E;      // a line: what a wave takes at once
    struct Shared {
        u64 bin[kSampleBins];            // also the sums of the row's pieces, and the sorted list's weights
        uint32_t key[kSampleList];
        int index[kSampleList];
        u64 wave[kWaves];
        float wave_z[kWaves], wave_low[kWaves];
        int wave_i[kWaves];
        u64 found_before;
        uint32_t low, high;              // keys of a bin
        int count, found, bad;
    };

    const SampleArgs& a;
    Shared& s;
    int64_t row0;
    int v;
    float top;                           // largest logit
    double zero;                         // the logit of weight 1: that, or the largest finite number for infinity, from which all other numbers are far
    double c;                            // log2(e) / temperature

    __device__ __forceinline__ float z(int i) const { return w4_load1<BF16>(a.z, row0 + i); }

    // E logits from `first` on.  What lies behind the row's end is -infinity: never kept in front of anything, and without weight.
    __device__ __forceinline__ uint4 piece(int first) const {
        constexpr uint32_t LOW = 0xFF800000u;
        uint32_t out[4];
        if (first + E <= v) {
            if constexpr (BF16) {
                const Vec16 q = *reinterpret_cast<const Vec16*>(static_cast<const uint16_t*>(a.z) + row0 + first);
                return make_uint4(q.v[0], q.v[1], q.v[2], q.v[3]);
            } else {
                const Vec16f q = *reinterpret_cast<const Vec16f*>(static_cast<const float*>(a.z) + row0 + first);
                return make_uint4(__float_as_uint(q.v[0]), __float_as_uint(q.v[1]), __float_as_uint(q.v[2]), __float_as_uint(q.v[3]));
            }
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (BF16) {
                const int i = first + 2 * w;
                const uint32_t lo = i < v ? __float_as_uint(z(i)) : LOW, hi = i + 1 < v ? __float_as_uint(z(i + 1)) : LOW;
                out[w] = lo >> 16 | (hi & 0xFFFF0000u);
            } else {
                out[w] = first + w < v ? __float_as_uint(z(first + w)) : LOW;
            }
        }
        return make_uint4(out[0], out[1], out[2], out[3]);
    }
    static __device__ __forceinline__ void elements(const uint4& q, float x[E]) {
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

    // f(first index, logits of a piece) for this thread's part of the row, by rising index
    template <typename F>
    __device__ __forceinline__ void pieces(F&& f) { pieces(0, v, f); }
    template <typename F>
    __device__ __forceinline__ void pieces(int from, int to, F&& f) {
        for (int64_t first = from + int64_t(threadIdx.x) * E; first < to; first += THREADS * E) {
            float x[E];
            elements(piece(int(first)), x);
            f(int(first), x);
        }
    }
    // f(index, logit)
    template <typename F>
    __device__ __forceinline__ void each(F&& f) {
        pieces([&](int first, const float x[E]) {
#pragma unroll
            for (int e = 0; e < E; ++e) f(first + e, x[e]);
        });
    }

    __device__ __forceinline__ double rounded(float x) const { return sample_rounded((double(x) - zero) * c, a.bits); }                   // of a finite x, or -infinity
    __device__ __forceinline__ u64 weight(float x) const { return sample_low_bits(sample_rounded(fmin((double(x) - zero) * c, 0.0), a.bits)); }

    // Sum over the workgroup, and what the threads before this one have (s.wave is free again after the caller's next barrier)
    __device__ __forceinline__ u64 scan(u64 x, u64& before) {
        const u64 with = wave_scan(x);
        if ((threadIdx.x & 63) == 63) s.wave[threadIdx.x >> 6] = with;
        __syncthreads();
        u64 all = 0, mine = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w == int(threadIdx.x >> 6)) mine = all;
            all += s.wave[w];
        }
        before = mine + with - x;
        return all;
    }

    // The first of bin[0 .. count) at which the running sum reaches target_of(the whole sum), which is from 1 to that sum; the sum in front of it.
    // ALL: count is kSampleBins.
    template <bool ALL, typename Target>
    __device__ __forceinline__ u64 crossing(int count, Target&& target_of, int& at, u64& before, u64& target, const u64* bins = nullptr) {
        const u64* bin = bins ? bins : s.bin;
        constexpr int EACH = kSampleBins / THREADS;
        const int each = ALL ? EACH : (count + THREADS - 1) / THREADS, first = threadIdx.x * each;
        u64 sum = 0;
        if constexpr (ALL) {
#pragma unroll
            for (int j = 0; j < EACH; ++j) sum += bin[first + j];
        } else {
            for (int j = first; j < min(first + each, count); ++j) sum += bin[j];
        }
        u64 ahead;
        const u64 all = scan(sum, ahead);
        target = target_of(all);
        if (ahead < target && ahead + sum >= target) {
            int j = first;
            while (ahead + bin[j] < target) ahead += bin[j++];
            s.found = j;
            s.found_before = ahead;
        }
        __syncthreads();
        at = s.found;
        before = s.found_before;
        return all;
    }

    // The lowest index at which the running sum of weights reaches target_of(the whole sum), which is returned in `all`: the sums of lines first, which a
    // wave takes at once, then of the lanes of the one in question, then its elements.  weights_of(first index, logits, weights) does a piece; false:
    // all of them are 0.
    template <typename Weight, typename Target>
    __device__ __forceinline__ int index_of(Weight&& weights_of, Target&& target_of, u64& all) {
        const int lines = (v + LINE - 1) / LINE, per = (lines + kSampleBins - 1) / kSampleBins, entries = (lines + per - 1) / per;
        const int lane = threadIdx.x & 63;
        for (int p = threadIdx.x >> 6; p < entries; p += kWaves) {
            u64 sum = 0;
            for (int l = p * per; l < min(lines, (p + 1) * per); ++l) sum += line_sum(l, weights_of);
            sum = wave_sum(sum);
            if (lane == 0) s.bin[p] = sum;
        }
        __syncthreads();
        int entry;
        u64 before, target;
        all = crossing<false>(entries, target_of, entry, before, target);
        return index_in(entry * per, min(lines, (entry + 1) * per), before, target, weights_of);
    }
    // this lane's part of a line
    template <typename Weight>
    __device__ __forceinline__ u64 line_sum(int l, Weight&& weights_of) {
        u64 sum = 0;
        const int first = l * LINE + int(threadIdx.x & 63) * E;
        if (first < v) {
            float x[E];
            elements(piece(first), x);
            u64 w[E];
            if (weights_of(first, x, w)) {
#pragma unroll
                for (int e = 0; e < E; ++e) sum += w[e];
            }
        }
        return sum;
    }
    // The index at which the running sum, `before` in front of line l0, reaches `target`, which is within the lines to l1
    template <typename Weight>
    __device__ __forceinline__ int index_in(int l0, int l1, u64 before, u64 target, Weight&& weights_of) {
        if (threadIdx.x < 64) {
            for (int l = l0; l < l1; ++l) {
                const u64 sum = line_sum(l, weights_of), with = wave_scan(sum), line = last_lane(with);
                if (before + line >= target) {
                    u64 ahead = before + with - sum;
                    if (ahead < target && ahead + sum >= target) {
                        const int first = l * LINE + int(threadIdx.x) * E;
                        int found = first;
                        float x[E];
                        elements(piece(first), x);
                        u64 w[E];
                        weights_of(first, x, w);
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            ahead += w[e];
                            if (ahead < target) found = first + e + 1;
                        }
                        s.found = found;
                    }
                    break;
                }
                before += line;
            }
        }
        __syncthreads();
        const int i = s.found;
        __syncthreads();
        return i;
    }

    __device__ __forceinline__ u64 place(int j) const { return u64(s.key[j]) << 32 | ~uint32_t(s.index[j]); }      // larger: further in front
    // Sorts the list by falling key, then rising index: short ones by counting for each what is in front of it, shared by groups of threads (s.bin is overwritten)
    __device__ __forceinline__ void sort(int count) {
        if (count <= kSampleFew) {
            constexpr int PARTS = THREADS / kSampleFew;
            const int i = threadIdx.x % kSampleFew, part = threadIdx.x / kSampleFew;
            const u64 mine = i < count ? place(i) : 0;
            if (part == 0) s.bin[i] = 0;
            __syncthreads();
            if (i < count) {
                u64 front = 0;
                for (int j = part; j < count; j += PARTS) front += place(j) > mine;
                if (front) atomicAdd(&s.bin[i], front);
            }
            __syncthreads();
            if (part == 0 && i < count) s.bin[kSampleFew + s.bin[i]] = mine;
            __syncthreads();
            if (part == 0 && i < count) {
                const u64 x = s.bin[kSampleFew + i];
                s.key[i] = uint32_t(x >> 32);
                s.index[i] = int(~uint32_t(x));
            }
            __syncthreads();
            return;
        }
        int size = 64;
        while (size < count) size *= 2;
        for (int j = count + threadIdx.x; j < size; j += THREADS) {      // behind all: nothing has a lower key and a higher index
            s.key[j] = 0;
            s.index[j] = 0x7FFFFFFF;
        }
        __syncthreads();
        for (int run = 2; run <= size; run *= 2)
            for (int gap = run / 2; gap > 0; gap /= 2) {
                for (int j = threadIdx.x; j < size / 2; j += THREADS) {
                    const int x = (j & ~(gap - 1)) * 2 + (j & (gap - 1)), y = x + gap;
                    const uint32_t kx = s.key[x], ky = s.key[y];
                    const int ix = s.index[x], iy = s.index[y];
                    const bool later = kx < ky || (kx == ky && ix > iy);
                    if (later == ((x & run) == 0)) {
                        s.key[x] = ky; s.key[y] = kx;
                        s.index[x] = iy; s.index[y] = ix;
                    }
                }
                __syncthreads();
            }
    }

    __device__ __forceinline__ void bins_clear() {
        for (int j = threadIdx.x; j < kSampleBins; j += THREADS) s.bin[j] = 0;
        if (threadIdx.x == 0) { s.count = 0; s.low = 0xFFFFFFFFu; s.high = 0; }
        __syncthreads();
    }
    // What is `in` goes into the list, a wave's at once
    __device__ __forceinline__ void enlist(bool in, int i, float x) {
        const u64 lanes = __ballot(in);
        if (lanes == 0) return;
        const int before_me = __builtin_amdgcn_mbcnt_hi(uint32_t(lanes >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(lanes), 0));
        int at = 0;
        if (in && before_me == 0) at = atomicAdd(&s.count, __popcll(lanes));
        at = __builtin_amdgcn_readlane(at, __builtin_ctzll(lanes)) + before_me;
        if (in && at < kSampleList) { s.key[at] = sample_key(x); s.index[at] = i; }
    }

    // Weights of a piece's logits that are kept.  ALL: every one is.  False: none is, in the whole wave.
    template <bool ALL>
    __device__ __forceinline__ bool weights(const SampleEnd& end, int first, const float x[E], u64 w[E]) const {
        if constexpr (ALL) {
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = weight(x[e]);
        } else {
            bool keep[E], any = false;
#pragma unroll
            for (int e = 0; e < E; ++e) any |= keep[e] = end.keeps(x[e], first + e);
            if (!__any(any)) {
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] = 0;
                return false;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const u64 y = weight(x[e]);
                w[e] = keep[e] ? y : 0;
            }
        }
        return true;
    }

    // Where, in the order of falling logits and over what `end` keeps, the running sum of weights (of 1 each, unless WEIGHTS) reaches what target_of
    // makes of the whole sum.  Bins of equal width in z, and as long as the bin in question has too many logits for a list, bins of its keys.
    // ALL: `end` keeps every logit.
    template <bool WEIGHTS, bool ALL, typename Target>
    __device__ __forceinline__ SampleEnd last_of(const SampleEnd& end, float width, Target&& target_of) {
        const float per = kSampleBins / width;
        // what is infinitely far is in the last bin; so is everything where the largest is infinity (a difference of NaN)
        auto coarse = [&](float x) { return int(fminf((top - x) * per, float(kSampleBins - 1))); };
        bins_clear();
        pieces([&](int first, const float x[E]) {
            u64 w[E];
            if constexpr (WEIGHTS) {
                if (!weights<ALL>(end, first, x, w)) return;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) atomicAdd(&s.bin[coarse(x[e])], WEIGHTS ? w[e] : u64(ALL || end.keeps(x[e], first + e)));
        });
        __syncthreads();
        int bin;
        u64 before, target, want;
        crossing<true>(kSampleBins, target_of, bin, before, target);
        u64 ahead = before;
        each([&](int i, float x) { enlist(coarse(x) == bin && (ALL || end.keeps(x, i)), i, x); });
        __syncthreads();
        uint32_t low = 0, high = 0;                                      // keys of the bin
        int shift = -1;
        auto inside = [&](int i, float x) {
            if (shift < 0) return coarse(x) == bin && end.keeps(x, i);
            const uint32_t key = sample_key(x);
            return key >= low && key <= high && end.keeps(x, i);
        };
        while (s.count > kSampleList) {
            __syncthreads();
            uint32_t lowest = 0xFFFFFFFFu, highest = 0;
            each([&](int i, float x) {
                if (!inside(i, x) || (shift >= 0 && int((high - sample_key(x)) >> shift) != bin)) return;
                lowest = min(lowest, sample_key(x));
                highest = max(highest, sample_key(x));
            });
            bins_clear();
            atomicMin(&s.low, lowest);
            atomicMax(&s.high, highest);
            __syncthreads();
            low = s.low;
            high = s.high;
            if (low == high) {
                // many equal ones: as many as it takes, by their index
                const float x = of_key(high);
                const u64 w = WEIGHTS ? weight(x) : 1, need = (target - ahead + w - 1) / w;
                u64 all;
                const int i = index_of([&](int first, const float y[E], u64 out[E]) {
#pragma unroll
                    for (int e = 0; e < E; ++e) out[e] = u64(y[e] == x && end.keeps(y[e], first + e));
                    return true;
                }, [&](u64) { return need; }, all);
                return SampleEnd{x, i};
            }
            shift = 0;
            while (((high - low) >> shift) >= uint32_t(kSampleBins)) ++shift;
            each([&](int i, float x) {
                if (inside(i, x)) atomicAdd(&s.bin[(high - sample_key(x)) >> shift], WEIGHTS ? weight(x) : u64(1));
            });
            __syncthreads();
            const u64 reached = ahead;
            crossing<true>(kSampleBins, [&](u64) { return target - reached; }, bin, before, want);
            ahead += before;
            each([&](int i, float x) { enlist(inside(i, x) && int((high - sample_key(x)) >> shift) == bin, i, x); });
            __syncthreads();
        }
        return end_of_list<WEIGHTS>(s.count, ahead, target);
    }

    // Where, in the order of the list's logits, the running sum from `ahead` on reaches `target`
    template <bool WEIGHTS>
    __device__ __forceinline__ SampleEnd end_of_list(const int count, const u64 ahead, const u64 target) {
        if (count <= kSampleFew) {
            // each logit's predecessors' weights, the comparisons shared by groups of threads
            constexpr int PARTS = THREADS / kSampleFew;
            const int i = threadIdx.x % kSampleFew, part = threadIdx.x / kSampleFew;
            u64* const weight_of = s.bin + kSampleFew;
            if (part == 0 && i < count) {
                s.bin[i] = 0;
                weight_of[i] = WEIGHTS ? weight(of_key(s.key[i])) : 1;
            }
            __syncthreads();
            const u64 mine = i < count ? place(i) : 0;
            if (i < count) {
                u64 sum = 0;
                for (int j = part; j < count; j += PARTS) sum += place(j) > mine ? weight_of[j] : 0;
                if (sum) atomicAdd(&s.bin[i], sum);
            }
            __syncthreads();
            if (part == 0 && i < count) {
                const u64 front = ahead + s.bin[i];
                if (front < target && front + weight_of[i] >= target) s.found = i;
            }
            __syncthreads();
            const SampleEnd found{of_key(s.key[s.found]), s.index[s.found]};
            __syncthreads();
            return found;
        }
        sort(count);
        for (int j = threadIdx.x; j < count; j += THREADS) s.bin[j] = WEIGHTS ? weight(of_key(s.key[j])) : 1;
        __syncthreads();
        int at;
        u64 before, want;
        crossing<false>(count, [&](u64) { return target - ahead; }, at, before, want);
        const SampleEnd found{of_key(s.key[at]), s.index[at]};
        __syncthreads();
        return found;
    }
    static __device__ __forceinline__ float of_key(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

    // Largest logit, with its lowest index if WHERE, and the smallest, if FINITE the smallest finite one, of logits from .. to; false if there is a NaN or nothing
    // above -infinity
    template <bool WHERE, bool FINITE>
    __device__ __forceinline__ bool extremes(int from, int to, int& where, float& least) {
        float best = -__builtin_inff(), low = __builtin_inff();
        int at = 0x7FFFFFFF;
        bool bad = false;
        pieces(from, to, [&](int first, const float x[E]) {
            if constexpr (WHERE) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    bad |= x[e] != x[e];
                    const bool more = x[e] > best;
                    best = more ? x[e] : best;
                    at = more ? first + e : at;
                    low = fminf(low, x[e] == -__builtin_inff() ? low : x[e]);
                }
            } else {
                // a NaN stays
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    best = __builtin_elementwise_maximum(best, x[e]);
                    low = __builtin_elementwise_minimum(low, FINITE && x[e] == -__builtin_inff() ? low : x[e]);
                }
            }
        });
        if constexpr (!WHERE) {
            bad = best != best;
            if (bad) best = low = 0.0f;
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const float x = __shfl_xor(best, m, 64);
            const int i = WHERE ? __shfl_xor(at, m, 64) : 0;
            if (x > best || (x == best && i < at)) { best = x; at = i; }
            low = fminf(low, __shfl_xor(low, m, 64));
        }
        if (threadIdx.x == 0) s.bad = 0;
        __syncthreads();
        if (bad) s.bad = 1;
        if ((threadIdx.x & 63) == 0) {
            s.wave_z[threadIdx.x >> 6] = best;
            s.wave_i[threadIdx.x >> 6] = at;
            s.wave_low[threadIdx.x >> 6] = low;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (s.wave_z[w] > best || (s.wave_z[w] == best && s.wave_i[w] < at)) { best = s.wave_z[w]; at = s.wave_i[w]; }
            low = fminf(low, s.wave_low[w]);
        }
        top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(best)));
        where = at;
        least = low;
        return !s.bad && best > -__builtin_inff();
    }

    struct Options {
        float heat, p, share, u;
        int k;                               // 0: all
    };
    __device__ __forceinline__ Options options(int row) const {
        Options o{a.temperatures ? a.temperatures[row] : a.temperature, a.top_ps ? a.top_ps[row] : a.top_p, a.min_ps ? a.min_ps[row] : a.min_p, a.u[row],
                  a.top_ks ? a.top_ks[row] : a.top_k};
        if (!(o.k > 0 && o.k < v)) o.k = 0;
        if (o.heat == __builtin_inff() && o.share <= 1.0f) o.share = 0.0f;           // all weights are 1: min_p leaves them (and infinity plus heat log(share) would be no border)
        return o;
    }
    // top is known
    __device__ __forceinline__ void measure(const Options& o) {
        c = fmax(1.4426950408889634 / double(o.heat), 1e-300);           // above 0: infinitely far stays so
        zero = top == __builtin_inff() ? 1.7976931348623157e308 : double(top);
    }
    static __device__ __forceinline__ float reach(float top, float least) { return fmaxf(fminf(top - least, 0x1p100f), 0x1p-100f); }
    static __device__ __forceinline__ float reach(float top, float least, float heat) { return fmaxf(fminf(reach(top, least), 28.0f * heat), 0x1p-100f); }
    static __device__ __forceinline__ u64 part_of(float p, u64 all) {
        const double want = ceil(double(p) * double(all));
        return want >= 1.0 ? min(u64(want), all) : u64(1);
    }
    static __device__ __forceinline__ u64 place_of(float u, u64 all) {
        const double at = double(u) * double(all);
        return !(at >= 0.0) ? u64(1) : at < double(all) ? min(u64(at) + 1, all) : all;          // NaN: the first
    }
    // The least logit that min_p leaves, for 0 < share < 1
    __device__ __forceinline__ float least_kept(const Options& o) const {
        const double border = double(top) + double(o.heat) * log(double(o.share));
        const float x = float(border);
        return double(x) < border ? next(x) : x;
    }
    __device__ __forceinline__ void say(int row, int token, float logprob) const {
        a.tokens[row] = token;
        a.logprob[row] = logprob;
    }
    __device__ __forceinline__ void say_drawn(int row, const Options& o, int token, u64 all) const {
        const float x = z(token);
        const double one = __longlong_as_double(int64_t(1023 + a.bits) << 52);
        say(row, token, float((x == top ? 0.0 : (double(x) - double(top)) / double(o.heat)) - log(double(all) / one)));
    }

    // Without top_k, and with min_p below 1: the border of the share p is first looked for in 32 bits, which leaves a range of logits, and one pass in 64 bits
    // gives the whole sum, the sums of what is above that range by lines, and the range's logits as a list.  False: the border is not in the range, or there
    // are too many logits in it.
    __device__ __forceinline__ bool draw_once(int row, const Options& o, float least) {
        const bool some = o.p < 1.0f;
        const float low = o.share > 0.0f ? least_kept(o) : -__builtin_inff();
        float sure = low, from = __builtin_inff();                       // kept: what is not below sure (if the border is in the range); the range: from there down to `from`
        if (some) {
            const float per = kSampleBins / reach(top, least, o.heat), slope = -fminf(float(c), 0x1.FFFFFEp127f);      // finite: the largest's weight is 1
            bins_clear();
            pieces([&](int, const float x[E]) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float below = top - x[e];
                    atomicAdd(&s.bin[int(fminf(below * per, float(kSampleBins - 1)))], u64(uint32_t(__builtin_amdgcn_exp2f(__builtin_fmaf(below, slope, 31.0f)))));
                }
            });
            __syncthreads();
            int bin;
            u64 before, lowest, highest = 0;
            crossing<true>(kSampleBins, [&](u64 all) {
                // these sums are off by some 2^-20 of the whole
                const u64 want = part_of(o.p, all), slack = (all >> 18) + 1;
                highest = min(want + slack, all);
                return want > slack ? want - slack : u64(1);
            }, bin, before, lowest);
            int last = bin;
            for (u64 sum = before + s.bin[bin]; sum < highest && last < kSampleBins - 1; sum += s.bin[last]) ++last;
            // a little more than these bins: a logit of theirs is in the range however the bin's number was rounded
            const float up = top - float(bin) / per * (1.0f - 0x1p-20f);
            if (up >= low) {
                sure = next(up);
                from = last == kSampleBins - 1 ? -__builtin_inff() : top - float(last + 1) / per * (1.0f + 0x1p-20f);
            }
            __syncthreads();
        }
        u64* const line = s.bin + kSampleLines;                          // the bins in front are the list's
        const int lines = (v + LINE - 1) / LINE, per = max(lines > 2 * kWaves ? 2 : 1, (lines + kSampleLines - 1) / kSampleLines), entries = (lines + per - 1) / per;
        const int lane = threadIdx.x & 63;
        if (threadIdx.x == 0) s.count = 0;
        __syncthreads();
        u64 all = 0, above = 0;
        for (int p = threadIdx.x >> 6; p < entries; p += kWaves) {
            u64 sum = 0;
            for (int l = p * per; l < min(lines, (p + 1) * per); ++l) {
                const int at = l * LINE + lane * E;
                float x[E];
                elements(piece(at), x);
                if (!some) {
                    bool any = false;
#pragma unroll
                    for (int e = 0; e < E; ++e) any |= x[e] >= sure;
                    if (!__any(any)) continue;
                    double upper = 0x1p52;
#pragma unroll
                    for (int e = 0; e < E; ++e) upper = __builtin_fma(rounded(x[e]) - 0x1p52, x[e] >= sure ? 1.0 : 0.0, upper);
                    sum += sample_low_bits(upper);
                    continue;
                }
                double every = 0x1p52, upper = 0x1p52;                   // with E weights below 2^53, and exact
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bool in = x[e] >= sure;
                    const double w = rounded(x[e]) - 0x1p52;
                    every += w;
                    upper = __builtin_fma(w, in ? 1.0 : 0.0, upper);
                    enlist(!in && x[e] >= from, at + e, x[e]);
                }
                all += sample_low_bits(every);
                sum += sample_low_bits(upper);
            }
            above += sum;
            sum = wave_sum(sum);
            if (lane == 0) line[p] = sum;
        }
        SampleEnd end{low, 0x7FFFFFFF};
        if (some) {
            u64 ahead;
            all = scan(all, ahead);
            __syncthreads();
            above = scan(above, ahead);
            const u64 target = part_of(o.p, all);
            const int count = s.count;
            if (above >= target) {
                __syncthreads();
                return false;
            }
            if (from < __builtin_inff()) {
                if (count > kSampleList) {
                    __syncthreads();
                    return false;
                }
                u64 sum = 0;
                for (int j = threadIdx.x; j < count; j += THREADS) sum += weight(of_key(s.key[j]));
                __syncthreads();
                sum = scan(sum, ahead);
                __syncthreads();
                if (above + sum < target) return false;
                end = end_of_list<true>(count, above, target);
                for (int j = threadIdx.x; j < count; j += THREADS) {     // the list may have been sorted
                    const float x = of_key(s.key[j]);
                    if (end.keeps(x, s.index[j]) && x >= low) atomicAdd(&line[s.index[j] / (LINE * per)], weight(x));
                }
                if (low > end.z) end = SampleEnd{low, 0x7FFFFFFF};
            }
        }
        __syncthreads();
        int entry;
        u64 before, target;
        all = crossing<false>(entries, [&](u64 sum) { return place_of(o.u, sum); }, entry, before, target, line);
        const int i = index_in(entry * per, min(lines, (entry + 1) * per), before, target, [&](int at, const float x[E], u64 w[E]) { return weights<false>(end, at, x, w); });
        if (threadIdx.x == 0) say_drawn(row, o, i, all);
        return true;
    }

    // With top_k, and with min_p below 1: the list has all logits down to the bin that holds the k-th, `count` of them, and everything else is done in it
    __device__ __forceinline__ void draw_listed(int row, const Options& o, int count) {
        const float low = o.share > 0.0f && o.share < 1.0f ? least_kept(o) : -__builtin_inff();
        int at, n = min(o.k, count);
        u64 before, target;
        sort(count);
        for (int j = threadIdx.x; j < n; j += THREADS) s.bin[j] = weight(of_key(s.key[j]));
        __syncthreads();
        if (o.p < 1.0f) {
            crossing<false>(n, [&](u64 sum) { return part_of(o.p, sum); }, at, before, target);
            n = at + 1;
        }
        // the first of the list stays, and of the others what min_p leaves, by index: behind these what it does not
        __syncthreads();
        for (int j = threadIdx.x; j < n; j += THREADS) s.key[j] = j == 0 || of_key(s.key[j]) >= low ? ~uint32_t(s.index[j]) : 0u;
        __syncthreads();
        sort(n);
        for (int j = threadIdx.x; j < n; j += THREADS) s.bin[j] = s.key[j] ? weight(z(s.index[j])) : 0;
        __syncthreads();
        const u64 all = crossing<false>(n, [&](u64 sum) { return place_of(o.u, sum); }, at, before, target);
        if (threadIdx.x == 0) say_drawn(row, o, s.index[at], all);
    }
    // False: too many logits in that bin
    __device__ __forceinline__ bool draw_first(int row, const Options& o, float least) {
        const float per = kSampleBins / reach(top, least);
        auto coarse = [&](float x) { return int(fminf((top - x) * per, float(kSampleBins - 1))); };
        bins_clear();
        each([&](int, float x) { atomicAdd(&s.bin[coarse(x)], u64(1)); });           // what lies behind the row's end is behind the k-th
        __syncthreads();
        int bin;
        u64 before, target;
        crossing<true>(kSampleBins, [&](u64) { return u64(o.k); }, bin, before, target);
        each([&](int i, float x) { enlist(coarse(x) <= bin && i < v, i, x); });
        __syncthreads();
        const int count = s.count;
        __syncthreads();
        if (count > kSampleList) return false;
        draw_listed(row, o, count);
        return true;
    }

    __device__ __forceinline__ void draw(int row) {
        const Options o = options(row);
        int first;
        float least;
        // the index is for the least of probabilities from 1 up and the temperature 0; top_k needs the smallest finite logit
        const bool simple = !(o.share >= 1.0f) && o.heat > 0.0f;
        if (!(!simple ? extremes<true, true>(0, v, first, least) : o.k ? extremes<false, true>(0, v, first, least) : extremes<false, false>(0, v, first, least))) {
            if (threadIdx.x == 0) say(row, -1, __builtin_nanf(""));
            return;
        }
        if (!(o.heat > 0.0f)) {
            if (threadIdx.x == 0) say(row, first, 0.0f);
            return;
        }
        measure(o);
        if (simple && (o.k ? draw_first(row, o, least) : top < __builtin_inff() && draw_once(row, o, least))) return;
        SampleEnd end{-__builtin_inff(), 0x7FFFFFFF};
        if (o.k) end = last_of<false, true>(end, reach(top, least), [&](u64 all) { return min(u64(o.k), all); });
        if (o.p < 1.0f) {
            const float width = reach(top, least, o.heat);
            auto target = [&](u64 all) { return part_of(o.p, all); };
            end = o.k ? last_of<true, false>(end, width, target) : last_of<true, true>(end, width, target);
        }
        if (o.share >= 1.0f) {
            const SampleEnd e = o.share > 1.0f ? SampleEnd{top, first} : SampleEnd{top, 0x7FFFFFFF};
            if (end.keeps(e.z, e.index)) end = e;
        } else if (o.share > 0.0f) {
            const float x = least_kept(o);
            if (x > end.z) end = SampleEnd{x, 0x7FFFFFFF};
        }
        u64 all;
        const int i = index_of([&](int at, const float x[E], u64 w[E]) { return weights<false>(end, at, x, w); }, [&](u64 sum) { return place_of(o.u, sum); }, all);
        if (threadIdx.x == 0) say_drawn(row, o, i, all);
    }

    static __device__ __forceinline__ float next(float x) {              // the next float up
        if (x == 0.0f) return __uint_as_float(1u);
        const uint32_t b = __float_as_uint(x);
        return __uint_as_float(x > 0.0f ? b + 1 : b - 1);
    }
};

// Bound by the vector units: of 62 instructions for a logit the weight in 64 bits is 25, the sums and comparisons beside it 8, the search in 32 bits 12 and the largest 3
// (the rest is by row), 91 percent of the time; the row is read three times, mostly from behind L2.  2048 x 32000 bf16, top_p 0.98: 130 us from a graph of 20 calls, 1.0 TB/s
// of logits; without top_p 84; with top_k 50 77, 500 143.  (The profiler's kernel time is 151; with two passes in 64 bits, one for the bins of the border and one for the sums, it was 211.)
// 1 x 16000 20 us, by the waits between the steps.  A row
// kept in LDS was 5 percent faster with one row a CU, and 1.4 times slower with many; in registers it spilled.  512 threads are held to 64 registers, so that four workgroups
// run on a CU (151 us without).
template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 512 ? 8 : 1) void sample_kernel(const SampleArgs a) {
    __shared__ typename SampleRow<BF16, THREADS>::Shared s;
    SampleRow<BF16, THREADS> row{a, s, int64_t(blockIdx.x) * a.z_stride, a.v, 0.0f, 0.0, 0.0};
    row.draw(blockIdx.x);
}

// ---- few rows: several workgroups a row -------------------------------------------------------------------------------------------
//
// Three launches, with the whole row read in each (1 x 32000 fp32 23 us, 1 x 131072 bf16 32, 16 x 50257 bf16 30: bound by the waits of the last workgroups, of
// one row 8.5 us for the bins and 10 for the end): the largest logit; the bins, from which the last workgroup of a row to finish finds the one in question; the sums of the lines
// above it and the list of its logits, from which the last one draws.  With top_k the list is of all logits down to the bin.  Lists that are too long, and min_p of 1
// and more, are left to the last workgroup as a whole.

constexpr int kSampleShares = 32, kSampleShareThreads = 256;

struct SampleWork {                      // of a row
    u64 bin[kSampleBins];
    u64 line[kSampleBins];               // sums of 64 pieces
    uint32_t key[kSampleList];
    int index[kSampleList];
    float top[kSampleShares], low[kSampleShares];       // of each workgroup's part
    int at[kSampleShares], bad[kSampleShares];
    u64 before, target;                  // of the bin in question
    int found;                           // that bin
    int count;                           // of the list
    uint32_t tickets[2];                 // workgroups that are done
};

// What other workgroups have written goes past the L2 of an XCD
template <typename T>
__device__ __forceinline__ T far_load(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T>
__device__ __forceinline__ void far_store(T* p, T v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

template <bool BF16>
struct SampleShare : SampleRow<BF16, kSampleShareThreads> {
    typedef SampleRow<BF16, kSampleShareThreads> Row;
    typedef typename Row::Options Options;
    using Row::E;
    using Row::LINE;
    using Row::a;
    using Row::s;
    using Row::v;
    using Row::top;
    static constexpr int T = kSampleShareThreads;
    SampleWork& w;
    int row, part, parts, from, to;      // from: a multiple of LINE

    __device__ __forceinline__ SampleShare(const SampleArgs& args, typename Row::Shared& shared, SampleWork* work, int per)
        : Row{args, shared, int64_t(blockIdx.y) * args.z_stride, args.v, 0.0f, 0.0, 0.0}, w(work[blockIdx.y]), row(blockIdx.y), part(blockIdx.x), parts(gridDim.x),
          from(int(blockIdx.x) * per * LINE), to(min(args.v, from + per * LINE)) {}

    __device__ __forceinline__ void largest() {
        for (int j = part * T + threadIdx.x; j < kSampleBins; j += parts * T) w.bin[j] = 0;
        int at;
        float low;
        Row::template extremes<true, true>(from, to, at, low);
        if (threadIdx.x == 0) {
            w.top[part] = top;
            w.at[part] = at;
            w.low[part] = low;
            w.bad[part] = s.bad;
            if (part == 0) w.count = w.tickets[0] = w.tickets[1] = 0;
        }
    }
    // of the whole row; false: nothing is left to do, workgroup 0 has said so
    __device__ __forceinline__ bool known(const Options& o, int& first, float& least) {
        const int g = min(int(threadIdx.x & (kSampleShares - 1)), parts - 1);
        float best = w.top[g], low = w.low[g];
        int at = w.at[g], bad = w.bad[g];
#pragma unroll
        for (int m = 1; m < kSampleShares; m *= 2) {
            const float x = __shfl_xor(best, m, 64);
            const int i = __shfl_xor(at, m, 64);
            if (x > best || (x == best && i < at)) { best = x; at = i; }
            low = fminf(low, __shfl_xor(low, m, 64));
            bad |= __shfl_xor(bad, m, 64);
        }
        least = low;
        top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(best)));
        first = at;
        if (bad || top == -__builtin_inff() || !(o.heat > 0.0f)) {
            if (part == 0 && threadIdx.x == 0) {
                if (bad || top == -__builtin_inff()) Row::say(row, -1, __builtin_nanf(""));
                else Row::say(row, first, 0.0f);
            }
            return false;
        }
        Row::measure(o);
        return true;
    }
    // True in the row's last workgroup, which then sees what the others have written past the L2 caches: every wave waits until its own writes have arrived there.  (A fence
    // would write back and discard whole caches, once for each wave: 61 x 50257 92 us.)
    __device__ __forceinline__ bool last_one(int which) {
        __builtin_amdgcn_s_waitcnt(0x0070);
        __syncthreads();
        if (threadIdx.x == 0) s.found = __hip_atomic_fetch_add(&w.tickets[which], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == uint32_t(parts - 1);
        __syncthreads();
        const bool last = s.found;
        __syncthreads();
        return last;
    }
    __device__ __forceinline__ float width(const Options& o, float least) const {
        return o.k ? Row::reach(top, least) : Row::reach(top, least, o.heat);
    }
    __device__ __forceinline__ int coarse(float x, float per) const { return int(fminf((top - x) * per, float(kSampleBins - 1))); }

    __device__ __forceinline__ void bins() {
        const Options o = Row::options(row);
        int first;
        float least;
        if (!known(o, first, least) || (!o.k && !(o.p < 1.0f))) return;
        const float per = kSampleBins / width(o, least);
        Row::bins_clear();
        Row::pieces(from, to, [&](int at, const float x[E]) {
            // what lies behind the row's end is behind all of top_k's
#pragma unroll
            for (int e = 0; e < E; ++e) atomicAdd(&s.bin[coarse(x[e], per)], o.k ? u64(1) : Row::weight(x[e]));
        });
        __syncthreads();
        for (int j = threadIdx.x; j < kSampleBins; j += T)
            if (s.bin[j]) __hip_atomic_fetch_add(&w.bin[j], s.bin[j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (!last_one(0)) return;
        for (int j = threadIdx.x; j < kSampleBins; j += T) s.bin[j] = far_load(&w.bin[j]);
        __syncthreads();
        int bin;
        u64 before, target;
        Row::template crossing<true>(kSampleBins, [&](u64 all) { return o.k ? min(u64(o.k), all) : Row::part_of(o.p, all); }, bin, before, target);
        if (threadIdx.x == 0) {
            w.found = bin;
            w.before = before;
            w.target = target;
        }
    }

    __device__ __forceinline__ void finish(u64* s_line) {
        const Options o = Row::options(row);
        int first;
        float least;
        if (!known(o, first, least)) return;
        const bool some = o.k || o.p < 1.0f;
        const float per = kSampleBins / width(o, least), low = o.share > 0.0f && o.share < 1.0f ? Row::least_kept(o) : -__builtin_inff();
        const int bin = some ? w.found : kSampleBins, lane = threadIdx.x & 63;
        if (threadIdx.x == 0) s.count = 0;
        __syncthreads();
        // a wave a line: the sums of what is above the bin
        const int l0 = from / LINE + (threadIdx.x >> 6);
        uint4 next = l0 * LINE + lane * E < to ? Row::piece(l0 * LINE + lane * E) : make_uint4(0, 0, 0, 0);
        for (int l = l0; l * LINE < to; l += T / 64) {
            const int at = l * LINE + lane * E, behind = at + T / 64 * LINE;
            const uint4 now = next;
            if (behind < to) next = Row::piece(behind);
            u64 sum = 0;
            if (at < v) {
                float x[E];
                Row::elements(now, x);
                bool above[E], any = false;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int b = coarse(x[e], per);
                    above[e] = b < bin && x[e] >= low;
                    any |= above[e];
                    if (some) Row::enlist(o.k ? b <= bin && at + e < v : b == bin, at + e, x[e]);
                }
                if (!o.k && __any(any)) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const u64 y = Row::weight(x[e]);
                        sum += above[e] ? y : 0;
                    }
                }
            }
            sum = wave_sum(sum);
            if (lane == 0) far_store(&w.line[l], sum);
        }
        if (some) {
            // this workgroup's list behind the others'
            __syncthreads();
            const int mine = s.count;
            if (threadIdx.x == 0 && mine) s.found = __hip_atomic_fetch_add(&w.count, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            const int behind = mine ? s.found : 0;
            for (int j = threadIdx.x; j < min(mine, kSampleList) && behind + j < kSampleList; j += T) {
                far_store(&w.key[behind + j], s.key[j]);
                far_store(&w.index[behind + j], s.index[j]);
            }
        }
        if (!last_one(1)) return;
        const int count = far_load(&w.count), lines = (v + LINE - 1) / LINE;
        if (count > kSampleList || o.share >= 1.0f) {
            Row::draw(row);
            return;
        }
        for (int j = threadIdx.x; j < count; j += T) {
            s.key[j] = far_load(&w.key[j]);
            s.index[j] = far_load(&w.index[j]);
        }
        __syncthreads();
        if (o.k) {
            Row::draw_listed(row, o, count);
            return;
        }
        SampleEnd end{-__builtin_inff(), 0x7FFFFFFF};
        if (some) end = Row::template end_of_list<true>(count, w.before, w.target);
        for (int j = threadIdx.x; j < lines; j += T) s_line[j] = far_load(&w.line[j]);
        __syncthreads();
        if (some) {
            // end_of_list may have sorted s.key and s.index, together
            for (int j = threadIdx.x; j < count; j += T) {
                const float x = Row::of_key(s.key[j]);
                if (end.keeps(x, s.index[j]) && x >= low) atomicAdd(&s_line[s.index[j] / LINE], Row::weight(x));
            }
            __syncthreads();
        }
        if (low > end.z) end = SampleEnd{low, 0x7FFFFFFF};
        for (int j = threadIdx.x; j < lines; j += T) s.bin[j] = s_line[j];
        __syncthreads();
        int line;
        u64 before, target;
        const u64 all = Row::template crossing<false>(lines, [&](u64 sum) { return Row::place_of(o.u, sum); }, line, before, target);
        if (threadIdx.x < 64) {
            const int at = line * LINE + lane * E;
            u64 y[E], sum = 0;
            if (at < v) {
                float x[E];
                Row::elements(Row::piece(at), x);
                if (Row::template weights<false>(end, at, x, y)) {
#pragma unroll
                    for (int e = 0; e < E; ++e) sum += y[e];
                }
            }
            u64 ahead = before + wave_scan(sum) - sum;
            if (ahead < target && ahead + sum >= target) {
                int found = at;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    ahead += y[e];
                    if (ahead < target) found = at + e + 1;
                }
                Row::say_drawn(row, o, found, all);
            }
        }
    }
};

template <bool BF16>
__global__ __launch_bounds__(kSampleShareThreads) void sample_largest_kernel(const SampleArgs a, SampleWork* work, int per) {
    __shared__ typename SampleShare<BF16>::Row::Shared s;
    SampleShare<BF16>(a, s, work, per).largest();
}
template <bool BF16>
__global__ __launch_bounds__(kSampleShareThreads) void sample_bins_kernel(const SampleArgs a, SampleWork* work, int per) {
    __shared__ typename SampleShare<BF16>::Row::Shared s;
    SampleShare<BF16>(a, s, work, per).bins();
}
template <bool BF16>
__global__ __launch_bounds__(kSampleShareThreads) void sample_finish_kernel(const SampleArgs a, SampleWork* work, int per) {
    __shared__ typename SampleShare<BF16>::Row::Shared s;
    __shared__ u64 s_line[kSampleBins];
    SampleShare<BF16>(a, s, work, per).finish(s_line);
}

}  // namespace lpmm
