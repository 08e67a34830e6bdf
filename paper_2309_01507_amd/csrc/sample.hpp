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

constexpr int kSampleBins = 2048, kSampleList = 1024, kSampleFew = 128;

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

// 2^bits times 2^y for y <= 0 to a whole number, to some 2^-47 of 1: y = n + f with |f| <= 1/2, the series of 2^f up to the 11th power (what is
// left is below 7e-15), and the sum with 2^52 rounds to a whole number in its low bits.
__device__ __forceinline__ u64 sample_weight(double y, int bits) {
    y = fmin(fmax(y, -100.0), 0.0);
    const double shifted = y + 0x1.8p52, f = y - (shifted - 0x1.8p52);
    const int n = int(uint32_t(u64(__double_as_longlong(shifted))));
    double p = fma_by(f, 7.0549116208011209e-09, 1.0178086009239699e-07);       // ln(2)^k / k!
    p = fma_by(p, f, 1.3215486790144307e-06);
    p = fma_by(p, f, 1.5252733804059838e-05);
    p = fma_by(p, f, 1.5403530393381606e-04);
    p = fma_by(p, f, 1.3333558146428441e-03);
    p = fma_by(p, f, 9.6181291076284769e-03);
    p = fma_by(p, f, 5.5504108664821576e-02);
    p = fma_by(p, f, 2.4022650695910069e-01);
    p = fma_by(p, f, 6.9314718055994529e-01);
    p = __builtin_fma(p, f, 1.0);
    const double power = __hiloint2double((1023 + bits + n) << 20, 0);
    return u64(__double_as_longlong(fma_by(p, power, 0x1p52))) & 0xFFFFFFFFFFFFFull;
}

template <bool BF16, int THREADS>
struct SampleRow {
    static constexpr int E = BF16 ? 8 : 4, kWaves = THREADS / 64;
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
    __device__ __forceinline__ void pieces(F&& f) {
        for (int64_t first = int64_t(threadIdx.x) * E; first < v; first += THREADS * E) {
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

    __device__ __forceinline__ u64 weight(float x) const { return sample_weight((double(x) - zero) * c, a.bits); }

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

    // The first of s.bin[0 .. count) at which the running sum reaches target_of(the whole sum), which is from 1 to that sum; the sum in front of it.
    // ALL: count is kSampleBins.
    template <bool ALL, typename Target>
    __device__ __forceinline__ u64 crossing(int count, Target&& target_of, int& at, u64& before, u64& target) {
        constexpr int EACH = kSampleBins / THREADS;
        const int each = ALL ? EACH : (count + THREADS - 1) / THREADS, first = threadIdx.x * each;
        u64 sum = 0;
        if constexpr (ALL) {
#pragma unroll
            for (int j = 0; j < EACH; ++j) sum += s.bin[first + j];
        } else {
            for (int j = first; j < min(first + each, count); ++j) sum += s.bin[j];
        }
        u64 ahead;
        const u64 all = scan(sum, ahead);
        target = target_of(all);
        if (ahead < target && ahead + sum >= target) {
            int j = first;
            while (ahead + s.bin[j] < target) ahead += s.bin[j++];
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
        constexpr int LINE = 64 * E;
        const int lines = (v + LINE - 1) / LINE, per = (lines + kSampleBins - 1) / kSampleBins, entries = (lines + per - 1) / per;
        const int lane = threadIdx.x & 63;
        auto line_sum = [&](int l) {
            u64 sum = 0;
            const int first = l * LINE + lane * E;
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
        };
        for (int p = threadIdx.x >> 6; p < entries; p += kWaves) {
            u64 sum = 0;
            for (int l = p * per; l < min(lines, (p + 1) * per); ++l) sum += line_sum(l);
            sum = wave_sum(sum);
            if (lane == 0) s.bin[p] = sum;
        }
        __syncthreads();
        int entry;
        u64 before, target;
        all = crossing<false>(entries, target_of, entry, before, target);
        if (threadIdx.x < 64) {
            for (int l = entry * per; l < min(lines, (entry + 1) * per); ++l) {
                const u64 sum = line_sum(l), with = wave_scan(sum), line = last_lane(with);
                if (before + line >= target) {
                    u64 ahead = before + with - sum;
                    if (ahead < target && ahead + sum >= target) {
                        const int first = l * LINE + lane * E;
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

    // Sorts the list by falling key, then rising index.
    __device__ __forceinline__ void sort(int count) {
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
        const int count = s.count;
        if (count <= kSampleFew) {
            // each logit's predecessors' weights, the comparisons shared by groups of threads
            constexpr int PARTS = THREADS / kSampleFew;
            const int i = threadIdx.x % kSampleFew, part = threadIdx.x / kSampleFew;
            if (part == 0 && i < count) s.bin[i] = 0;
            __syncthreads();
            const uint32_t key = i < count ? s.key[i] : 0u;
            const int index = i < count ? s.index[i] : 0;
            if (i < count) {
                u64 sum = 0;
                for (int j = part; j < count; j += PARTS) {
                    const uint32_t other = s.key[j];
                    if (other > key || (other == key && s.index[j] < index)) sum += WEIGHTS ? weight(of_key(other)) : 1;
                }
                if (sum) atomicAdd(&s.bin[i], sum);
            }
            __syncthreads();
            if (part == 0 && i < count) {
                const u64 front = ahead + s.bin[i];
                if (front < target && front + (WEIGHTS ? weight(of_key(key)) : 1) >= target) s.found = i;
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
        crossing<false>(count, [&](u64) { return target - ahead; }, at, before, want);
        const SampleEnd found{of_key(s.key[at]), s.index[at]};
        __syncthreads();
        return found;
    }
    static __device__ __forceinline__ float of_key(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

    // Largest logit with its lowest index, smallest finite one; false if there is a NaN or nothing above -infinity
    __device__ __forceinline__ bool extremes(int& where, float& least) {
        float best = -__builtin_inff(), low = __builtin_inff();
        int at = 0x7FFFFFFF;
        bool bad = false;
        pieces([&](int first, const float x[E]) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                bad |= x[e] != x[e];
                const bool more = x[e] > best;
                best = more ? x[e] : best;
                at = more ? first + e : at;
                low = fminf(low, x[e] == -__builtin_inff() ? low : x[e]);
            }
        });
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const float x = __shfl_xor(best, m, 64);
            const int i = __shfl_xor(at, m, 64);
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

    __device__ __forceinline__ void draw(int row) {
        const float heat = a.temperatures ? a.temperatures[row] : a.temperature, p = a.top_ps ? a.top_ps[row] : a.top_p;
        const float share = a.min_ps ? a.min_ps[row] : a.min_p, u = a.u[row];
        const int k = a.top_ks ? a.top_ks[row] : a.top_k;
        int first;
        float least;
        if (!extremes(first, least)) {
            if (threadIdx.x == 0) { a.tokens[row] = -1; a.logprob[row] = __builtin_nanf(""); }
            return;
        }
        if (!(heat > 0.0f)) {
            if (threadIdx.x == 0) { a.tokens[row] = first; a.logprob[row] = 0.0f; }
            return;
        }
        c = fmax(1.4426950408889634 / double(heat), 1e-300);             // above 0: infinitely far stays so
        zero = top == __builtin_inff() ? 1.7976931348623157e308 : double(top);
        SampleEnd end{-__builtin_inff(), 0x7FFFFFFF};
        const float span = fmaxf(fminf(top - least, 0x1p100f), 0x1p-100f);
        const bool some = k > 0 && k < v;
        if (some) end = last_of<false, true>(end, span, [&](u64 all) { return min(u64(k), all); });
        if (p < 1.0f) {
            const float width = fmaxf(fminf(span, 28.0f * heat), 0x1p-100f);
            auto share_of = [&](u64 all) {
                const double want = ceil(double(p) * double(all));
                return want >= 1.0 ? min(u64(want), all) : u64(1);
            };
            end = some ? last_of<true, false>(end, width, share_of) : last_of<true, true>(end, width, share_of);
        }
        if (share >= 1.0f) {
            const SampleEnd e = share > 1.0f ? SampleEnd{top, first} : SampleEnd{top, 0x7FFFFFFF};
            if (end.keeps(e.z, e.index)) end = e;
        } else if (share > 0.0f) {
            const double border = double(top) + double(heat) * log(double(share));
            float x = float(border);
            if (double(x) < border) x = next(x);
            if (x > end.z) end = SampleEnd{x, 0x7FFFFFFF};
        }
        u64 all;
        const int i = index_of([&](int at, const float x[E], u64 w[E]) { return weights<false>(end, at, x, w); }, [&](u64 sum) {
            const double at = double(u) * double(sum);
            return !(at >= 0.0) ? u64(1) : at < double(sum) ? min(u64(at) + 1, sum) : sum;          // NaN: the first
        }, all);
        if (threadIdx.x == 0) {
            const float x = z(i);
            const double one = __longlong_as_double(int64_t(1023 + a.bits) << 52);
            a.tokens[row] = i;
            a.logprob[row] = float((x == top ? 0.0 : (double(x) - double(top)) / double(heat)) - log(double(all) / one));
        }
    }

    static __device__ __forceinline__ float next(float x) {              // the next float up
        if (x == 0.0f) return __uint_as_float(1u);
        const uint32_t b = __float_as_uint(x);
        return __uint_as_float(x > 0.0f ? b + 1 : b - 1);
    }
};

// Bound by arithmetic: a logit takes two weights (some 25 instructions in 64 bits each), two bins and an atomic, read four times from L2; with few rows, whose
// workgroups have a CU each, by the waits between its steps (some 12 us).  2048 x 32000 bf16, top_p 0.98: 211 us, 620 GB/s (512 threads; without top_p 105); 1 x 32000
// fp32 35 us; 61 x 50257 bf16 with all options 54.  A row kept in LDS was 5 percent faster with one row a CU, and 1.4 times slower with many; in registers it spilled.
template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_kernel(const SampleArgs a) {
    __shared__ typename SampleRow<BF16, THREADS>::Shared s;
    SampleRow<BF16, THREADS> row{a, s, int64_t(blockIdx.x) * a.z_stride, a.v, 0.0f, 0.0, 0.0};
    row.draw(blockIdx.x);
}

}  // namespace lpmm
