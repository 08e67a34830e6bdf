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

constexpr int kSampleBins = 2048, kSampleList = 1024;

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

__device__ __forceinline__ u64 wave_sum(u64 x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m, 64);
    return x;
}
__device__ __forceinline__ u64 wave_scan(u64 x) {                        // with the lane's own
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const u64 y = __shfl_up(x, m, 64);
        if (lane >= m) x += y;
    }
    return x;
}

// What of a row is kept: logits above `z`, and those equal to it up to index `index`
struct SampleEnd {
    float z;
    int index;
    __device__ __forceinline__ bool keeps(float x, int i) const { return x > z || (x == z && i <= index); }
};

template <bool BF16, int THREADS>
struct SampleRow {
    static constexpr int kWaves = THREADS / 64, kBinsEach = kSampleBins / THREADS;
    struct Shared {
        u64 bin[kSampleBins];            // also the sums of the row's pieces, and the sorted list's weights
        uint32_t key[kSampleList];
        int index[kSampleList];
        u64 wave[kWaves];
        float wave_z[kWaves], wave_low[kWaves];
        int wave_i[kWaves];
        u64 found_before, found_self;
        uint32_t low, high;              // keys of a bin
        int count, found, bad;
    };

    const SampleArgs& a;
    Shared& s;
    int64_t row0;
    int v;
    float top;                           // largest logit
    double c;                            // log2(e) / temperature

    __device__ __forceinline__ float z(int i) const { return w4_load1<BF16>(a.z, row0 + i); }

    __device__ __forceinline__ u64 weight(float x) const {
        const double one = __longlong_as_double(int64_t(1023 + a.bits) << 52);
        if (x == top) return u64(one);
        if (x == -__builtin_inff() || top == __builtin_inff()) return 0;
        const double y = (double(x) - double(top)) * c;
        return y > -double(a.bits + 1) ? u64(exp2(y) * one + 0.5) : 0;
    }

    // Sum over the workgroup, and what the threads before this one have
    __device__ __forceinline__ u64 scan(u64 x, u64& before) {
        const u64 with = wave_scan(x);
        if ((threadIdx.x & 63) == 63) s.wave[threadIdx.x >> 6] = with;
        __syncthreads();
        u64 all = 0, mine = 0;
        for (int w = 0; w < kWaves; ++w) {
            if (w == int(threadIdx.x >> 6)) mine = all;
            all += s.wave[w];
        }
        before = mine + with - x;
        __syncthreads();
        return all;
    }

    // The first of s.bin[0 .. count) at which the running sum reaches `target`, and the sum in front of it; `target` is at most the sum of
    // all, which is returned.
    template <typename Target>
    __device__ __forceinline__ u64 crossing(int count, Target&& target_of, int& at, u64& before, u64& target) {
        const int each = (count + THREADS - 1) / THREADS, first = threadIdx.x * each;
        u64 sum = 0;
        for (int j = first; j < min(first + each, count); ++j) sum += s.bin[j];
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
        __syncthreads();
        return all;
    }

    // The lowest index at which the running sum of `weight_of(index)` over the row reaches `target` (at least 1, at most the whole sum)
    template <typename Weight, typename Target>
    __device__ __forceinline__ int index_of(Weight&& weight_of, Target&& target_of, u64& all) {
        constexpr int LINE = 64 * 4;                                     // what a wave takes at once: 4 neighbours a lane
        const int lines = (v + LINE - 1) / LINE, per = (lines + kSampleBins - 1) / kSampleBins, pieces = (lines + per - 1) / per;
        const int lane = threadIdx.x & 63;
        for (int p = threadIdx.x >> 6; p < pieces; p += kWaves) {
            u64 sum = 0;
            for (int l = p * per; l < min(lines, (p + 1) * per); ++l)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = l * LINE + lane * 4 + e;
                    if (i < v) sum += weight_of(i);
                }
            sum = wave_sum(sum);
            if (lane == 0) s.bin[p] = sum;
        }
        __syncthreads();
        int piece;
        u64 before, target;
        all = crossing(pieces, target_of, piece, before, target);
        if (threadIdx.x < 64) {
            for (int l = piece * per; l < min(lines, (piece + 1) * per); ++l) {
                u64 w[4], sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = l * LINE + lane * 4 + e;
                    w[e] = i < v ? weight_of(i) : 0;
                    sum += w[e];
                }
                const u64 with = wave_scan(sum), line = __shfl(with, 63, 64);
                if (before + line >= target) {
                    u64 ahead = before + with - sum;
                    if (ahead < target && ahead + sum >= target) {
                        int e = 0;
                        while (ahead + w[e] < target) ahead += w[e++];
                        s.found = l * LINE + lane * 4 + e;
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
                    const int x = j / gap * 2 * gap + j % gap, y = x + gap;
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

    // Where, in the order of falling logits and over what `end` keeps, the running sum of weights (of 1 each, unless WEIGHTS) reaches what target_of
    // makes of the whole sum.  Bins of equal width in z, and as long as the bin in question has too many logits for a list, bins of its keys.
    template <bool WEIGHTS, typename Target>
    __device__ __forceinline__ SampleEnd last_of(const SampleEnd& end, float width, Target&& target_of) {
        const float per = kSampleBins / width;
        auto coarse = [&](float x) {
            if (x == top) return 0;
            const float d = (top - x) * per;                             // never NaN: `per` is above 0 and x below top
            return d < float(kSampleBins - 1) ? int(d) : kSampleBins - 1;
        };
        auto worth = [&](float x) -> u64 { if constexpr (WEIGHTS) return weight(x); else return 1; };
        u64 ahead = 0, target = 0;
        uint32_t low = 0, high = 0xFFFFFFFFu;                            // keys of the logits in question
        int shift = -1;                                                  // -1: bins of z
        for (;;) {
            for (int j = threadIdx.x; j < kSampleBins; j += THREADS) s.bin[j] = 0;
            if (threadIdx.x == 0) { s.count = 0; s.low = 0xFFFFFFFFu; s.high = 0; }
            __syncthreads();
            for (int i = threadIdx.x; i < v; i += THREADS) {
                const float x = z(i);
                const uint32_t key = sample_key(x);
                if (!end.keeps(x, i) || key < low || key > high) continue;
                const u64 w = worth(x);
                if (w) atomicAdd(&s.bin[shift < 0 ? coarse(x) : int((high - key) >> shift)], w);
            }
            __syncthreads();
            int bin;
            u64 before, want;
            const bool first = shift < 0;
            const u64 reached = ahead;
            crossing(kSampleBins, [&](u64 all) { return first ? target_of(all) : target - reached; }, bin, before, want);
            if (first) target = want;
            ahead += before;
            for (int i = threadIdx.x; i < v; i += THREADS) {
                const float x = z(i);
                const uint32_t key = sample_key(x);
                if (!end.keeps(x, i) || key < low || key > high || (shift < 0 ? coarse(x) : int((high - key) >> shift)) != bin || worth(x) == 0) continue;
                const int at = atomicAdd(&s.count, 1);
                if (at < kSampleList) { s.key[at] = key; s.index[at] = i; }
                atomicMin(&s.low, key);
                atomicMax(&s.high, key);
            }
            __syncthreads();
            const int count = s.count;
            low = s.low;
            high = s.high;
            __syncthreads();
            if (count <= kSampleList) {
                sort(count);
                for (int j = threadIdx.x; j < count; j += THREADS) s.bin[j] = worth(z(s.index[j]));
                __syncthreads();
                int at;
                crossing(count, [&](u64) { return target - ahead; }, at, before, want);
                const int i = s.index[at];
                const SampleEnd found{z(i), i};
                __syncthreads();
                return found;
            }
            if (low == high) break;
            shift = 0;
            while (((high - low) >> shift) >= uint32_t(kSampleBins)) ++shift;
        }
        // many equal ones: as many as it takes, by their index
        const float x = __uint_as_float(high & 0x80000000u ? high & 0x7FFFFFFFu : ~high);
        const u64 w = worth(x);
        const u64 need = (target - ahead + w - 1) / w;
        u64 all;
        const int i = index_of([&](int j) { return u64(z(j) == x && end.keeps(x, j)); }, [&](u64) { return need; }, all);
        return SampleEnd{x, i};
    }

    // Largest logit with its lowest index, smallest finite one; false if there is a NaN or nothing above -infinity
    __device__ __forceinline__ bool extremes(int& where, float& least) {
        float best = -__builtin_inff(), low = __builtin_inff();
        int at = 0x7FFFFFFF;
        bool bad = false;
        for (int i = threadIdx.x; i < v; i += THREADS) {
            const float x = z(i);
            bad |= x != x;
            if (x > best) { best = x; at = i; }
            if (x > -__builtin_inff()) low = fminf(low, x);
        }
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
        for (int w = 0; w < kWaves; ++w) {
            if (s.wave_z[w] > best || (s.wave_z[w] == best && s.wave_i[w] < at)) { best = s.wave_z[w]; at = s.wave_i[w]; }
            low = fminf(low, s.wave_low[w]);
        }
        top = best;
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
        c = 1.4426950408889634 / double(heat);
        SampleEnd end{-__builtin_inff(), 0x7FFFFFFF};
        const float span = fmaxf(fminf(top - least, 0x1p100f), 0x1p-100f);
        if (k > 0 && k < v) end = last_of<false>(end, span, [&](u64 all) { return min(u64(k), all); });
        if (p < 1.0f) {
            const float width = fmaxf(fminf(span, 28.0f * heat), 0x1p-100f);
            end = last_of<true>(end, width, [&](u64 all) {
                const double want = ceil(double(p) * double(all));
                return want >= 1.0 ? min(u64(want), all) : u64(1);
            });
        }
        if (share >= 1.0f) {
            const SampleEnd e = share > 1.0f ? SampleEnd{top, first} : SampleEnd{top, 0x7FFFFFFF};
            if (end.keeps(e.z, e.index)) end = e;
        } else if (share > 0.0f) {
            const double border = double(top) + double(heat) * log(double(share));
            float x = float(border);
            if (double(x) < border) x = sample_after(x);
            if (x > end.z) end = SampleEnd{x, 0x7FFFFFFF};
        }
        u64 all;
        const int i = index_of([&](int j) { const float x = z(j); return end.keeps(x, j) ? weight(x) : u64(0); }, [&](u64 sum) {
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

    static __device__ __forceinline__ float sample_after(float x) {      // the next float up
        if (x == 0.0f) return __uint_as_float(1u);
        const uint32_t b = __float_as_uint(x);
        return __uint_as_float(x > 0.0f ? b + 1 : b - 1);
    }
};

template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_kernel(const SampleArgs a) {
    __shared__ typename SampleRow<BF16, THREADS>::Shared s;
    SampleRow<BF16, THREADS> row{a, s, int64_t(blockIdx.x) * a.z_stride, a.v, 0.0f, 0.0};
    row.draw(blockIdx.x);
}

}  // namespace lpmm
